// Attention of new tokens over a paged cache on AMD MI355X (gfx950).
//
// For row i of sequence b at position p and query head h, over the keys and
// values j of the pages that the row may see (j <= p, and j > p - window):
//   o = sum_j softmax_j(scale q . k_j) v_j,   lse = ln sum_j e^(scale q . k_j).
//
// The new rows of one sequence and the Hq / Hkv query heads of one key head
// make one matrix of queries, row r = token * GQ + head, cut into tiles.  Keys
// and values go through LDS once per tile of queries.  Everything is laid out
// transposed, so that softmax needs next to no exchange between lanes:
//  * S^T = K Q^T (v_mfma_f32_32x32x16): A holds 32 keys, B 32 queries, so a
//    query's scores lie in one lane's registers and its neighbour's 32 lanes
//    on; its maximum and sum are taken there.
//  * O^T = V^T P^T: the weights are the B operand as they lie; V comes
//    transposed from LDS (ds_read_b64_tr_b16) in the same order of tokens; a
//    query's output lies in its two lanes, where one factor rescales it.
// The maximum is a running one, kept until a tile exceeds it by 2^8, and
// weights are 2^(s - m + 6): at most 2^14, and the float16 subnormals, which
// lose bits, begin 2^-20 below the maximum.  Weights are rounded to the
// pages' type (their sum is of the unrounded ones), all sums are float32.
#include <algorithm>

#include "gsrq_paged.h"

namespace {

constexpr int PT_THREADS = 256;
constexpr int PT_WAVES = PT_THREADS / 64;
constexpr int PT_ROWS = 32 * PT_WAVES;     // queries per workgroup
constexpr float PT_HEADROOM = 8.f;         // log2 by which a tile may exceed the maximum in use
constexpr float PT_SHIFT = 6.f;            // log2 of the largest weight at a fresh maximum

typedef __attribute__((address_space(3))) char lds_char;
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));

template <typename T> struct Vec;
template <> struct Vec<_Float16> {
  typedef h8 v8;
  typedef h4 v4;
  static __device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ h4 read_tr(lds_char* p) {
    typedef __fp16 fp16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4f16(
                                      (__attribute__((address_space(3))) fp16x4*)p));
  }
};
template <> struct Vec<__bf16> {
  typedef b8 v8;
  typedef b4 v4;
  static __device__ __forceinline__ f16v mfma(b8 a, b8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ b4 read_tr(lds_char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) b4*)p);
  }
};

struct PtArgs {
  PagePool pool;
  const void* q;
  int64_t qst[2];                 // token, head
  void* out;
  float* lse;                     // or null
  const int32_t *q_start, *seq_len;
  float* part;                    // [row][split][HD] unscaled sums, then [row][split][2]
  float* part_ml;
  int T, Hq, GQ, ns, window, slots;
  float c;                        // scale * log2(e)
};

// What a tile of queries reads: keys lo .. hi - 1, in `parts` pieces of
// `step` keys.
struct Span {
  int lo, hi, step, parts;
};

// Sequence b's lengths: new rows [first, first + n), keys [0, keys), and the
// position of its first new row.
struct Seq {
  int first, n, keys;
  int64_t pos0;
};

__device__ __forceinline__ Seq sequence(const PtArgs& a, int b) {
  Seq s;
  new_rows(a.q_start, b, a.T, s.first, s.n);
  const int len = a.seq_len[b];
  const int64_t cap = (int64_t)a.pool.per << a.pool.shift;
  s.keys = len < 0 ? 0 : (len < cap ? len : (int)cap);
  s.pos0 = (int64_t)len - s.n;
  return s;
}

// Queries r0 .. r0 + rows - 1 of a sequence, keys cut at multiples of `unit`
// into at most ns pieces.
__device__ __forceinline__ Span span_of(const PtArgs& a, const Seq& s, int r0, int rows, int unit,
                                        int ns) {
  const int64_t most = (int64_t)s.n * a.GQ - 1;
  const int64_t last = r0 + rows - 1 < most ? r0 + rows - 1 : most;
  const int64_t top = s.pos0 + last / a.GQ + 1;
  const int64_t bottom = a.window ? s.pos0 + r0 / a.GQ - a.window + 1 : 0;
  Span w;
  w.hi = (int)(top < s.keys ? top : s.keys);
  w.lo = bottom > 0 ? (int)(bottom < s.keys ? bottom : s.keys) / unit * unit : 0;
  const int units = w.hi > w.lo ? (w.hi - w.lo + unit - 1) / unit : 0;
  const int per = (units + ns - 1) / ns;
  w.step = per * unit;
  w.parts = units ? (units + per - 1) / per : 1;
  return w;
}

// Tile slot of a launch: sequence b owns the slots from its first row's tile
// number on, one more than it can need at most.
__device__ __forceinline__ int64_t slot_of(const PtArgs& a, int b) {
  const int q = a.q_start[b];
  return (int64_t)(q < 0 ? 0 : (q > a.T ? a.T : q)) * a.GQ / PT_ROWS + b;
}

// The two halves of a wave: a lane's value and that of the lane 32 on.
__device__ __forceinline__ float2 both_halves(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return make_float2(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// Places of a tile's 16-byte chunk c of row r in LDS: rows of a key tile are
// read 32 at a time at one chunk, rows of a value tile four at a time at four
// chunks, both without bank conflicts in these orders.
template <int HD> __device__ __forceinline__ int key_at(int r, int c) {
  return r * (HD * 2) + ((c ^ (HD == 64 ? (r >> 1) & 7 : r & 15)) << 4);
}
template <int HD> __device__ __forceinline__ int value_at(int r, int c) {
  return r * (HD * 2) + ((c ^ (4 * (HD == 64 ? (r >> 1) & 1 : r & 3))) << 4);
}

template <typename T, int HD> struct PtCfg {
  static constexpr int TN = HD == 256 ? 32 : 64;       // keys per tile
  static constexpr int CH = HD / 8;                    // 16-byte chunks per row
  static constexpr int BYTES = TN * HD * 2;
  static constexpr int PER = TN * CH / PT_THREADS;     // chunks per thread
};

// One workgroup per (tile of 128 queries, key head, piece of the keys), 32
// queries a wave.
template <typename T, int HD>
__global__ void __launch_bounds__(PT_THREADS, HD == 256 ? 1 : 2) paged_attn_tile_kernel(PtArgs a) {
  typedef PtCfg<T, HD> C;
  typedef typename Vec<T>::v8 v8;
  typedef typename Vec<T>::v4 v4;
  constexpr int NB = C::TN / 32, KS = HD / 16, DT = HD / 32;
  __shared__ __align__(16) char lds[2 * C::BYTES];
  char* kt = lds;
  char* vt = lds + C::BYTES;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int head = blockIdx.x % a.pool.Hkv;
  int rest = blockIdx.x / a.pool.Hkv;
  const int part = rest % a.ns;
  const int slot = a.slots - 1 - rest / a.ns;          // a prompt's longest rows first
  int b = 0;
  for (int i = 0; i < a.pool.B; i += 64) {
    const bool done = i + lane < a.pool.B && slot_of(a, i + lane + 1) <= slot;
    b += (int)__popcll(__ballot(done));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  if (b >= a.pool.B) return;
  const Seq s = sequence(a, b);
  const int64_t tile = slot - slot_of(a, b);
  if (tile < 0 || tile * PT_ROWS >= (int64_t)s.n * a.GQ) return;
  const int r0 = (int)tile * PT_ROWS;
  const Span w = span_of(a, s, r0, PT_ROWS, C::TN, a.ns);
  if (part >= w.parts) return;
  const int begin = w.lo + part * w.step;
  const int end = min(w.hi, begin + w.step);

  // this lane's query
  const int r = r0 + 32 * wave + col;
  const bool real = r < s.n * a.GQ;
  const int tok = real ? r / a.GQ : 0, g = real ? r - tok * a.GQ : 0;
  const int64_t pos = s.pos0 + tok;
  const int see_hi = real ? (int)(pos + 1 < s.keys ? (pos + 1 > 0 ? pos + 1 : 0) : s.keys) : 0;
  const int64_t from = a.window ? pos - a.window + 1 : 0;
  const int see_lo = from > 0 ? (int)(from < s.keys ? from : s.keys) : 0;
  v8 qf[KS];
  {
    const T* qp = (const T*)a.q + (int64_t)(s.first + tok) * a.qst[0] +
                  (int64_t)(head * a.GQ + g) * a.qst[1] + 8 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *(const v8*)(qp + 16 * k);
  }
  // keys that every query of the wave sees: no mask between these
  int all_hi = see_hi, all_lo = see_lo;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    all_hi = min(all_hi, __shfl_xor(all_hi, m));
    all_lo = max(all_lo, __shfl_xor(all_lo, m));
  }
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);

  f16v o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float m = -INFINITY, l = 0.f;                        // of the scaled scores, log2

  for (int t0 = begin; t0 < end; t0 += C::TN) {
    // the pages of the tile's tokens, one a lane
    const int mine = t0 + (lane & (C::TN - 1));
    const int page = mine < end ? page_of(a.pool, b, mine) : -1;
    const uint64_t absent = __ballot(page < 0);
    __syncthreads();                                   // the last tile has been read
#pragma unroll
    for (int u = 0; u < C::PER; ++u) {
      const int i = u * PT_THREADS + tid, row = i / C::CH, ch = i % C::CH;
      const int pg = __shfl(page, row);
      u4 kx = {0u, 0u, 0u, 0u}, vx = {0u, 0u, 0u, 0u};
      if (pg >= 0) {
        const int64_t in = (t0 + row) & ((1 << a.pool.shift) - 1);
        kx = *(const u4*)((const T*)a.pool.k + pg * a.pool.ks[0] + in * a.pool.ks[1] +
                          head * a.pool.ks[2] + 8 * ch);
        vx = *(const u4*)((const T*)a.pool.v + pg * a.pool.vs[0] + in * a.pool.vs[1] +
                          head * a.pool.vs[2] + 8 * ch);
      }
      *(u4*)(kt + key_at<HD>(row, ch)) = kx;
      *(u4*)(vt + value_at<HD>(row, ch)) = vx;
    }
    __syncthreads();
    f16v sc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const v8 kf = *(const v8*)(kt + key_at<HD>(32 * n + col, 2 * k + half));
        sc[n] = Vec<T>::mfma(kf, qf[k], sc[n]);
      }
    }
    if (absent || t0 + C::TN > all_hi || t0 < all_lo) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = 32 * n + 8 * (i / 4) + 4 * half + i % 4, j = t0 + row;
          const bool seen = j < see_hi && j >= see_lo && !((absent >> row) & 1);
          sc[n][i] = seen ? sc[n][i] : -INFINITY;
        }
    }
    float top = sc[0][0];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[n][i]);
    const float2 tops = both_halves(top);
    top = fmaxf(tops.x, tops.y) * a.c;
    if (__any(top > m + PT_HEADROOM)) {
      const float now = fmaxf(m, top);
      // a query that has seen nothing keeps -inf, and a factor of its own
      const float f = now == -INFINITY ? 1.f : exp2f(m - now);
      m = now;
      l *= f;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= f;
    }
    const float sub = m == -INFINITY ? 0.f : PT_SHIFT - m;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[n][i] = __builtin_amdgcn_exp2f(fmaf(sc[n][i], a.c, sub));
        l += sc[n][i];
      }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (T)sc[n][8 * k + e];
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const int row = 32 * n + 16 * k + 4 * half + ((lane & 15) >> 2);
          const int ch = 4 * t + ((lane >> 3) & 2) + ((lane & 3) >> 1);
          const v4 lo = Vec<T>::read_tr((lds_char*)(vt + value_at<HD>(row, ch) + 8 * (lane & 1)));
          const v4 hi = Vec<T>::read_tr((lds_char*)(vt + value_at<HD>(row + 8, ch) + 8 * (lane & 1)));
          const v8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          o[t] = Vec<T>::mfma(vf, p, o[t]);
        }
      }
  }

  const float2 ls = both_halves(l);
  l = ls.x + ls.y;
  if (!real) return;
  const float base = m == -INFINITY ? m : m - PT_SHIFT;
  const int64_t orow = (int64_t)(s.first + tok) * a.Hq + head * a.GQ + g;
  if (w.parts == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* dst = (T*)a.out + orow * HD + 4 * half;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (T)(o[t][4 * i + e] * inv);
        *(v4*)(dst + 32 * t + 8 * i) = x;
      }
    if (a.lse && half == 0)
      a.lse[orow] = l == 0.f ? -INFINITY : (base + log2f(l)) * 0.69314718055994531f;
  } else {
    float* dst = a.part + (orow * a.ns + part) * HD + 4 * half;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f4*)(dst + 32 * t + 8 * i) =
            (f4){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
    if (half == 0) {
      a.part_ml[2 * (orow * a.ns + part)] = base;
      a.part_ml[2 * (orow * a.ns + part) + 1] = l;
    }
  }
}

// Joins the pieces of every row whose keys were cut: one wave per (row, head).
template <typename T, int HD>
__global__ void __launch_bounds__(256) paged_attn_merge_kernel(PtArgs a) {
  constexpr int E = HD / 64;
  const int64_t orow = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (orow >= (int64_t)a.T * a.Hq) return;
  const int row = (int)(orow / a.Hq), head = (int)(orow % a.Hq);
  const int b = sequence_of(a.q_start, a.pool.B, row);
  if (b < 0) return;
  const Seq s = sequence(a, b);
  const int r = (row - s.first) * a.GQ + head % a.GQ;
  const Span w = span_of(a, s, r / PT_ROWS * PT_ROWS, PT_ROWS, PtCfg<T, HD>::TN, a.ns);
  if (w.parts < 2) return;
  const float* ml = a.part_ml + 2 * orow * a.ns;
  float top = -INFINITY;
  for (int i = 0; i < w.parts; ++i) top = fmaxf(top, ml[2 * i]);
  float l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i = 0; i < w.parts; ++i) {
    const float f = ml[2 * i] == -INFINITY ? 0.f : exp2f(ml[2 * i] - top);
    const float* p = a.part + (orow * a.ns + i) * HD + lane * E;
    l += f * ml[2 * i + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += f * p[e];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) ((T*)a.out)[orow * HD + lane * E + e] = (T)(o[e] * inv);
  if (a.lse && lane == 0)
    a.lse[orow] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
}

// --------------------------------------------------------------- host side

struct PtPlan {
  PagePool pool;
  int64_t slots;
  int ns;
  size_t off_ml, bytes;
};

gsrq_status pt_plan(const gsrq_paged_attn* s, const gsrq_pages* pages, PtPlan& p) {
  gsrq_status e = page_pool(pages, p.pool);
  if (e) return e;
  if (!s || s->T < 1 || s->Hq < 1 || s->Hq % pages->Hkv || s->window < 0 || s->flags)
    return GSRQ_E_ARG;
  if (!(s->scale > 0.f) || !(s->scale < INFINITY)) return GSRQ_E_ARG;
  const int64_t GQ = s->Hq / pages->Hkv;
  if (s->T * GQ > INT32_MAX / 2 || pages->B > (1 << 20)) return GSRQ_E_UNSUPPORTED;
  p.slots = s->T * GQ / PT_ROWS + pages->B;
  // keys are cut until the launch has two workgroups per CU, into pieces of
  // 512 at the least
  const int64_t wgs = p.slots * pages->Hkv, cap = (int64_t)pages->per * pages->page_size;
  int64_t ns = std::min<int64_t>((512 + wgs - 1) / wgs, (cap + 511) / 512);
  if (ns < 1) ns = 1;
  p.ns = (int)ns;
  if (wgs * ns > MAX_BLOCKS || (s->T * s->Hq + 3) / 4 > MAX_BLOCKS) return GSRQ_E_UNSUPPORTED;
  const size_t rows = ns > 1 ? (size_t)(s->T * s->Hq * ns) : 0;
  p.off_ml = align256(rows * pages->head_dim * sizeof(float));
  p.bytes = p.off_ml + align256(rows * 2 * sizeof(float));
  return GSRQ_OK;
}

template <typename T, int HD> gsrq_status pt_launch(const PtArgs& a, hipStream_t st) {
  TimedLaunch tl(GSRQ_KERNEL_ATTENTION, st);
  const unsigned blocks = (unsigned)a.slots * a.ns * a.pool.Hkv;
  paged_attn_tile_kernel<T, HD><<<blocks, PT_THREADS, 0, st>>>(a);
  gsrq_status e = launch_ok();
  if (e || a.ns == 1) return e;
  paged_attn_merge_kernel<T, HD><<<(unsigned)(((int64_t)a.T * a.Hq + 3) / 4), 256, 0, st>>>(a);
  return launch_ok();
}

}  // namespace

extern "C" {

gsrq_status gsrq_attn_paged_workspace_bytes(const gsrq_paged_attn* s, const gsrq_pages* pages,
                                            size_t* bytes) {
  if (!bytes) return GSRQ_E_ARG;
  PtPlan p;
  gsrq_status e = pt_plan(s, pages, p);
  if (e) return e;
  *bytes = p.bytes;
  return GSRQ_OK;
}

gsrq_status gsrq_attn_paged(const gsrq_paged_attn* s, const gsrq_pages* pages,
                            const int32_t* q_start, const int32_t* seq_len, const gsrq_heads* q,
                            void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  PtPlan p;
  gsrq_status e = pt_plan(s, pages, p);
  if (e) return e;
  if (!q_start || !seq_len || !out || (uintptr_t)out % 16) return GSRQ_E_ARG;
  if ((e = head_rows(q, 2))) return e;
  if (p.bytes && (!workspace || (uintptr_t)workspace % 256)) return GSRQ_E_ARG;
  if (ws_bytes < p.bytes) return GSRQ_E_WORKSPACE;
  PtArgs a;
  a.pool = p.pool;
  a.q = q->data;
  a.qst[0] = q->token_stride;
  a.qst[1] = q->head_stride;
  a.out = out;
  a.lse = lse;
  a.q_start = q_start;
  a.seq_len = seq_len;
  a.part = (float*)workspace;
  a.part_ml = p.bytes ? (float*)((char*)workspace + p.off_ml) : nullptr;
  a.T = (int)s->T;
  a.Hq = s->Hq;
  a.GQ = s->Hq / pages->Hkv;
  a.ns = p.ns;
  a.window = s->window;
  a.slots = (int)p.slots;
  a.c = (float)((double)s->scale * 1.4426950408889634);
  hipStream_t st = (hipStream_t)stream;
  const int hd = pages->head_dim;
  if (pages->dtype == GSRQ_F16) {
    if (hd == 64) return pt_launch<_Float16, 64>(a, st);
    if (hd == 128) return pt_launch<_Float16, 128>(a, st);
    return pt_launch<_Float16, 256>(a, st);
  }
  if (hd == 64) return pt_launch<__bf16, 64>(a, st);
  if (hd == 128) return pt_launch<__bf16, 128>(a, st);
  return pt_launch<__bf16, 256>(a, st);
}

}  // extern "C"
