// Attention of new tokens over a paged cache on AMD MI355X (gfx950).
//
// For row i of sequence b at position p and query head h, over the keys and
// values j of the pages that the row may see (j <= p, and j > p - window):
//   o = sum_j softmax_j(scale q . k_j) v_j,   lse = ln sum_j e^(scale q . k_j).
//
// The new rows of one sequence and the GQ = Hq / Hkv query heads of one key
// head make one matrix of queries, row r = token * GQ + head.  One launch holds
// two kinds of workgroups:
//  * few: a sequence with at most 32 queries per key head (a decoding step, a
//    few drafts).  Its cost is reading keys and values once, so its keys are
//    cut into pieces, and each of a workgroup's four waves streams tiles of
//    32 keys of its own, without a barrier.
//  * many: 128 queries, 32 a wave; tiles of 64 keys go through LDS for all
//    four waves.  Keys are cut too where the queries alone do not fill the GPU.
// A second launch joins the pieces.  In both kinds everything is laid out
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
// pages' type for the product alone (their own sum, which is also a result,
// is of the unrounded ones); all sums are float32.  A weight that comes to zero
// makes NaN of an infinite value: such sums are looked through again at the
// end (a check of the sums, 0.2 to 0.5 us a call).
#include "gsrq_attn_paged.h"

namespace {

// 128 queries of one sequence and key head, 32 a wave, and a piece of the keys.
template <typename T, int HD>
__device__ __forceinline__ void many(const PtArgs& a, char* lds, int block) {
  typedef PtCfg<HD> C;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = block % a.pool.Hkv;
  const int rest = block / a.pool.Hkv;
  const int part = rest % a.ns_many;
  const int slot = a.slots - 1 - rest / a.ns_many;     // a prompt's longest rows first
  int b = 0;
  for (int i = 0; i < a.pool.B; i += 64) {
    const bool done = i + lane < a.pool.B && slot_of(a, i + lane + 1) <= slot;
    b += (int)__popcll(__ballot(done));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  if (b >= a.pool.B) return;
  const Seq s = sequence(a, b);
  const int64_t tile = slot - slot_of(a, b);
  if (is_few(a, s) || tile < 0 || tile * PT_ROWS >= (int64_t)s.n * a.GQ) return;
  const int r0 = (int)tile * PT_ROWS;
  const Span w = span_of(a, s, r0, PT_ROWS, C::TN, a.ns_many);
  if (part >= w.parts) return;
  const int begin = w.lo + part * w.step;
  const int end = min(w.hi, begin + w.step);
  // keys that every query of the workgroup sees
  const int64_t first = s.pos0 + r0 / a.GQ;
  const int64_t last = s.pos0 + (min(r0 + PT_ROWS, s.n * a.GQ) - 1) / a.GQ;
  const int64_t wg_hi = min((int64_t)s.keys, first + 1);
  const int64_t wg_lo = a.window ? last - a.window + 1 : 0;

  const int r = r0 + 32 * wave + (lane & 31);
  Columns<T, HD> c;
  c.start(a, s, head, r);
  int* odd_tiles = (int*)(lds + 4 * C::BYTES);         // first and last tile with infinities or NaN
  if (tid == 0) {
    odd_tiles[0] = INT32_MAX;
    odd_tiles[1] = -1;
  }

  // a tile's keys or values to LDS, pages found one a lane; a wave's load fills
  // 1 KiB
  constexpr int NB = C::TN / 32, RL = 64 / C::CH;      // RL: rows of one load
  const int lrow = lane / C::CH, lch = lane % C::CH;
  const char* const kbase = a.pool.k + sizeof(T) * head * a.pool.ks[2];
  const char* const vbase = a.pool.v + sizeof(T) * head * a.pool.vs[2];
  auto fetch = [&](bool key, int t0, int page, const char* at) __attribute__((always_inline)) {
    const int64_t (&st)[3] = key ? a.pool.ks : a.pool.vs;
    const uint64_t offset = token_offset(a.pool, st, page, t0 + (lane & (C::TN - 1)));
#pragma unroll
    for (int u = 0; u < C::PER; ++u) {
      const int row = (u * PT_WAVES + wave) * RL;
      const int ch = key ? key_chunk<HD>(row + lrow, lch) : value_chunk<HD>(row + lrow, lch);
      load_to_lds(rows_at(key ? kbase : vbase, offset, row),
                  2 * (lrow * (uint32_t)st[1] + 8 * ch),
                  lds_offset(at) + 1024 * (u * PT_WAVES + wave));
    }
  };
  const int mine = lane & (C::TN - 1);
  auto page_at = [&](int t0, int entry) __attribute__((always_inline)) {
    return t0 + mine < end ? checked(a.pool, entry) : -1;
  };
  // Keys run one tile ahead of values: while a tile's weights are taken and its
  // values added, the next one's scores are formed, so that the matrix unit
  // works through the exponentials.
  char* const kt = lds;
  char* const vt = lds + 2 * C::BYTES;
  int page = page_at(begin, entry_of(a.pool, b, begin + mine));
  int next = page_at(begin + C::TN, entry_of(a.pool, b, begin + C::TN + mine));
  uint64_t absent = __ballot(page < 0), next_absent = __ballot(next < 0);
  fetch(true, begin, page, kt);
  wait_loads<0>();
  __syncthreads();                                     // (odd_tiles, too)
  if (begin < end) {                                   // (none that nothing waits for)
    fetch(false, begin, page, vt);
    fetch(true, begin + C::TN, next, kt + C::BYTES);
  }
  int entry = entry_of(a.pool, b, begin + 2 * C::TN + mine);
  f16v even_scores[NB], odd_scores[NB];
  c.template scores<NB>(kt, even_scores);
  c.template settle<NB>(a, begin, absent, even_scores);
  auto step = [&](int t0, int odd, f16v (&sc)[NB], f16v (&ahead)[NB])
                  __attribute__((always_inline)) {
    char* const v = vt + odd * C::BYTES;
    wait_loads<0>();                                   // values of t0, keys of the next
    if (absent || t0 + C::TN > wg_hi || t0 < wg_lo) {
      // each thread looks at the values that it has loaded; rows of absent
      // pages become zeros
      // (opaque: addresses are formed here, not kept in registers)
      int me = tid;
      asm volatile("" : "+v"(me));
#pragma unroll
      for (int u = 0; u < C::PER; ++u) {
        const int i = u * PT_THREADS + me, row = i / C::CH;
        u4* at = (u4*)(v + 16 * i);
        if ((absent >> row) & 1) {
          *at = (u4){0u, 0u, 0u, 0u};
        } else if (without_infinities<T>(at)) {
          atomicMin(&odd_tiles[0], t0);
          atomicMax(&odd_tiles[1], t0);
        }
      }
    }
    wait_lds();
    __builtin_amdgcn_s_barrier();                      // both are there, the other halves free
    asm volatile("" : : : "memory");
    page = next;
    next = page_at(t0 + 2 * C::TN, entry);
    absent = next_absent;
    next_absent = __ballot(next < 0);
    if (t0 + C::TN < end) {
      fetch(false, t0 + C::TN, page, vt + (odd ^ 1) * C::BYTES);
      fetch(true, t0 + 2 * C::TN, next, kt + odd * C::BYTES);
      entry = entry_of(a.pool, b, t0 + 3 * C::TN + mine);
    }
    // (past the last tile the scores are those of stale keys, never used)
    typename Vec<T>::v8 p[NB][2];
    c.template scores<NB>(kt + (odd ^ 1) * C::BYTES, ahead);
    c.template weights<NB>(a, sc, p);
    c.template add_values<NB>(v, p);
    // one product of the scores, one key read, and a share of the weights in
    // turn; then the values, read two products ahead
    constexpr int N = NB * (HD / 16), W = NB * 16;     // products, weights
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < N - 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 5 * W / (2 * N), 0);
      __builtin_amdgcn_sched_group_barrier(0x400, W / N, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < N - 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    if (t0 + C::TN < end) c.template settle<NB>(a, t0 + C::TN, absent, ahead);
  };
  for (int t0 = begin; t0 < end; t0 += 2 * C::TN) {
    step(t0, 0, even_scores, odd_scores);
    if (t0 + C::TN >= end) break;
    step(t0 + C::TN, 1, odd_scores, even_scores);
  }
  __syncthreads();
  const float2 ls = both_halves(c.l);
  c.l = ls.x + ls.y;
  const bool real = r < s.n * a.GQ;
  c.add_infinities(a, b, head, real, __builtin_amdgcn_readfirstlane(odd_tiles[0]),
                   __builtin_amdgcn_readfirstlane(odd_tiles[1]), begin, end, C::TN, C::TN);
  if (!real) return;
  const int tok = r / a.GQ, g = r - tok * a.GQ;
  const int64_t orow = (int64_t)(s.first + tok) * a.Hq + head * a.GQ + g;
  if (w.parts == 1) {
    put_row<T, HD>(a, c, orow);
    return;
  }
  const int64_t rec = a.many0 + orow * a.ns_many + part;
  const int half = lane >> 5;
  float* dst = a.part + rec * HD + 4 * half;
#pragma unroll
  for (int t = 0; t < HD / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f4*)(dst + 32 * t + 8 * i) =
          (f4){c.o[t][4 * i], c.o[t][4 * i + 1], c.o[t][4 * i + 2], c.o[t][4 * i + 3]};
  if (half == 0) *(float2*)(a.part_ml + 2 * rec) = make_float2(c.m, c.l);
}

// The same for four of a row's sums, from dimension `dim` on, over a piece
// of the keys: where one is NaN, what the row sees there that is not finite.
template <typename T>
__device__ __forceinline__ void see_row_infinities(const PtArgs& a, const Seq& s, int b, int head,
                                                   int tok, int dim, int from, int to, f4& o) {
  const int64_t pos = s.pos0 + tok, low = a.window ? pos - a.window + 1 : 0;
  f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int64_t j = low > from ? low : from; j < to && j <= pos; ++j) {
    const int page = page_of(a.pool, b, j);
    if (page < 0) continue;
    const T* v = (const T*)a.pool.v + page * a.pool.vs[0] +
                 (j & ((1 << a.pool.shift) - 1)) * a.pool.vs[1] + head * a.pool.vs[2] + dim;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += is_finite((float)v[e]) ? 0.f : (float)v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = o[e] != o[e] && !is_finite(y[e]) ? y[e] : o[e];
}

// All queries (32 at most) of one sequence and key head, and a piece of the
// keys: each wave takes every fourth tile of 32 keys, and the waves' sums are
// joined in LDS.
template <typename T, int HD>
__device__ __forceinline__ void few(const PtArgs& a, char* lds, int block) {
  typedef PtCfg<HD> C;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = block % a.pool.Hkv;
  const int rest = block / a.pool.Hkv;
  const int part = rest % a.ns_few, b = rest / a.ns_few;
  const Seq s = sequence(a, b);
  if (s.n == 0 || !is_few(a, s)) return;
  const Span w = span_of(a, s, 0, PT_FEW, PT_FEW_UNIT, a.ns_few);
  if (part >= w.parts) return;
  const int begin = w.lo + part * w.step + 32 * wave;
  const int end = min(w.hi, w.lo + (part + 1) * w.step);
  char* kt = lds + wave * 2 * C::FEW_BYTES;
  char* vt = kt + C::FEW_BYTES;
  Columns<T, HD> c;
  c.start(a, s, head, lane & 31);
  // keys that every query of the sequence sees
  const int64_t q_hi = min((int64_t)s.keys, s.pos0 + 1);
  const int64_t q_lo = a.window ? s.pos0 + s.n - a.window : 0;

  // Where the wave's tiles lie: pages are looked up for 16 tiles at once, one
  // group of 8 tokens (which lie in one page) a lane, lane 4 (tile mod 16) +
  // group.  A lookup per tile would be waited for with all loads behind it.
  constexpr int RL = 64 / C::CH;                       // rows of one load
  const int lrow = lane / C::CH, lch = lane % C::CH;
  const char* const kbase = a.pool.k + sizeof(T) * head * a.pool.ks[2];
  const char* const vbase = a.pool.v + sizeof(T) * head * a.pool.vs[2];
  uint64_t k_at = 0, v_at = 0, there = 0;              // offsets; lanes whose page is there
  auto look_up = [&](int i) __attribute__((always_inline)) {
    const int t = begin + (i + (lane >> 2)) * PT_FEW_UNIT + 8 * (lane & 3);
    const int page = t < end ? checked(a.pool, entry_of(a.pool, b, t)) : -1;
    k_at = token_offset(a.pool, a.pool.ks, page, t);
    v_at = token_offset(a.pool, a.pool.vs, page, t);
    there = __ballot(page >= 0);
  };
  // rows of tile i that are not there: by groups, and behind the last key
  auto gone = [&](int i, int t0) {
    const uint32_t groups = (uint32_t)(there >> (4 * (i & 15))) & 15u;
    const uint32_t held = (groups * 0x00204081u & 0x01010101u) * 0xffu;
    const int left = end - t0;
    return ~held | (left >= 32 ? 0u : left <= 0 ? ~0u : ~0u << left);
  };
  // the keys or the values of tile i to LDS
  auto fetch = [&](bool key, int i, const char* to) __attribute__((always_inline)) {
    const int64_t (&st)[3] = key ? a.pool.ks : a.pool.vs;
#pragma unroll
    for (int u = 0; u < C::FEW_PER; ++u) {
      const int row = u * RL, in = row % 8;
      const int ch = key ? key_chunk<HD>(row + lrow, lch) : value_chunk<HD>(row + lrow, lch);
      load_to_lds(rows_at(key ? kbase : vbase, key ? k_at : v_at, 4 * (i & 15) + row / 8),
                  2 * ((in + lrow) * (uint32_t)st[1] + 8 * ch), lds_offset(to) + 1024 * u);
    }
  };
  int odd_from = INT32_MAX, odd_to = -1;               // tiles with infinities or NaN
  // Keys and values have one tile's place each: while weights are computed
  // the values are on their way, and while these are added the next keys.
  uint32_t absent = 0;
  if (begin < end) {
    look_up(0);
    absent = gone(0, begin);
    fetch(true, 0, kt);
    fetch(false, 0, vt);
  }
  int i = 0;
  for (int t0 = begin; t0 < end; t0 += PT_FEW_UNIT) {
    wait_loads<C::FEW_PER>();                          // the keys are there
    f16v sc[1];
    typename Vec<T>::v8 p[1][2];
    c.template scores<1>(kt, sc);
    c.template settle<1>(a, t0, absent, sc);
    c.template weights<1>(a, sc, p);
    wait_lds();                                        // the keys have been read
    if ((++i & 15) == 0) look_up(i);
    fetch(true, i, kt);
    wait_loads<C::FEW_PER>();                          // the values are there
    if (absent || t0 + 32 > q_hi || t0 < q_lo) {
      bool odd = false;
      int me = lane;
      asm volatile("" : "+v"(me));
#pragma unroll
      for (int u = 0; u < C::FEW_PER; ++u) {
        u4* v = (u4*)(vt + 16 * (u * 64 + me));
        if ((absent >> ((u * 64 + me) / C::CH)) & 1) *v = (u4){0u, 0u, 0u, 0u};
        else odd = without_infinities<T>(v) || odd;
      }
      if (__any(odd)) {
        odd_from = min(odd_from, t0);
        odd_to = t0;
      }
    }
    c.template add_values<1>(vt, p);
    wait_lds();                                        // the values have been read
    fetch(false, i, vt);
    absent = gone(i, t0 + PT_FEW_UNIT);
  }
  wait_loads<0>();                                     // no load writes to LDS from here on
  c.see_infinities(a, b, head, odd_from, odd_to, PT_FEW_UNIT, 32);

  // join the four waves: [wave][32 queries][HD] sums, in the tiles' LDS
  const float2 ls = both_halves(c.l);
  c.l = ls.x + ls.y;
  __shared__ float ml[PT_WAVES][2][32];
  const int col = lane & 31, half = lane >> 5;
  const int rows = s.n * a.GQ;
  __syncthreads();
  float* sums = (float*)lds;
  if (half == 0) {
    ml[wave][0][col] = c.m;
    ml[wave][1][col] = c.l;
  }
  if (col < rows) {
#pragma unroll
    for (int t = 0; t < HD / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // 16-byte chunks in an order of the row's own against bank conflicts
        const int ch = (8 * t + 2 * i + half) ^ (col & 7);
        *(f4*)(sums + (wave * 32 + col) * HD + 4 * ch) =
            (f4){c.o[t][4 * i], c.o[t][4 * i + 1], c.o[t][4 * i + 2], c.o[t][4 * i + 3]};
      }
  }
  __syncthreads();
  constexpr int L = HD / 4;                            // lanes per row
  for (int r = tid / L; r < rows; r += PT_THREADS / L) {
    float top = ml[0][0][r];
#pragma unroll
    for (int x = 1; x < PT_WAVES; ++x) top = fmaxf(top, ml[x][0][r]);
    const int ch = tid % L;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < PT_WAVES; ++x) {
      const float f = ml[x][0][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[x][0][r] - top);
      const f4 v = *(const f4*)(sums + (x * 32 + r) * HD + 4 * (ch ^ (r & 7)));
      l += f * ml[x][1][r];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += f * v[e];
    }
    const int tok = r / a.GQ, g = r - tok * a.GQ;
    bool lost = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) lost = lost || o[e] != o[e];
    if (__builtin_expect(lost && l == l, 0))
      see_row_infinities<T>(a, s, b, head, tok, 4 * ch, w.lo + part * w.step,
                            min(w.hi, w.lo + (part + 1) * w.step), o);
    const int64_t orow = (int64_t)(s.first + tok) * a.Hq + head * a.GQ + g;
    if (w.parts == 1) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      typename Vec<T>::v4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = result<T>(o[e] * inv);
      *(typename Vec<T>::v4*)((T*)a.out + orow * HD + 4 * ch) = x;
      if (a.lse && ch == 0)
        a.lse[orow] = l == 0.f ? -INFINITY : (top - PT_SHIFT + log2f(l)) * 0.69314718055994531f;
    } else {
      const int64_t at = a.few_by_row ? orow : ((int64_t)b * a.pool.Hkv + head) * PT_FEW + r;
      const int64_t rec = at * a.ns_few + part;
      *(f4*)(a.part + rec * HD + 4 * ch) = o;
      if (ch == 0) *(float2*)(a.part_ml + 2 * rec) = make_float2(top, l);
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(PT_THREADS, HD == 256 ? 1 : HD == 128 ? 2 : 3) paged_attn_kernel(PtArgs a) {
  __shared__ __align__(16) char lds[PtCfg<HD>::LDS];
  const bool first = (int)blockIdx.x < a.first_blocks;
  const int block = first ? blockIdx.x : blockIdx.x - a.first_blocks;
  if (first == a.many_first) many<T, HD>(a, lds, block);
  else few<T, HD>(a, lds, block);
}

template <typename T, int HD>
gsrq_status pt_launch(const PtArgs& a, const PtPlan& p, hipStream_t st) {
  static_assert(PtCfg<HD>::LDS <= 160 * 1024 - 2048, "LDS of a CU");
  TimedLaunch tl(GSRQ_KERNEL_ATTENTION, st);
  paged_attn_kernel<T, HD><<<p.few_blocks + p.many_blocks, PT_THREADS, 0, st>>>(a);
  gsrq_status e = launch_ok();
  if (e || p.merge_few + p.merge_rows == 0) return e;
  paged_attn_merge_kernel<T, HD, PT_FEW_UNIT><<<p.merge_few + p.merge_rows, 256, 0, st>>>(a);
  return launch_ok();
}

}  // namespace

extern "C" {

gsrq_status gsrq_attn_paged_workspace_bytes(const gsrq_paged_attn* s, const gsrq_pages* pages,
                                            size_t* bytes) {
  if (!bytes) return GSRQ_E_ARG;
  PtPlan p;
  gsrq_status e = pt_plan(s, pages, false, PT_FEW_UNIT, p);
  if (e) return e;
  *bytes = p.bytes;
  return GSRQ_OK;
}

gsrq_status gsrq_attn_paged(const gsrq_paged_attn* s, const gsrq_pages* pages,
                            const int32_t* q_start, const int32_t* seq_len, const gsrq_heads* q,
                            void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  PtPlan p;
  gsrq_status e = pt_plan(s, pages, false, PT_FEW_UNIT, p);
  if (e) return e;
  PtArgs a;
  if ((e = pt_args(s, pages, p, q_start, seq_len, q, out, lse, workspace, ws_bytes, a))) return e;
  hipStream_t st = (hipStream_t)stream;
  const int hd = pages->head_dim;
  if (pages->dtype == GSRQ_F16) {
    if (hd == 64) return pt_launch<_Float16, 64>(a, p, st);
    if (hd == 128) return pt_launch<_Float16, 128>(a, p, st);
    return pt_launch<_Float16, 256>(a, p, st);
  }
  if (hd == 64) return pt_launch<__bf16, 64>(a, p, st);
  if (hd == 128) return pt_launch<__bf16, 128>(a, p, st);
  return pt_launch<__bf16, 256>(a, p, st);
}

}  // extern "C"
