// Appending new tokens to a paged cache, and restoring coded contexts into
// one, on AMD MI355X (gfx950).  (Attention over the pages: gsrq_attn_paged.hip.)
//
// Appending.  For every head x of a new token's row at position p
//   y = x / sqrt(mean(x^2) + eps) * norm,   (y_j, y_{j + h/2}) turned by p theta_j
// for keys and queries, values as they are; keys and values go to
// page table[b][p / page_size].  One pass over the data: hd/16 lanes share a
// head, each with 8 elements of its lower half and the 8 they are turned with,
// so a rotation needs no exchange and every access is 16 bytes (float32: 32).
//
// Restoring.  A token's row is the sum of its stages' codewords fl32(g s),
// keys then turned in float32 at the token's position.
#include "gsrq_paged.h"

namespace {

constexpr int PA_THREADS = 256;

__device__ __forceinline__ void load8(const _Float16* p, float (&x)[8]) {
  const h8 v = *(const h8*)p;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
}
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  const b8 v = *(const b8*)p;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f4 lo = ((const f4*)p)[0], hi = ((const f4*)p)[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) { x[j] = lo[j]; x[4 + j] = hi[j]; }
}
// Rounded to the pages' type here, once (to the nearest, ties to even).
__device__ __forceinline__ void store8(_Float16* p, const float (&x)[8]) {
  h8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (_Float16)x[j];
  *(h8*)p = v;
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  b8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (__bf16)x[j];
  *(b8*)p = v;
}

// Cosine and sine of pos * theta.  In 64 bits up to the whole turns: at
// position 2^20 a float32 product would be off by 0.06 radians.
__device__ __forceinline__ void turn_of(int64_t pos, double theta, float& c, float& s) {
  double r = (double)pos * (theta * 0.15915494309189533577);   // 1 / (2 pi)
  r -= rint(r);
  sincospif(2.f * (float)r, &s, &c);
}

struct AppendArgs {
  PagePool pool;
  const void *k, *v, *q;
  int64_t kst[2], vst[2], qst[2];     // token, head
  const int32_t *q_start, *seq_len;
  const double* theta;
  const float *k_norm, *q_norm;
  void* q_out;
  int T, Hq;
  float eps;
};

// One workgroup per token and group of 256 / (hd/16) heads.
template <typename TI, typename TP, int HD>
__global__ void __launch_bounds__(PA_THREADS) paged_append_kernel(AppendArgs a) {
  constexpr int L = HD / 16;                    // lanes per head
  __shared__ float cs[HD / 2], sn[HD / 2];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int b = sequence_of(a.q_start, a.pool.B, row);
  if (b < 0) return;
  int first, n;
  new_rows(a.q_start, b, a.T, first, n);
  const int64_t pos = (int64_t)a.seq_len[b] - n + (row - first);
  if (a.theta) {
    for (int j = tid; j < HD / 2; j += PA_THREADS) turn_of(pos, a.theta[j], cs[j], sn[j]);
    __syncthreads();
  }
  const int l = tid % L;
  int h = blockIdx.y * (PA_THREADS / L) + tid / L;
  const int Hkv = a.pool.Hkv;
  if (h >= 2 * Hkv + a.Hq) return;
  const TI* src;
  TP* dst;
  const float* norm = nullptr;
  bool turn = a.theta != nullptr;
  if (h < 2 * Hkv) {
    const bool key = h < Hkv;
    h -= key ? 0 : Hkv;
    const int page = page_of(a.pool, b, pos);
    if (page < 0) return;
    const int64_t* ps = key ? a.pool.ks : a.pool.vs;
    const int64_t slot = pos & ((1 << a.pool.shift) - 1);
    dst = (TP*)(key ? a.pool.k : a.pool.v) + page * ps[0] + slot * ps[1] + h * ps[2];
    src = key ? (const TI*)a.k + row * a.kst[0] + h * a.kst[1]
              : (const TI*)a.v + row * a.vst[0] + h * a.vst[1];
    norm = key ? a.k_norm : nullptr;
    turn = turn && key;
  } else {
    h -= 2 * Hkv;
    src = (const TI*)a.q + row * a.qst[0] + h * a.qst[1];
    dst = (TP*)a.q_out + ((int64_t)row * a.Hq + h) * HD;
    norm = a.q_norm;
  }
  float lo[8], hi[8];
  load8(src + 8 * l, lo);
  load8(src + HD / 2 + 8 * l, hi);
  if (norm) {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(lo[j], lo[j], fmaf(hi[j], hi[j], ss));
#pragma unroll
    for (int m = 1; m < L; m <<= 1) ss += __shfl_xor(ss, m);
    const float r = 1.f / sqrtf(ss * (1.f / HD) + a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      lo[j] *= r * norm[8 * l + j];
      hi[j] *= r * norm[HD / 2 + 8 * l + j];
    }
  }
  if (turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = cs[8 * l + j], s = sn[8 * l + j], x = lo[j], y = hi[j];
      lo[j] = x * c - y * s;
      hi[j] = y * c + x * s;
    }
  }
  store8(dst + 8 * l, lo);
  store8(dst + HD / 2 + 8 * l, hi);
}

struct RestoreArgs {
  PagePool pool;
  const uint32_t *k_codes, *v_codes;
  const float *k_gain, *k_shape, *v_gain, *v_shape;
  const int32_t* seq_len;
  const double* theta;
  int64_t words;
  int cap, M, G, K, b, d, hd;
};

__device__ __forceinline__ int code_at(const uint32_t* row, int64_t bit, int b) {
  const int64_t w = bit >> 5;
  const int o = (int)(bit & 31);
  uint32_t v = row[w] >> o;
  if (o + b > 32) v |= row[w + 1] << (32 - o);
  return (int)(v & ((1u << b) - 1u));
}

// Eight elements from element e of a row: the stages' codewords, each rounded
// to float32 before the sum (no fused multiply-add).
__device__ __forceinline__ void codeword_sum(const RestoreArgs& a, const uint32_t* codes,
                                             const float* gain, const float* shape, int e,
                                             float (&x)[8]) {
#pragma clang fp contract(off)
  const int g = e / a.d;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
  for (int m = 0; m < a.M; ++m) {
    const int64_t cb = (int64_t)m * a.G + g;
    const int k = code_at(codes, cb * a.b, a.b);
    const float gk = gain[cb * a.K + k];
    float s[8];
    load8(shape + (cb * a.K + k) * a.d + (e - g * a.d), s);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += gk * s[j];
  }
}

// A lane per 16 elements of a head of one token's key or value row.
template <typename TP>
__global__ void __launch_bounds__(PA_THREADS) paged_row_decode_kernel(RestoreArgs a) {
  const int L = a.hd / 16;
  const int64_t per = (int64_t)a.pool.Hkv * L;            // lanes per row
  const int64_t item = (int64_t)blockIdx.x * PA_THREADS + threadIdx.x;
  const int b = blockIdx.z;
  const bool key = blockIdx.y == 0;
  const int64_t pos = item / per;
  const int h = (int)(item % per) / L, l = (int)(item % L);
  const int len = min(a.seq_len[b], a.cap);
  if (pos >= len) return;
  const int page = page_of(a.pool, b, pos);
  if (page < 0) return;
  const uint32_t* codes = (key ? a.k_codes : a.v_codes) + ((int64_t)b * a.cap + pos) * a.words;
  float lo[8], hi[8];
  codeword_sum(a, codes, key ? a.k_gain : a.v_gain, key ? a.k_shape : a.v_shape,
               h * a.hd + 8 * l, lo);
  codeword_sum(a, codes, key ? a.k_gain : a.v_gain, key ? a.k_shape : a.v_shape,
               h * a.hd + a.hd / 2 + 8 * l, hi);
  if (key && a.theta) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float c, s;
      turn_of(pos, a.theta[8 * l + j], c, s);
      const float x = lo[j], y = hi[j];
      lo[j] = x * c - y * s;
      hi[j] = y * c + x * s;
    }
  }
  const int64_t* ps = key ? a.pool.ks : a.pool.vs;
  TP* dst = (TP*)(key ? a.pool.k : a.pool.v) + page * ps[0] +
            (pos & ((1 << a.pool.shift) - 1)) * ps[1] + h * ps[2];
  store8(dst + 8 * l, lo);
  store8(dst + a.hd / 2 + 8 * l, hi);
}

template <typename TI, typename TP>
gsrq_status append_launch(const AppendArgs& a, int hd, hipStream_t st) {
  TimedLaunch tl(GSRQ_KERNEL_APPEND, st);
  const int heads = 2 * a.pool.Hkv + a.Hq, group = PA_THREADS * 16 / hd;
  const dim3 grid((unsigned)a.T, (unsigned)((heads + group - 1) / group));
  if (hd == 64) paged_append_kernel<TI, TP, 64><<<grid, PA_THREADS, 0, st>>>(a);
  else if (hd == 128) paged_append_kernel<TI, TP, 128><<<grid, PA_THREADS, 0, st>>>(a);
  else paged_append_kernel<TI, TP, 256><<<grid, PA_THREADS, 0, st>>>(a);
  return launch_ok();
}

}  // namespace

extern "C" {

gsrq_status gsrq_paged_append(const gsrq_pages* pages, int64_t T, const int32_t* q_start,
                              const int32_t* seq_len, const gsrq_heads* k, const gsrq_heads* v,
                              const gsrq_heads* q, int32_t Hq, gsrq_dtype dtype,
                              const double* theta, const float* k_norm, const float* q_norm,
                              float eps, void* q_out, void* stream) {
  AppendArgs a;
  gsrq_status e = page_pool(pages, a.pool);
  if (e) return e;
  if (T < 1 || !q_start || !seq_len) return GSRQ_E_ARG;
  if (dtype != GSRQ_F32 && dtype != GSRQ_F16 && dtype != GSRQ_BF16) return GSRQ_E_ARG;
  const int64_t esz = dtype == GSRQ_F32 ? 4 : 2;
  if ((e = head_rows(k, esz)) || (e = head_rows(v, esz))) return e;
  if (q) {
    if ((e = head_rows(q, esz))) return e;
    if (Hq < 1 || !q_out || (uintptr_t)q_out % 16) return GSRQ_E_ARG;
  } else if (q_norm || q_out) {
    return GSRQ_E_ARG;
  }
  if (!(eps >= 0.f) || !(eps < INFINITY)) return GSRQ_E_ARG;
  if ((uintptr_t)theta % 8) return GSRQ_E_ARG;
  if (T > MAX_BLOCKS || 2ll * a.pool.Hkv + (q ? Hq : 0) > 65535) return GSRQ_E_UNSUPPORTED;
  a.k = k->data;
  a.v = v->data;
  a.q = q ? q->data : nullptr;
  a.kst[0] = k->token_stride; a.kst[1] = k->head_stride;
  a.vst[0] = v->token_stride; a.vst[1] = v->head_stride;
  a.qst[0] = q ? q->token_stride : 0; a.qst[1] = q ? q->head_stride : 0;
  a.q_start = q_start;
  a.seq_len = seq_len;
  a.theta = theta;
  a.k_norm = k_norm;
  a.q_norm = q_norm;
  a.q_out = q_out;
  a.T = (int)T;
  a.Hq = q ? Hq : 0;
  a.eps = eps;
  const int hd = pages->head_dim;
  hipStream_t st = (hipStream_t)stream;
  if (pages->dtype == GSRQ_F16) {
    if (dtype == GSRQ_F32) return append_launch<float, _Float16>(a, hd, st);
    if (dtype == GSRQ_F16) return append_launch<_Float16, _Float16>(a, hd, st);
    return append_launch<__bf16, _Float16>(a, hd, st);
  }
  if (dtype == GSRQ_F32) return append_launch<float, __bf16>(a, hd, st);
  if (dtype == GSRQ_F16) return append_launch<_Float16, __bf16>(a, hd, st);
  return append_launch<__bf16, __bf16>(a, hd, st);
}

gsrq_status gsrq_paged_restore(const gsrq_pages* pages, const gsrq_shape* kv, int32_t cap,
                               const uint32_t* k_codes, const uint32_t* v_codes,
                               const int32_t* seq_len, const float* k_gain, const float* k_shape,
                               const float* v_gain, const float* v_shape, const double* theta,
                               void* stream) {
  RestoreArgs a;
  gsrq_status e = page_pool(pages, a.pool);
  if (e) return e;
  if (!kv || cap < 1 || kv->N < 1 || kv->D < 1 || kv->d < 1 || kv->K < 2 || kv->M < 1)
    return GSRQ_E_ARG;
  if (kv->D % kv->d || !is_pow2(kv->K) || kv->K > 65536) return GSRQ_E_ARG;
  if (kv->D != (int64_t)pages->Hkv * pages->head_dim) return GSRQ_E_ARG;
  if (kv->N < (int64_t)pages->B * cap) return GSRQ_E_ARG;
  if (kv->d < 8 || kv->d > 256 || !is_pow2(kv->d)) return GSRQ_E_UNSUPPORTED;
  if (!k_codes || !v_codes || !seq_len || !k_gain || !k_shape || !v_gain || !v_shape)
    return GSRQ_E_ARG;
  if ((uintptr_t)k_shape % 16 || (uintptr_t)v_shape % 16 || (uintptr_t)theta % 8)
    return GSRQ_E_ARG;
  a.k_codes = k_codes;
  a.v_codes = v_codes;
  a.k_gain = k_gain;
  a.k_shape = k_shape;
  a.v_gain = v_gain;
  a.v_shape = v_shape;
  a.seq_len = seq_len;
  a.theta = theta;
  a.words = (int64_t)gsrq_code_words(kv);
  a.cap = cap;
  a.M = kv->M;
  a.d = kv->d;
  a.G = kv->D / kv->d;
  a.K = kv->K;
  a.b = log2i(kv->K);
  a.hd = pages->head_dim;
  const int64_t items = (int64_t)cap * pages->Hkv * (a.hd / 16);
  const int64_t blocks = (items + PA_THREADS - 1) / PA_THREADS;
  if (blocks > MAX_BLOCKS || pages->B > 65535) return GSRQ_E_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  TimedLaunch tl(GSRQ_KERNEL_DECODE, st);
  const dim3 grid((unsigned)blocks, 2, (unsigned)pages->B);
  if (pages->dtype == GSRQ_F16)
    paged_row_decode_kernel<_Float16><<<grid, PA_THREADS, 0, st>>>(a);
  else
    paged_row_decode_kernel<__bf16><<<grid, PA_THREADS, 0, st>>>(a);
  return launch_ok();
}

}  // extern "C"
