// Private header of the paged cache's translation units (gsrq_paged.hip:
// appending and restoring; gsrq_attn_paged.hip: attention over the pages;
// gsrq_cache8.hip: both over 8-bit pages; gsrq_serving.hip: planning and drafts):
// the pool of pages as the kernels see it, host checks, the search for a
// row's sequence, and accesses to its elements.
#ifndef GSRQ_PAGED_H
#define GSRQ_PAGED_H

#include "gsrq_common.h"

namespace {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// Workgroups of 256 threads in one grid dimension: HIP counts threads in 32 bits.
constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;

// A pool of pages (gsrq_pages): strides in elements, a page of 1 << shift
// tokens, `per` pages a sequence in `table` [B][ldt].
struct PagePool {
  char* k;
  char* v;
  const int32_t* table;
  int64_t ks[3], vs[3];     // page, token, head
  int64_t ldt;
  int pages, shift, per, B, Hkv;
};

// Host checks of a pool (no HIP call), of 8-bit pages or of 16-bit ones.
inline gsrq_status page_pool(const gsrq_pages* p, bool eight, PagePool& o) {
  if (!p || !p->k || !p->v || !p->table) return GSRQ_E_ARG;
  if (p->pages < 1 || p->page_size < 1 || p->per < 1 || p->B < 1 || p->Hkv < 1) return GSRQ_E_ARG;
  if (p->ldt < p->per || p->head_dim < 1) return GSRQ_E_ARG;
  if (eight && p->dtype != GSRQ_E4M3) return GSRQ_E_ARG;
  if (!eight && p->dtype != GSRQ_F16 && p->dtype != GSRQ_BF16)
    return p->dtype == GSRQ_F32 ? GSRQ_E_UNSUPPORTED : GSRQ_E_ARG;
  if ((int64_t)p->page_size * p->per > (1 << 30)) return GSRQ_E_ARG;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return GSRQ_E_UNSUPPORTED;
  if (!is_pow2(p->page_size) || p->page_size < 8) return GSRQ_E_UNSUPPORTED;
  if (p->k_stride[1] >= 1 << 26 || p->v_stride[1] >= 1 << 26 || p->k_stride[0] > INT32_MAX ||
      p->v_stride[0] > INT32_MAX)
    return GSRQ_E_UNSUPPORTED;
  if ((uintptr_t)p->k % 16 || (uintptr_t)p->v % 16) return GSRQ_E_ARG;
  const int count[3] = {p->pages, p->page_size, p->Hkv};
  for (int i = 0; i < 3; ++i) {
    const int64_t least = count[i] > 1 ? 1 : 0;      // no two tokens in one place
    if (p->k_stride[i] < least || p->v_stride[i] < least) return GSRQ_E_ARG;
    if (p->k_stride[i] % (eight ? 16 : 8) || p->v_stride[i] % (eight ? 16 : 8)) return GSRQ_E_ARG;
    o.ks[i] = p->k_stride[i];
    o.vs[i] = p->v_stride[i];
  }
  o.k = (char*)p->k;
  o.v = (char*)p->v;
  o.table = p->table;
  o.ldt = p->ldt;
  o.pages = p->pages;
  o.shift = log2i(p->page_size);
  o.per = p->per;
  o.B = p->B;
  o.Hkv = p->Hkv;
  return GSRQ_OK;
}

// Rows of heads (gsrq_heads): 16-byte accesses need 16-byte rows.
inline gsrq_status head_rows(const gsrq_heads* h, int64_t esz) {
  if (!h || !h->data || (uintptr_t)h->data % 16) return GSRQ_E_ARG;
  if (h->token_stride < 0 || h->head_stride < 0) return GSRQ_E_ARG;
  if (h->token_stride * esz % 16 || h->head_stride * esz % 16) return GSRQ_E_ARG;
  return GSRQ_OK;
}

// The page that holds a sequence's position, or -1: positions outside the
// table's row and entries outside [0, pages) have none.
__device__ __forceinline__ int page_of(const PagePool& p, int b, int64_t pos) {
  if (pos < 0 || (pos >> p.shift) >= p.per) return -1;
  const int page = p.table[b * p.ldt + (pos >> p.shift)];
  return page >= 0 && page < p.pages ? page : -1;
}

// The table's entry for a position >= 0 (past the row's end: its last), to be
// looked at only by checked(): a load that nothing waits for yet.
__device__ __forceinline__ int entry_of(const PagePool& p, int b, int pos) {
  const int i = pos >> p.shift;
  return p.table[b * p.ldt + (i < p.per ? i : p.per - 1)];
}
__device__ __forceinline__ bool in_table(const PagePool& p, int pos) {
  return (pos >> p.shift) < p.per;
}
__device__ __forceinline__ int checked(const PagePool& p, int entry) {
  return entry >= 0 && entry < p.pages ? entry : -1;
}

// First new row and number of new rows of sequence b, held inside [0, T).
__device__ __forceinline__ void new_rows(const int32_t* q_start, int b, int T, int& first, int& n) {
  const int lo = q_start[b], hi = q_start[b + 1];
  first = lo < 0 ? 0 : (lo > T ? T : lo);
  const int end = hi < first ? first : (hi > T ? T : hi);
  n = end - first;
}

// The sequence of row `row`, for a whole wave at once: the number of
// sequences that end at or before it (q_start ascends), 64 ends per load; -1
// for a row of no sequence.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int B, int row) {
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int i = 0; i < B; i += 64) {
    const bool done = i + lane < B && q_start[i + lane + 1] <= row;
    b += (int)__popcll(__ballot(done));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  return b < B && q_start[b] <= row ? b : -1;
}

// Eight elements of a row, in float32.
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

// The sum of a head's squares, in F; its HD / 16 lanes (16 elements each) all active.
template <typename F, int HD>
__device__ __forceinline__ F sum_of_squares(const float (&lo)[8], const float (&hi)[8]) {
  F ss = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) ss = fma((F)lo[j], (F)lo[j], fma((F)hi[j], (F)hi[j], ss));
#pragma unroll
  for (int m = 1; m < HD / 16; m <<= 1) ss += __shfl_xor(ss, m);
  return ss;
}

// 1 / sqrt(mean square + eps) of a head.  Where float32 does not hold the squares (elements from
// 2^60 on, or a mean and eps below 2^-100 together), the elements are scaled, by a power of two,
// and the factor is that of the scaled ones: their product is the same.  (The
// comparison costs appending to 8-bit pages 1%: 20000 rows of 32 / 8 heads of 128 take
// 101.3 us, 100.3 without; to 16-bit pages nothing, 94.)
template <int HD>
__device__ __forceinline__ float norm_factor(float (&lo)[8], float (&hi)[8], float eps, bool& scaled) {
  float t = sum_of_squares<float, HD>(lo, hi) * (1.f / HD) + eps;
  scaled = !(t >= 0x1p-100f && t < INFINITY);
  if (__builtin_expect(scaled, 0)) {
    const float s = t < 1.f ? 0x1p100f : 0x1p-72f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      lo[j] *= s;
      hi[j] *= s;
    }
    t = sum_of_squares<float, HD>(lo, hi) * (1.f / HD) + eps * s * s;
  }
  return 1.f / sqrtf(t);
}

// Cosine and sine of pos * theta.  In 64 bits up to the whole turns: at
// position 2^20 a float32 product would be off by 0.06 radians.
__device__ __forceinline__ void turn_of(int64_t pos, double theta, float& c, float& s) {
  double r = (double)pos * (theta * 0.15915494309189533577);   // 1 / (2 pi)
  r -= rint(r);
  sincospif(2.f * (float)r, &s, &c);
}

}  // namespace

#endif  // GSRQ_PAGED_H
