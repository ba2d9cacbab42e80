// Private header of the paged cache's translation units (gsrq_paged.hip:
// appending and restoring; gsrq_attn_paged.hip: attention over the pages):
// the pool of pages as the kernels see it, host checks, and the search for a
// row's sequence.
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

// Host checks of a pool (no HIP call).
inline gsrq_status page_pool(const gsrq_pages* p, PagePool& o) {
  if (!p || !p->k || !p->v || !p->table) return GSRQ_E_ARG;
  if (p->pages < 1 || p->page_size < 1 || p->per < 1 || p->B < 1 || p->Hkv < 1) return GSRQ_E_ARG;
  if (p->ldt < p->per || p->head_dim < 1) return GSRQ_E_ARG;
  if (p->dtype != GSRQ_F16 && p->dtype != GSRQ_BF16)
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
    if (p->k_stride[i] % 8 || p->v_stride[i] % 8) return GSRQ_E_ARG;
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

}  // namespace

#endif  // GSRQ_PAGED_H
