// What a serving step does around attention over pages, on AMD MI355X (gfx950):
// pages and slots for the batch's new tokens, and the verification of drafts.
//
// Planning.  Sequence b of L tokens changes by c tokens, L' = max(L + c, 0), and
// needs ceil(L' / P) pages.  Pages given back go on the free list, those needed
// come from it; who gets which is an exclusive sum over the batch.  The whole
// batch is one workgroup's (a few reads and sums per sequence: the time is that of
// a launch), the rows' slots a second launch's.
//
// Verification.  Row r of the target's probabilities p and the draft's q decides
// about draft t: accepted iff u q(t) < p(t).  The first rejected row's token is
// drawn from max(p - q, 0), after the last draft from p:
//   token = min { v : w_0 + .. + w_v > draw * sum w },
// with all sums in 64 bits (float32 would lose a token's weight in the sum of a
// vocabulary).  The first launch decides how far a sequence gets and sums its
// row's weights in chunks; the second finds the chunk and the token in it.
#include <algorithm>

#include "gsrq_paged.h"

namespace {

// ---------------------------------------------------------------- planning

constexpr int PL_THREADS = 1024;
constexpr int PL_MOST = 8192;             // sequences of a call

struct PlanArgs {
  int32_t *table, *free, *n_free, *seq_len;
  const int32_t* change;
  int32_t* q_start;
  int64_t* slots;
  int32_t* positions;
  int64_t ldt;
  int B, per, shift, F, T;
};

// a + b for 0 <= a, b < 2^31, at most 2^31 - 1.
__device__ __forceinline__ int sum_of(int a, int b) {
  const uint32_t s = (uint32_t)a + (uint32_t)b;
  return s > (uint32_t)INT32_MAX ? INT32_MAX : (int)s;
}

// The sum of the threads' x in front of this one, and of all (in `all`); for the
// whole workgroup.
__device__ __forceinline__ int sum_before(int x, int* wave_sums, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(s, d);
    s = lane >= d ? sum_of(s, y) : s;
  }
  if (lane == 63) wave_sums[wave] = s;
  const int up = __shfl_up(s, 1);
  int before = lane ? up : 0;
  __syncthreads();
  all = 0;
  for (int i = 0; i < PL_THREADS / 64; ++i) {
    if (i < wave) before = sum_of(before, wave_sums[i]);
    all = sum_of(all, wave_sums[i]);
  }
  __syncthreads();
  return before;
}

// What a sequence asks for.
struct Ask {
  int had, want;                  // tokens (want < 0: more than the table holds)
  int old_pages, new_pages;
};
__device__ __forceinline__ Ask ask_of(const PlanArgs& a, int b) {
  Ask x;
  const int64_t cap = (int64_t)a.per << a.shift;
  const int len = a.seq_len[b];
  x.had = len < 0 ? 0 : (len < cap ? len : (int)cap);
  const int64_t want = (int64_t)x.had + a.change[b];
  x.want = want > cap ? -1 : want < 0 ? 0 : (int)want;
  const int up = (1 << a.shift) - 1;
  x.old_pages = (x.had + up) >> a.shift;
  x.new_pages = x.want < 0 ? x.old_pages : (x.want + up) >> a.shift;
  return x;
}

// The last i of first[0 .. n] (ascending, first[0] = 0) with first[i] <= x.
template <typename P> __device__ __forceinline__ int owner(const P* first, int n, int x) {
  int lo = 0, hi = n;             // (first[n] is the sum of all: x is below it)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ void write_slot(const PlanArgs& a, int row) {
  if (row >= a.q_start[a.B]) {
    a.slots[row] = -1;
    a.positions[row] = -1;
    return;
  }
  const int b = owner(a.q_start, a.B, row);
  const int pos = a.seq_len[b] - (a.q_start[b + 1] - row);
  const int page = a.table[b * a.ldt + (pos >> a.shift)];
  a.slots[row] = page < 0 ? -1 : ((int64_t)page << a.shift) + (pos & ((1 << a.shift) - 1));
  a.positions[row] = pos;
}

__global__ void __launch_bounds__(PL_THREADS) plan_update_kernel(PlanArgs a, int rows_too) {
  __shared__ int first[PL_MOST + 1], who[PL_MOST];
  __shared__ int wave_sums[PL_THREADS / 64];
  const int tid = threadIdx.x;
  // pages that are given back: how many entries each sequence has of them
  int base = 0, all;
  for (int b0 = 0; b0 < a.B; b0 += PL_THREADS) {
    const int b = b0 + tid;
    int x = 0;
    if (b < a.B) {
      const Ask q = ask_of(a, b);
      x = max(q.old_pages - q.new_pages, 0);
    }
    const int before = sum_before(x, wave_sums, all);
    if (b < a.B) first[b] = sum_of(base, before);
    base = sum_of(base, all);
  }
  if (tid == 0) first[a.B] = base;
  __syncthreads();
  // from the last entry to the first, so that taking as many again brings them
  // in the order of the sequences; entries without a page are left out
  int count = *a.n_free;
  count = count < 0 ? 0 : (count > a.F ? a.F : count);
  for (int i0 = 0; i0 < base; i0 += PL_THREADS) {
    const int i = base - 1 - i0 - tid;
    int page = -1;
    if (i >= 0) {
      const int b = owner(first, a.B, i);
      const Ask q = ask_of(a, b);
      int32_t* entry = a.table + b * a.ldt + q.new_pages + (i - first[b]);
      page = *entry;
      *entry = -1;
    }
    const int at = sum_before(page >= 0, wave_sums, all);
    if (page >= 0 && count + (int64_t)at < a.F) a.free[count + at] = page;
    count = (int)min((int64_t)a.F, (int64_t)count + all);
  }
  __syncthreads();                                     // (workgroup: the list is one CU's)
  // who fits, in order, and what those who fit take
  int pages = 0, rows = 0, got = 0, out = 0;
  for (int b0 = 0; b0 < a.B; b0 += PL_THREADS) {
    const int b = b0 + tid;
    Ask q = {};
    int need = 0, more = 0;
    if (b < a.B) {
      q = ask_of(a, b);
      need = max(q.new_pages - q.old_pages, 0);
      more = q.want < 0 ? 0 : max(q.want - q.had, 0);
    }
    int all_pages, all_rows;
    const int p = sum_of(sum_of(pages, sum_before(need, wave_sums, all_pages)), need);
    const int r = sum_of(sum_of(rows, sum_before(more, wave_sums, all_rows)), more);
    pages = sum_of(pages, all_pages);
    rows = sum_of(rows, all_rows);
    const bool served = b < a.B && q.want >= 0 && (more == 0 || (p <= count && r <= a.T));
    need = served ? need : 0;
    more = served ? more : 0;
    const int p0 = sum_before(need, wave_sums, all_pages);
    const int r0 = sum_before(more, wave_sums, all_rows);
    if (b < a.B) {
      first[b] = got + p0;
      who[b] = q.old_pages;
      a.q_start[b] = out + r0;
      a.seq_len[b] = served ? q.want : q.had;
    }
    got += all_pages;
    out += all_rows;
  }
  if (tid == 0) {
    first[a.B] = got;
    a.q_start[a.B] = out;
    *a.n_free = count - got;
  }
  __syncthreads();
  for (int i = tid; i < got; i += PL_THREADS) {
    const int b = owner(first, a.B, i);
    int32_t* from = a.free + (count - 1 - i);
    a.table[b * a.ldt + who[b] + (i - first[b])] = *from;
    *from = -1;
  }
  if (!rows_too) return;
  __syncthreads();
  for (int row = tid; row < a.T; row += PL_THREADS) write_slot(a, row);
}

__global__ void __launch_bounds__(256) plan_slots_finalize_kernel(PlanArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row < a.T) write_slot(a, (int)row);
}

// ------------------------------------------------------------- verification

constexpr int VD_THREADS = 256;

struct VerifyArgs {
  const int32_t *tokens, *q_start;
  const void *target, *draft;     // draft: or null (a draft's probability is 1)
  const float *uniform, *draw;
  int32_t *accepted, *next;
  double* sums;                   // [B][2][chunks]: of max(p - q, 0), and of p
  int64_t ldp, ldq;
  int T, V, B, chunk, chunks;
};

// Weights below zero, and NaN, count as zero.
__device__ __forceinline__ double weight_of(double x) { return x > 0.0 ? x : 0.0; }

// How far a sequence gets: the row whose probabilities give its next token, and
// whether a draft was rejected there.  -1: it has no rows.
template <typename T>
__device__ __forceinline__ int stop_of(const VerifyArgs& a, int b, int& first, bool& rejected) {
  const int lane = threadIdx.x & 63;
  int n;
  new_rows(a.q_start, b, a.T, first, n);
  rejected = false;
  if (n == 0) return -1;
  for (int i0 = 0; i0 < n - 1; i0 += 64) {
    const int i = i0 + lane;
    bool no = false;
    if (i < n - 1) {
      const int row = first + i, t = a.tokens[row + 1];
      double p = 0.0, q = 0.0;
      if (t >= 0 && t < a.V) {
        p = (double)(float)((const T*)a.target)[row * a.ldp + t];
        q = a.draft ? (double)(float)((const T*)a.draft)[row * a.ldq + t] : 1.0;
      }
      no = !((double)a.uniform[row] * q < p);
    }
    const uint64_t where = __ballot(no);
    if (where) {
      rejected = true;
      return first + i0 + __builtin_ctzll(where);
    }
  }
  return first + n - 1;
}

// The two weights of token v: of what a rejection leaves, and of the target.
template <typename T> struct Weights {
  const T *p, *q;
  int one;                        // the token that a rejection takes out, where q is null
  bool rejected;
  __device__ __forceinline__ Weights(const VerifyArgs& a, int row, bool rej) : rejected(rej) {
    p = (const T*)a.target + row * a.ldp;
    q = a.draft ? (const T*)a.draft + row * a.ldq : nullptr;
    one = rej && !q ? a.tokens[row + 1] : -1;
  }
  __device__ __forceinline__ void get(int v, double& rest, double& all) const {
    all = weight_of((double)(float)p[v]);
    rest = 0.0;
    if (rejected) rest = q ? weight_of((double)(float)p[v] - (double)(float)q[v]) : v == one ? 0.0 : all;
  }
};

template <typename F> __device__ __forceinline__ double wave_sum(F x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

template <typename T>
__global__ void __launch_bounds__(VD_THREADS) verify_sums_kernel(VerifyArgs a) {
  __shared__ double part[2][VD_THREADS / 64];
  const int b = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
  int first;
  bool rejected;
  const int row = stop_of<T>(a, b, first, rejected);
  if (row < 0) return;
  const Weights<T> w(a, row, rejected);
  const int end = min(a.V, (c + 1) * a.chunk);
  double rest = 0.0, all = 0.0;
  for (int v = c * a.chunk + tid; v < end; v += VD_THREADS) {
    double x, y;
    w.get(v, x, y);
    rest += x;
    all += y;
  }
  rest = wave_sum(rest);
  all = wave_sum(all);
  if ((tid & 63) == 0) {
    part[0][tid >> 6] = rest;
    part[1][tid >> 6] = all;
  }
  __syncthreads();
  if (tid < 2) {
    double s = 0.0;
    for (int i = 0; i < VD_THREADS / 64; ++i) s += part[tid][i];
    a.sums[((int64_t)b * 2 + tid) * a.chunks + c] = s;
  }
}

// One workgroup per sequence: the chunk that holds the drawn point, by one
// thread's running sum; then the token, by the threads' sums of what each has of
// the chunk and one thread's running sum through its share.
template <typename T>
__global__ void __launch_bounds__(VD_THREADS) verify_finalize_kernel(VerifyArgs a) {
  __shared__ double shares[VD_THREADS];
  __shared__ double base, point;
  __shared__ int at, plain, best;
  const int b = blockIdx.x, tid = threadIdx.x;
  int first;
  bool rejected;
  const int row = stop_of<T>(a, b, first, rejected);
  if (row < 0) {
    if (tid == 0) {
      a.accepted[b] = 0;
      a.next[b] = -1;
    }
    return;
  }
  if (tid == 0) {
    const double* s = a.sums + (int64_t)b * 2 * a.chunks;
    double total = 0.0;
    for (int c = 0; c < a.chunks; ++c) total += s[c];
    plain = !(total > 0.0);
    if (plain) {
      s += a.chunks;
      total = 0.0;
      for (int c = 0; c < a.chunks; ++c) total += s[c];
    }
    point = (double)a.draw[b] * total;
    // the first chunk that passes the point; without one (a draw of 1 or more)
    // the last that has any weight
    double run = 0.0;
    int found = -1, last = -1;
    for (int c = 0; c < a.chunks && found < 0; ++c) {
      if (s[c] > 0.0) {
        last = c;
        base = run;
      }
      run += s[c];
      if (s[c] > 0.0 && run > point) found = c;
    }
    at = found >= 0 ? found : last;
    best = -1;
  }
  __syncthreads();
  if (at >= 0) {
    const Weights<T> w(a, row, rejected && !plain);
    const int begin = at * a.chunk, end = min(a.V, begin + a.chunk);
    const int each = (end - begin + VD_THREADS - 1) / VD_THREADS;
    const int from = min(end, begin + tid * each), to = min(end, from + each);
    double s = 0.0;
    for (int v = from; v < to; ++v) {
      double x, y;
      w.get(v, x, y);
      s += w.rejected ? x : y;
    }
    shares[tid] = s;
    __syncthreads();
    double run = base;
    for (int i = 0; i < tid; ++i) run += shares[i];
    // the token that passes the point in this thread's share, or the last with
    // any weight up to here (taken where no thread's passes it)
    int mine = -1;
    bool passed = false;
    for (int v = from; v < to && !passed; ++v) {
      double x, y;
      w.get(v, x, y);
      x = w.rejected ? x : y;
      run += x;
      if (x > 0.0) mine = v;
      passed = x > 0.0 && run > point;
    }
    // (the first thread that passes it, or else the last token of all)
    shares[tid] = passed ? 1.0 : 0.0;
    __syncthreads();
    bool before = false, any = false;
    for (int i = 0; i < VD_THREADS; ++i) {
      const bool x = shares[i] > 0.0;
      any = any || x;
      before = before || (x && i < tid);
    }
    if (any ? passed && !before : mine >= 0) atomicMax(&best, mine);
    __syncthreads();
  }
  if (tid == 0) {
    a.accepted[b] = row - first;
    a.next[b] = best;
  }
}

// Elements of a row that one workgroup sums: 4096 and more, a power of two, in
// at most 64 chunks.
void verify_chunks(int64_t V, int& chunk, int& chunks) {
  int64_t c = 4096;
  while (c * 64 < V) c *= 2;
  chunk = (int)c;
  chunks = (int)((V + c - 1) / c);
}

gsrq_status verify_shape(int64_t T, int64_t V, int64_t B) {
  if (T < 0 || V < 1 || B < 1) return GSRQ_E_ARG;
  if (T > INT32_MAX / 2 || V > INT32_MAX / 2 || B > (1 << 16)) return GSRQ_E_UNSUPPORTED;
  return GSRQ_OK;
}

template <typename T> gsrq_status verify_launch(const VerifyArgs& a, hipStream_t st) {
  TimedLaunch tl(GSRQ_KERNEL_SERVING, st);
  verify_sums_kernel<T><<<(unsigned)a.B * (unsigned)a.chunks, VD_THREADS, 0, st>>>(a);
  gsrq_status e = launch_ok();
  if (e) return e;
  verify_finalize_kernel<T><<<(unsigned)a.B, VD_THREADS, 0, st>>>(a);
  return launch_ok();
}

}  // namespace

extern "C" {

gsrq_status gsrq_paged_plan(const gsrq_paged_batch* s, int32_t* table, int32_t* free_pages,
                            int32_t* n_free, int32_t* seq_len, const int32_t* change,
                            int32_t* q_start, int64_t* slots, int32_t* positions, void* stream) {
  if (!s || !table || !free_pages || !n_free || !seq_len || !change || !q_start) return GSRQ_E_ARG;
  if (s->B < 1 || s->per < 1 || s->page_size < 1 || s->ldt < s->per || s->F < 1 || s->T < 0)
    return GSRQ_E_ARG;
  if (s->T > 0 && (!slots || !positions)) return GSRQ_E_ARG;
  if ((int64_t)s->page_size * s->per > (1 << 30)) return GSRQ_E_ARG;
  if (!is_pow2(s->page_size) || s->page_size < 8) return GSRQ_E_UNSUPPORTED;
  if (s->B > PL_MOST || s->T > INT32_MAX / 2 || (int64_t)s->B * s->per > INT32_MAX)
    return GSRQ_E_UNSUPPORTED;
  PlanArgs a;
  a.table = table;
  a.free = free_pages;
  a.n_free = n_free;
  a.seq_len = seq_len;
  a.change = change;
  a.q_start = q_start;
  a.slots = slots;
  a.positions = positions;
  a.ldt = s->ldt;
  a.B = s->B;
  a.per = s->per;
  a.shift = log2i(s->page_size);
  a.F = s->F;
  a.T = (int)s->T;
  hipStream_t st = (hipStream_t)stream;
  TimedLaunch tl(GSRQ_KERNEL_SERVING, st);
  const bool one = s->T <= 2 * PL_THREADS;
  plan_update_kernel<<<1, PL_THREADS, 0, st>>>(a, one);
  gsrq_status e = launch_ok();
  if (e || one) return e;
  plan_slots_finalize_kernel<<<(unsigned)((s->T + 255) / 256), 256, 0, st>>>(a);
  return launch_ok();
}

gsrq_status gsrq_verify_drafts_workspace_bytes(int64_t T, int64_t V, int32_t B, size_t* bytes) {
  if (!bytes) return GSRQ_E_ARG;
  gsrq_status e = verify_shape(T, V, B);
  if (e) return e;
  int chunk, chunks;
  verify_chunks(V, chunk, chunks);
  *bytes = align256((size_t)B * 2 * chunks * sizeof(double));
  return GSRQ_OK;
}

gsrq_status gsrq_verify_drafts(int64_t T, int64_t V, int32_t B, const int32_t* tokens,
                               const void* target, int64_t ldp, const void* draft, int64_t ldq,
                               gsrq_dtype dtype, const float* uniform, const float* draw,
                               const int32_t* q_start, int32_t* accepted, int32_t* next,
                               void* workspace, size_t ws_bytes, void* stream) {
  gsrq_status e = verify_shape(T, V, B);
  if (e) return e;
  if (!q_start || !draw || !accepted || !next || !workspace) return GSRQ_E_ARG;
  if (T > 0 && (!tokens || !target || !uniform)) return GSRQ_E_ARG;
  if (T > 1 && (ldp < V || (draft && ldq < V))) return GSRQ_E_ARG;
  if (dtype != GSRQ_F32 && dtype != GSRQ_F16 && dtype != GSRQ_BF16) return GSRQ_E_ARG;
  const uintptr_t esz = dtype == GSRQ_F32 ? 4 : 2;
  if ((uintptr_t)target % esz || (uintptr_t)draft % esz || (uintptr_t)workspace % 256)
    return GSRQ_E_ARG;
  VerifyArgs a;
  verify_chunks(V, a.chunk, a.chunks);
  if (ws_bytes < align256((size_t)B * 2 * a.chunks * sizeof(double))) return GSRQ_E_WORKSPACE;
  a.tokens = tokens;
  a.q_start = q_start;
  a.target = target;
  a.draft = draft;
  a.uniform = uniform;
  a.draw = draw;
  a.accepted = accepted;
  a.next = next;
  a.sums = (double*)workspace;
  a.ldp = ldp;
  a.ldq = ldq;
  a.T = (int)T;
  a.V = (int)V;
  a.B = B;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == GSRQ_F32) return verify_launch<float>(a, st);
  if (dtype == GSRQ_F16) return verify_launch<_Float16>(a, st);
  return verify_launch<__bf16>(a, st);
}

}  // extern "C"
