// What a serving step does around attention over pages, on AMD MI355X (gfx950):
// pages and slots for the batch's new tokens, and the verification of drafts.
//
// Planning.  Sequence b of L tokens changes by c tokens, L' = max(L + c, 0), and
// needs ceil(L' / P) pages.  Pages given back go on the free list, those needed
// come from it; who gets which is an exclusive sum over the batch.  The whole
// batch is one workgroup's: a few reads and sums per sequence (32 sequences of one
// token: 3 us), and rounds of reads and stores per page that moves (8600 pages: 12 us
// taking them, 16 giving them back).  Up to 2048 rows it writes their slots too; those
// of more rows are a second launch's.
//
// Verification.  Row r of the target's probabilities p and the draft's q decides
// about draft t: accepted iff u q(t) < p(t).  The first rejected row's token is
// drawn from max(p - q, 0), after the last draft from p:
//   token = min { v : w_0 + .. + w_v > draw * sum w },
// with all sums in 64 bits (float32 would lose a token's weight in the sum of a
// vocabulary).  Rows of at most 4096 tokens are one workgroup's; for longer ones
// a first launch decides how far a sequence gets and sums its row's weights in
// chunks, and a second finds the chunk and the token in it.
#include <algorithm>

#include "gsrq_paged.h"

namespace {

// ---------------------------------------------------------------- planning

constexpr int PL_THREADS = 1024;
constexpr int PL_MOST = 8192;             // sequences of a call
constexpr int PL_EACH = 4;                // entries that a thread moves at once (64 / waves)

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

// One step of a sum over the lanes before: x plus that of the lane that CTRL
// names, where there is one, in the rows of 16 lanes of ROWS.
template <int CTRL, int ROWS> __device__ __forceinline__ int step_sum(int x) {
  return sum_of(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false));
}
// The sum of x up to and with this lane's: in rows of 16 (1, 2, 4, 8 lanes on),
// then the last of a row to the next one's, then lane 31 to the upper half.  (All
// lanes active.  By shuffles each step is a trip through LDS.)
__device__ __forceinline__ int lane_sum(int x) {
  x = step_sum<0x111, 0xf>(x);
  x = step_sum<0x112, 0xf>(x);
  x = step_sum<0x114, 0xf>(x);
  x = step_sum<0x118, 0xf>(x);
  x = step_sum<0x142, 0xa>(x);
  return step_sum<0x143, 0xc>(x);
}
__device__ __forceinline__ int2 lane_sums(int2 x) { return make_int2(lane_sum(x.x), lane_sum(x.y)); }

// The sums of the threads' x in front of this one, and of all (in `all`); for
// the whole workgroup, of whole waves.
__device__ __forceinline__ int2 sums_before(int2 x, int2* wave_sums, int2& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int2 s = lane_sums(x);
  const int up = __shfl_up(s.x, 1), up2 = __shfl_up(s.y, 1);
  const int2 before = make_int2(lane ? up : 0, lane ? up2 : 0);
  if (waves == 1) {
    all = make_int2(__shfl(s.x, 63), __shfl(s.y, 63));
    return before;
  }
  if (lane == 63) wave_sums[wave] = s;
  __syncthreads();
  const int2 sums = lane_sums(lane < waves ? wave_sums[lane] : make_int2(0, 0));
  all = make_int2(__shfl(sums.x, 63), __shfl(sums.y, 63));
  const int w = __shfl(sums.x, wave ? wave - 1 : 0), w2 = __shfl(sums.y, wave ? wave - 1 : 0);
  __syncthreads();
  return wave ? make_int2(sum_of(before.x, w), sum_of(before.y, w2)) : before;
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

// For each x the last i < n with first[i] <= x (first ascends from 0): E searches
// side by side.
template <int E>
__device__ __forceinline__ void owners(const int* first, int n, const int (&x)[E], int (&b)[E]) {
#pragma unroll
  for (int u = 0; u < E; ++u) b[u] = 0;
  for (int w = 1 << (31 - __clz(n)); w; w >>= 1) {
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const int i = b[u] + w;
      const bool fits = i < n && first[i < n ? i : 0] <= x[u];
      b[u] = fits ? i : b[u];
    }
  }
}

// `start`: q_start, or a copy of it.
__device__ __forceinline__ void write_slot(const PlanArgs& a, const int* start, int row) {
  if (row >= start[a.B]) {
    a.slots[row] = -1;
    a.positions[row] = -1;
    return;
  }
  int own[1];
  owners<1>(start, a.B, {row}, own);
  const int b = own[0], pos = a.seq_len[b] - (start[b + 1] - row);
  const int page = a.table[b * a.ldt + (pos >> a.shift)];
  a.slots[row] = page < 0 ? -1 : ((int64_t)page << a.shift) + (pos & ((1 << a.shift) - 1));
  a.positions[row] = pos;
}

__global__ void __launch_bounds__(PL_THREADS) plan_update_kernel(PlanArgs a, int rows_too) {
  __shared__ int first[PL_MOST + 1], who[PL_MOST], start[PL_MOST + 1];
  __shared__ int2 wave_sums[PL_THREADS / 64];
  __shared__ int counts[64];
  const int tid = threadIdx.x, NT = blockDim.x;
  const int lane = tid & 63, wave = tid >> 6, waves = NT >> 6;
  int count = *a.n_free;
  // pages that are given back: how many entries each sequence has of them
  int base = 0;
  Ask q = {};
  for (int b0 = 0; b0 < a.B; b0 += NT) {
    const int b = b0 + tid;
    q = (Ask){};
    if (b < a.B) q = ask_of(a, b);
    int2 all;
    const int2 before = sums_before(make_int2(max(q.old_pages - q.new_pages, 0), 0), wave_sums, all);
    if (b < a.B) {
      first[b] = sum_of(base, before.x);
      who[b] = q.new_pages;
    }
    base = sum_of(base, all.x);
  }
  count = count < 0 ? 0 : (count > a.F ? a.F : count);
  if (base) {
    if (tid == 0) first[a.B] = base;
    __syncthreads();
    // from the last entry to the first, so that taking as many again brings them
    // in the order of the sequences; entries without a page are left out
    // (neighbours in neighbouring threads, one access for a wave's; the next
    // entries are read before these are stored: a load waits for the stores
    // before it)
    int32_t* next[PL_EACH];
    int next_page[PL_EACH];
    auto read = [&](int i0) __attribute__((always_inline)) {
      int at[PL_EACH], own[PL_EACH];
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u) at[u] = base - 1 - i0 - (u * NT + tid);
      owners<PL_EACH>(first, a.B, at, own);
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u) {
        const int b = own[u];
        next[u] = at[u] >= 0 ? a.table + b * a.ldt + who[b] + (at[u] - first[b]) : nullptr;
        next_page[u] = next[u] ? *next[u] : -1;
      }
    };
    read(0);
    for (int i0 = 0; i0 < base; i0 += NT * PL_EACH) {
      int32_t* entry[PL_EACH];
      int page[PL_EACH], rank[PL_EACH];
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u) {
        entry[u] = next[u];
        page[u] = next_page[u];
      }
      if (i0 + NT * PL_EACH < base) read(i0 + NT * PL_EACH);
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u)
        if (entry[u]) *entry[u] = -1;
      // how many pages lie before: in the wave's step, and in those before it
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u) {
        const uint64_t held = __ballot(page[u] >= 0);
        rank[u] = (int)__popcll(held & ((1ull << lane) - 1));
        if (lane == 0) counts[u * waves + wave] = (int)__popcll(held);
      }
      __syncthreads();
      const int held = lane < PL_EACH * waves ? counts[lane] : 0;
      const int sum = lane_sum(held), before = sum - held;
#pragma unroll
      for (int u = 0; u < PL_EACH; ++u) {
        const int64_t at = (int64_t)count + __shfl(before, u * waves + wave) + rank[u];
        if (page[u] >= 0 && at < a.F) a.free[at] = page[u];
      }
      count = (int)min((int64_t)a.F, (int64_t)count + __shfl(sum, 63));
      __syncthreads();
    }
  }
  // who fits, in order, and what those who fit take
  int2 asked = make_int2(0, 0), given = make_int2(0, 0);       // pages, rows
  for (int b0 = 0; b0 < a.B; b0 += NT) {
    const int b = b0 + tid;
    if (a.B > NT) {                                            // (else as above)
      q = (Ask){};
      if (b < a.B) q = ask_of(a, b);
    }
    int2 x = make_int2(0, 0), all;
    if (b < a.B && q.want >= 0)
      x = make_int2(max(q.new_pages - q.old_pages, 0), max(q.want - q.had, 0));
    const int2 before = sums_before(x, wave_sums, all);
    const int p = sum_of(sum_of(asked.x, before.x), x.x), r = sum_of(sum_of(asked.y, before.y), x.y);
    asked = make_int2(sum_of(asked.x, all.x), sum_of(asked.y, all.y));
    const bool served = b < a.B && q.want >= 0 && (x.y == 0 || (p <= count && r <= a.T));
    const int2 y = served ? x : make_int2(0, 0);
    const int2 own = sums_before(y, wave_sums, all);
    if (b < a.B) {
      first[b] = given.x + own.x;
      who[b] = q.old_pages;
      a.q_start[b] = start[b] = given.y + own.y;
      a.seq_len[b] = served ? q.want : q.had;
    }
    given = make_int2(given.x + all.x, given.y + all.y);
  }
  if (tid == 0) {
    first[a.B] = given.x;
    a.q_start[a.B] = start[a.B] = given.y;
    *a.n_free = count - given.x;
  }
  __syncthreads();
  int coming[PL_EACH];
  auto read = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < PL_EACH; ++u)
      coming[u] = i0 + u * NT < given.x ? a.free[count - 1 - i0 - u * NT] : -1;
  };
  read(tid);
  for (int i0 = tid; i0 < given.x; i0 += NT * PL_EACH) {
    int i[PL_EACH], own[PL_EACH], page[PL_EACH];
#pragma unroll
    for (int u = 0; u < PL_EACH; ++u) {
      i[u] = i0 + u * NT;
      page[u] = coming[u];
    }
    if (i0 + NT * PL_EACH < given.x) read(i0 + NT * PL_EACH);
    owners<PL_EACH>(first, a.B, i, own);
#pragma unroll
    for (int u = 0; u < PL_EACH; ++u) {
      if (i[u] >= given.x) break;
      a.table[own[u] * a.ldt + who[own[u]] + (i[u] - first[own[u]])] = page[u];
      a.free[count - 1 - i[u]] = -1;
    }
  }
  if (!rows_too) return;
  __syncthreads();
  for (int row = tid; row < a.T; row += NT) write_slot(a, start, row);
}

__global__ void __launch_bounds__(256) plan_slots_finalize_kernel(PlanArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row < a.T) write_slot(a, a.q_start, (int)row);
}

// ------------------------------------------------------------- verification

constexpr int VD_THREADS = 256;

struct VerifyArgs {
  const int32_t *tokens, *q_start;
  const void *target, *draft;     // draft: or null (a draft's probability is 1)
  const float *uniform, *draw;
  int32_t *accepted, *next;
  double* sums;                   // [B][2][chunks]: of max(p - q, 0), and of p
  int4* stops;                    // [B] where each sequence's drafts end
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

// 16 bytes of a row, which starts at any element.
template <typename T> struct Some {
  static constexpr int N = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// The two weights of a token: of what a rejection leaves, and of the target.
template <typename T> struct Weights {
  static constexpr int N = Some<T>::N;
  const T *p, *q;
  int one;                        // the token that a rejection takes out, where q is null
  bool rejected;
  __device__ __forceinline__ Weights(const VerifyArgs& a, int row, bool rej) : rejected(rej) {
    p = (const T*)a.target + row * a.ldp;
    q = a.draft ? (const T*)a.draft + row * a.ldq : nullptr;
    one = rej && !q ? a.tokens[row + 1] : -1;
  }
  __device__ __forceinline__ void of(int v, double x, double y, double& rest, double& all) const {
    all = weight_of(x);
    rest = rejected ? q ? weight_of(x - y) : v == one ? 0.0 : all : 0.0;
  }
  // E tokens from v on, those from `end` on as if p and q were zero: f(index, p, q).
  template <int E, typename F> __device__ __forceinline__ void load(int v, int end, F f) const {
    static_assert(E % N == 0, "whole loads");
    const bool both = rejected && q;
    if (v + E <= end) {
      typename Some<T>::vec x[E / N], y[E / N] = {};
#pragma unroll
      for (int i = 0; i < E / N; ++i) x[i] = *(const typename Some<T>::vec*)(p + v + i * N);
      if (both) {
#pragma unroll
        for (int i = 0; i < E / N; ++i) y[i] = *(const typename Some<T>::vec*)(q + v + i * N);
      }
#pragma unroll
      for (int i = 0; i < E; ++i)
        f(i, (double)(float)x[i / N][i % N], (double)(float)y[i / N][i % N]);
      return;
    }
    // (the last one's place for those behind it: loads without branches, side by side)
    T x[E], y[E] = {};
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = p[min(v + i, end - 1)];
    if (both) {
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = q[min(v + i, end - 1)];
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool in = v + i < end;
      f(i, in ? (double)(float)x[i] : 0.0, in ? (double)(float)y[i] : 0.0);
    }
  }
  // Both weights: f(index, rest, all).
  template <int E, typename F> __device__ __forceinline__ void each(int v, int end, F f) const {
    load<E>(v, end, [&](int i, double x, double y) __attribute__((always_inline)) {
      double rest, all;
      of(v + i, x, y, rest, all);
      f(i, rest, all);
    });
  }
  // The one that counts (q is zero where none was rejected): f(index, weight).
  template <int E, typename F> __device__ __forceinline__ void chosen(int v, int end, F f) const {
    load<E>(v, end, [&](int i, double x, double y) __attribute__((always_inline)) {
      f(i, v + i == one ? 0.0 : weight_of(x - y));
    });
  }
};

// The sum up to and with this lane's, in a wave (steps as lane_sum's).
template <int CTRL, int ROWS> __device__ __forceinline__ double step_sum(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xf, false);
  return x + __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double sum_up_to(double x) {
  x = step_sum<0x111, 0xf>(x);
  x = step_sum<0x112, 0xf>(x);
  x = step_sum<0x114, 0xf>(x);
  x = step_sum<0x118, 0xf>(x);
  x = step_sum<0x142, 0xa>(x);
  return step_sum<0x143, 0xc>(x);
}

template <typename T>
__global__ void __launch_bounds__(VD_THREADS) verify_sums_kernel(VerifyArgs a) {
  __shared__ double part[2][VD_THREADS / 64];
  const int b = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
  int first;
  bool rejected;
  const int row = stop_of<T>(a, b, first, rejected);
  if (c == 0 && tid == 0) a.stops[b] = make_int4(row, rejected, first, 0);
  if (row < 0) return;
  const Weights<T> w(a, row, rejected);
  const int end = min(a.V, (c + 1) * a.chunk);
  double rest = 0.0, all = 0.0;
  // (one 16-byte load of a row a lane and step, next to its neighbours')
  constexpr int E = Weights<T>::N;
#pragma unroll 4
  for (int v = c * a.chunk + tid * E; v < end; v += VD_THREADS * E)
    w.template each<E>(v, end, [&](int, double x, double y) __attribute__((always_inline)) {
      rest += x;
      all += y;
    });
  rest = sum_up_to(rest);
  all = sum_up_to(all);
  if ((tid & 63) == 63) {
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

// One workgroup per sequence: the chunk that holds the drawn point, from the
// chunks' sums, one a lane; then the token, VD_EACH neighbours a thread: the
// threads' sums in front of each other, and a running sum through the share of
// the one that passes the point.  (One thread's running sums through chunks and
// threads: 24 us for 64 sequences.)
constexpr int VD_EACH = 16;
constexpr int VD_SPAN = VD_THREADS * VD_EACH;

template <typename T>
__global__ void __launch_bounds__(VD_THREADS) verify_finalize_kernel(VerifyArgs a) {
  __shared__ double ends[VD_THREADS / 64];
  __shared__ int hit[VD_THREADS / 64], last[VD_THREADS / 64];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int4 stop = a.stops[b];       // row, whether a draft was rejected there, first row
  const bool some = lane < a.chunks;
  const double* s = a.sums + (int64_t)b * 2 * a.chunks + (some ? lane : 0);
  double mine = s[0], all = s[a.chunks];
  const int row = stop.x;
  if (row < 0) {
    if (tid == 0) {
      a.accepted[b] = 0;
      a.next[b] = -1;
    }
    return;
  }
  mine = some ? mine : 0.0;
  all = some ? all : 0.0;
  const bool rejected = stop.y && __any(mine > 0.0);
  mine = rejected ? mine : all;
  const double upto = sum_up_to(mine);
  const double point = (double)a.draw[b] * __shfl(upto, 63);
  // the first chunk that passes the point; without one (a draw of 1 or more) the
  // last that has any weight
  const uint64_t weighty = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && upto > point);
  int token = -1;
  if (weighty) {
    const int c = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(weighty);
    double run = c ? __shfl(upto, c - 1) : 0.0;
    const Weights<T> w(a, row, rejected);
    const int begin = c * a.chunk, end = min(a.V, begin + a.chunk);
    for (int v0 = begin; v0 < end; v0 += VD_SPAN) {
      double x[VD_EACH], share = 0.0;
      w.template each<VD_EACH>(v0 + tid * VD_EACH, end, [&](int i, double rest, double full)
                                                            __attribute__((always_inline)) {
        x[i] = rejected ? rest : full;
        share += x[i];
      });
      const double up = sum_up_to(share), before = __shfl_up(up, 1);
      if (lane == 63) ends[wave] = up;
      __syncthreads();
      double at = run, total = 0.0;
#pragma unroll
      for (int i = 0; i < VD_THREADS / 64; ++i) {
        at += i < wave ? ends[i] : 0.0;
        total += ends[i];
      }
      at += lane ? before : 0.0;
      // the token that passes the point, and the last of any weight
      int here = -1, heavy = -1;
#pragma unroll
      for (int i = 0; i < VD_EACH; ++i) {
        at += x[i];
        if (x[i] > 0.0) {
          heavy = i;
          if (here < 0 && at > point) here = i;
        }
      }
      const uint64_t passes = __ballot(here >= 0), holds = __ballot(heavy >= 0);
      const int p = passes ? __builtin_ctzll(passes) : 0;
      const int h = holds ? 63 - __builtin_clzll(holds) : 0;
      const int first_here = (wave * 64 + p) * VD_EACH + __shfl(here, p);
      const int last_heavy = (wave * 64 + h) * VD_EACH + __shfl(heavy, h);
      if (lane == 0) {
        hit[wave] = passes ? v0 + first_here : -1;
        last[wave] = holds ? v0 + last_heavy : -1;
      }
      __syncthreads();
      int found = -1;
#pragma unroll
      for (int i = 0; i < VD_THREADS / 64; ++i) {
        if (last[i] >= 0) token = last[i];
        if (found < 0) found = hit[i];
      }
      if (found >= 0) {
        token = found;
        break;
      }
      run += total;
      __syncthreads();
    }
  }
  if (tid == 0) {
    a.accepted[b] = row - stop.z;
    a.next[b] = token;
  }
}

// A row of at most VD_ROW tokens by one workgroup, in one launch: sums of
// neighbours by thread, then the thread that holds the drawn point goes through
// its share once more.  (Longer rows are too much work in 64 bits for one CU: 4000
// tokens take 8.1 us so and 8.8 in two launches, which cost the caller 3 us more;
// 8000 took 10.9 and 9.8, 32000 15 and 9.)
constexpr int VD_MOST = 512, VD_LANE = 8, VD_ROW = VD_MOST * VD_LANE;

template <typename T>
__global__ void __launch_bounds__(VD_MOST) verify_row_kernel(VerifyArgs a) {
  __shared__ double ends[VD_MOST / 64];
  __shared__ int hit, last;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int first;
  bool rejected;
  const int row = stop_of<T>(a, b, first, rejected);
  if (tid == 0) {
    a.accepted[b] = row < 0 ? 0 : row - first;
    if (row < 0) a.next[b] = -1;
    hit = INT32_MAX;
    last = -1;
  }
  if (row < 0) return;
  Weights<T> w(a, row, rejected);
  double x[VD_LANE], share, up, from, total;
  for (;;) {
    share = 0.0;
    w.template chosen<VD_LANE>(tid * VD_LANE, a.V, [&](int i, double y) __attribute__((always_inline)) {
      x[i] = y;
      share += y;
    });
    up = sum_up_to(share);
    if (lane == 63) ends[wave] = up;
    __syncthreads();
    from = total = 0.0;
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
      from = i == wave ? total : from;
      total += ends[i];
    }
    if (!w.rejected || total > 0.0) break;
    w = Weights<T>(a, row, false);                     // (p <= q everywhere: from p)
    __syncthreads();
  }
  const double point = (double)a.draw[b] * total, in = __shfl_up(up, 1);
  if (share > 0.0) {
    atomicMax(&last, tid);
    if (from + up > point) atomicMin(&hit, tid);
  }
  __syncthreads();
  const int who = hit < INT32_MAX ? hit : last;
  if (who < 0 && tid == 0) a.next[b] = -1;
  if (tid != who) return;
  // the token that passes the point, or the last of any weight
  double at = from + (lane ? in : 0.0);
  int here = -1, heavy = 0;
#pragma unroll
  for (int i = 0; i < VD_LANE; ++i) {
    at += x[i];
    if (x[i] > 0.0) {
      heavy = i;
      if (here < 0 && at > point) here = i;
    }
  }
  a.next[b] = tid * VD_LANE + (here >= 0 ? here : heavy);
}

// Elements of a row that one workgroup sums: 4096 and more, a power of two, in
// at most 64 chunks.
void verify_chunks(int64_t V, int& chunk, int& chunks) {
  int64_t c = 4096;
  while (c * 64 < V) c *= 2;
  chunk = (int)c;
  chunks = (int)((V + c - 1) / c);
}

size_t verify_bytes(int64_t V, int64_t B, int chunks) {
  if (V <= VD_ROW) return 0;
  return align256((size_t)B * sizeof(int4)) + align256((size_t)B * 2 * chunks * sizeof(double));
}

gsrq_status verify_shape(int64_t T, int64_t V, int64_t B) {
  if (T < 0 || V < 1 || B < 1) return GSRQ_E_ARG;
  if (T > INT32_MAX / 2 || V > INT32_MAX / 2 || B > (1 << 16)) return GSRQ_E_UNSUPPORTED;
  return GSRQ_OK;
}

template <typename T> gsrq_status verify_launch(const VerifyArgs& a, hipStream_t st) {
  TimedLaunch tl(GSRQ_KERNEL_SERVING, st);
  if (a.V <= VD_ROW) {
    const int threads = ((a.V + VD_LANE - 1) / VD_LANE + 63) / 64 * 64;
    verify_row_kernel<T><<<(unsigned)a.B, threads, 0, st>>>(a);
    return launch_ok();
  }
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
  // (a round of moved entries behind the last is still counted in 32 bits)
  if (s->B > PL_MOST || s->T > INT32_MAX / 2 ||
      (int64_t)s->B * s->per > INT32_MAX - PL_THREADS * PL_EACH)
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
  // as many threads as there are sequences, or rows that are written too
  const bool one = s->T <= 2 * PL_THREADS;
  const int64_t work = std::max<int64_t>(s->B, one ? s->T : s->T / s->page_size);
  int threads = 64;
  while (threads < PL_THREADS && threads < work) threads *= 2;
  plan_update_kernel<<<1, threads, 0, st>>>(a, one);
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
  *bytes = verify_bytes(V, B, chunks);
  return GSRQ_OK;
}

gsrq_status gsrq_verify_drafts(int64_t T, int64_t V, int32_t B, const int32_t* tokens,
                               const void* target, int64_t ldp, const void* draft, int64_t ldq,
                               gsrq_dtype dtype, const float* uniform, const float* draw,
                               const int32_t* q_start, int32_t* accepted, int32_t* next,
                               void* workspace, size_t ws_bytes, void* stream) {
  gsrq_status e = verify_shape(T, V, B);
  if (e) return e;
  if (!q_start || !draw || !accepted || !next) return GSRQ_E_ARG;
  if (T > 0 && (!tokens || !target || !uniform)) return GSRQ_E_ARG;
  if (T > 1 && (ldp < V || (draft && ldq < V))) return GSRQ_E_ARG;
  if (dtype != GSRQ_F32 && dtype != GSRQ_F16 && dtype != GSRQ_BF16) return GSRQ_E_ARG;
  const uintptr_t esz = dtype == GSRQ_F32 ? 4 : 2;
  if ((uintptr_t)target % esz || (uintptr_t)draft % esz) return GSRQ_E_ARG;
  VerifyArgs a;
  verify_chunks(V, a.chunk, a.chunks);
  const size_t bytes = verify_bytes(V, B, a.chunks);
  if (bytes && (!workspace || (uintptr_t)workspace % 256)) return GSRQ_E_ARG;
  if (ws_bytes < bytes) return GSRQ_E_WORKSPACE;
  a.tokens = tokens;
  a.q_start = q_start;
  a.target = target;
  a.draft = draft;
  a.uniform = uniform;
  a.draw = draw;
  a.accepted = accepted;
  a.next = next;
  a.stops = (int4*)workspace;
  a.sums = (double*)((char*)workspace + align256((size_t)B * sizeof(int4)));
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
