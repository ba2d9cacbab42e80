// The paged cache in 8 bits on AMD MI355X (gfx950): appending new tokens, and
// attention over the pages.
//
// A code c (e4m3) of page g and head h stands for c 2^e[g][h].
//
// Appending.  With y a new token's key after norm and rotation (or its value),
// and a the largest |y| of the page's new tokens in a head,
//   e = min { e >= -40 : a <= 448 2^e }, at least the exponent before unless
//   the page starts anew;   code = rne(y 2^-e).
// A workgroup owns the new tokens of one page in some heads, of the keys or of
// the values, so that the largest |y| is known before anything is written.
//
// Attention.  As over 16-bit pages (two kinds of workgroups, transposed
// products, pieces joined by a second launch); with the scales out of the
// products: for the codes c of keys and d of values, and their exponents,
//   s_j = (scale 2^ek) q . c_j,   o = sum_j w_j d_j / sum_j w_j 2^-ev,
//   w_j = 2^(s_j log2(e) + ev - m + 6),   m = a running maximum of s_j log2(e) + ev.
// One subtraction and one factor per page and tile take the place of a product
// per element.  m is raised only by a tile that exceeds it by 2^8, so w_j is at
// most 2^14 whatever the scales (float16 ends at 65504), and its float16 rounding is
// relative to the largest product of weight and scale.  Codes are exact in
// float16 and bfloat16.
#include "gsrq_attn_paged.h"

namespace {

constexpr int E8_THREADS = 256;

struct PageExps {
  int8_t *k, *v;
  int64_t ks[2], vs[2];     // page, head
};

__device__ __forceinline__ int held_exp(int e) {
  return e < GSRQ_EXP_MIN ? GSRQ_EXP_MIN : (e > GSRQ_EXP_MAX ? GSRQ_EXP_MAX : e);
}

// The smallest e of the range with a <= 448 2^e, a >= 0.
template <typename F> __device__ __forceinline__ int exp_for(F a) {
  if (!(a > 0)) return GSRQ_EXP_MIN;
  int e;
  const F m = frexp(a, &e);               // a = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
  return held_exp(e - 9 + (m > (F)0.875));
}

__device__ __forceinline__ float pow2(int e) {      // (normal numbers)
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// --------------------------------------------------------------- appending

// Four numbers as codes: to the nearest, ties to even, beyond 448 held there;
// infinities and NaN become NaN (the conversion alone would make NaN of
// numbers beyond 448).
__device__ __forceinline__ uint32_t codes4(float x0, float x1, float x2, float x3) {
  const float in[4] = {x0, x1, x2, x3};
  float x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    x[j] = is_finite(in[j]) ? __builtin_amdgcn_fmed3f(in[j], -448.f, 448.f) : NAN;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
}

struct Append8Args {
  PagePool pool;
  PageExps exps;
  const void *k, *v, *q;
  int64_t kst[2], vst[2], qst[2];     // token, head
  const int32_t *q_start, *seq_len;
  const double* theta;
  const float *k_norm, *q_norm;
  void* q_out;
  int T, Hq;
  int HG, groups;                     // heads per workgroup, and groups of so many
  int rows;                           // tokens of a workgroup of queries
  int64_t page_wgs;                   // workgroups of pages; the others turn queries
  float eps;
};

// Page slot: sequence b owns the slots from its first row's on; n rows touch at
// most n / page_size + 2 pages.
__device__ __forceinline__ int64_t page_slot_of(const Append8Args& a, int b) {
  const int q = a.q_start[b];
  return (int64_t)((q < 0 ? 0 : (q > a.T ? a.T : q)) >> a.pool.shift) + 2 * (int64_t)b;
}

// A head's 16 elements of one lane: 8 of the lower half and the 8 they are turned
// with.  As they come (two or four registers for four elements), and as numbers.
template <typename TI> struct Raw {
  typedef u4 part[sizeof(TI) == 4 ? 2 : 1];
  part lo, hi;
  __device__ __forceinline__ void load(const TI* src, int half) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(part) / 16); ++i) {
      lo[i] = ((const u4*)src)[i];
      hi[i] = ((const u4*)(src + half))[i];
    }
  }
  __device__ __forceinline__ void get(float (&x)[8], float (&y)[8]) const {
    load8((const TI*)&lo, x);
    load8((const TI*)&hi, y);
  }
};

template <typename F> __device__ __forceinline__ void turned(F& lo, F& hi, F c, F s) {
  const F x = lo, y = hi;
  lo = x * c - y * s;
  hi = y * c + x * s;
}

// The turns of a lane's 8 pairs at a token of a page: those of each eighth token
// and of the eight steps from it on come from LDS, a product of two for each
// token (keys and values of 25540 rows, 8 heads, pages of 64 tokens: 75 us with a
// sine and cosine for each, 52 so).  The angle is still that of 64 bits, c and s
// carry six roundings.
struct Turns {
  float c[8], s[8];
  __device__ __forceinline__ void at(int64_t pos, const double* theta) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      turn_of(pos, theta[j], c[j], s[j]);
      __builtin_amdgcn_sched_barrier(0);             // (one after another: in few registers)
    }
  }
  __device__ __forceinline__ void from(const float2* far, const float2* near) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 x = far[j], y = near[j];
      c[j] = x.x * y.x - x.y * y.y;
      s[j] = x.y * y.x + x.x * y.y;
    }
  }
};

__device__ __forceinline__ float finite_size(float x) { return is_finite(x) ? fabsf(x) : 0.f; }

// What an append workgroup of a page works on.
template <typename TI> struct PageRows {
  const TI* src;                  // the first new token's first head
  uint8_t* dst;                   // its page's first place there
  int64_t st0, st1, ps1, ps2;     // rows: token, head; places: token, head
  const double* theta;            // or null
  const float* norm;              // or null
  int64_t pos;                    // of the first new token
  float eps;
  int tokens, heads, kept;        // new tokens, heads, tokens of the page before them
};

// The largest size of the page's elements by heads, in 64 bits; for a whole
// workgroup, which has set top64 to zeros.  (Rare: one pair of elements at a
// time, so that it asks for few registers.)
template <typename TI, int HD>
__device__ __forceinline__ void exact_sizes(const PageRows<TI>& w, unsigned long long* top64) {
  constexpr int L = HD / 16;
  const int l = threadIdx.x % L;
  for (int i = threadIdx.x / L; i < w.tokens * w.heads; i += E8_THREADS / L) {
    const int h = i % w.heads, t = i / w.heads;
    const TI* src = w.src + t * w.st0 + h * w.st1;
    double r = 1.0, m = 0.0;
    if (w.norm) {
      Raw<TI> x;
      float lo[8], hi[8];
      x.load(src + 8 * l, HD / 2);
      x.get(lo, hi);
      r = 1.0 / sqrt(sum_of_squares<double, HD>(lo, hi) * (1.0 / HD) + (double)w.eps);
    }
#pragma unroll 1
    for (int j = 8 * l; j < 8 * l + 8; ++j) {
      double x = (double)(float)src[j], y = (double)(float)src[j + HD / 2];
      if (w.norm) {
        x *= r * (double)w.norm[j];
        y *= r * (double)w.norm[j + HD / 2];
      }
      if (w.theta) {
        double a = (double)(w.pos + t) * (w.theta[j] * 0.15915494309189533577), s, c;
        a -= rint(a);
        sincospi(2.0 * a, &s, &c);
        turned(x, y, c, s);
      }
      if (is_finite((float)x)) m = fmax(m, fabs(x));
      if (is_finite((float)y)) m = fmax(m, fabs(y));
    }
    atomicMax(&top64[h], (unsigned long long)__double_as_longlong(m));
  }
}

// Items of a page workgroup: a row (token and head) for L lanes, E8_KEEP of them
// a thread at most where they are kept in registers from the search for the
// largest size to the rounding; a thread's items share their token as far as
// they can, so that its 8 sines and cosines serve several heads.
constexpr int E8_KEEP = 4;

template <typename TI, int HD>
__device__ __forceinline__ void append_page(const Append8Args& a, int64_t wg) {
  constexpr int L = HD / 16, RP = E8_THREADS / L;             // lanes of a row, rows at once
  __shared__ uint32_t top[E8_THREADS];                        // bits of the largest sizes, by head
  __shared__ unsigned long long top64[E8_THREADS];
  __shared__ int was[E8_THREADS], now[E8_THREADS];
  __shared__ int close, risen;
  constexpr int HALF = HD / 2, EIGHTHS = E8_KEEP * RP / 8;    // (of the most tokens that are kept)
  __shared__ float2 far[EIGHTHS][HALF], near[8][HALF];
  __shared__ float weight[HD];                                // of the norm
  const int tid = threadIdx.x, lane = tid & 63, l = tid % L, row = tid / L;
  const int sub = (int)(wg % (2 * a.groups));
  const int64_t slot = wg / (2 * a.groups);
  const bool key = sub < a.groups;
  const int h0 = (key ? sub : sub - a.groups) * a.HG;
  int b = 0;
  for (int i = 0; i < a.pool.B; i += 64) {
    const bool done = i + lane < a.pool.B && page_slot_of(a, i + lane + 1) <= slot;
    b += (int)__popcll(__ballot(done));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  if (b >= a.pool.B) return;
  int first, n;
  new_rows(a.q_start, b, a.T, first, n);
  const int64_t pos0 = (int64_t)a.seq_len[b] - n;
  const int64_t from = pos0 < 0 ? 0 : pos0;
  const int64_t index = (from >> a.pool.shift) + (slot - page_slot_of(a, b));
  const int64_t begin = max(from, index << a.pool.shift);
  const int64_t end = min(pos0 + n, (index + 1) << a.pool.shift);
  if (begin >= end) return;
  // (the page is looked up while the rows are on their way)
  const int64_t in_row = begin >> a.pool.shift;
  const int entry = in_row < a.pool.per ? a.pool.table[b * a.pool.ldt + in_row] : -1;
  const int64_t* st = key ? a.kst : a.vst;
  const int64_t* ps = key ? a.pool.ks : a.pool.vs;
  const int64_t* es = key ? a.exps.ks : a.exps.vs;
  PageRows<TI> w;
  w.src = (const TI*)(key ? a.k : a.v) + (first + (begin - pos0)) * st[0] + h0 * st[1];
  w.st0 = st[0]; w.st1 = st[1]; w.ps1 = ps[1]; w.ps2 = ps[2];
  w.theta = key ? a.theta : nullptr;
  w.norm = key ? a.k_norm : nullptr;
  w.pos = begin;
  w.eps = a.eps;
  w.tokens = (int)(end - begin);
  w.heads = min(a.HG, a.pool.Hkv - h0);
  w.kept = (int)(begin & ((1 << a.pool.shift) - 1));

  // item i of this thread; whether there is one (whole for its L lanes)
  const bool wide = w.tokens <= RP;
  const int beside = wide ? RP / w.tokens : 1;                // heads side by side
  const int token0 = wide ? row % w.tokens : row, head0 = wide ? row / w.tokens : 0;
  const int items = wide ? (w.heads + beside - 1) / beside : w.heads * ((w.tokens + RP - 1) / RP);
  auto item = [&](int i, int& t, int& h) __attribute__((always_inline)) {
    t = wide ? token0 : token0 + RP * (i / w.heads);
    h = wide ? head0 + i * beside : i % w.heads;
    return i < items && t < w.tokens && h < w.heads && (!wide || head0 < beside);
  };
  // `factor`: of the norm, taken where it is `unknown` (or below zero)
  auto numbers_of = [&](const Raw<TI>& x, int t, int& turned_to, Turns& turns, bool kept,
                        bool unknown, float& factor, float (&lo)[8], float (&hi)[8])
                        __attribute__((always_inline)) {
    asm volatile("" : : : "memory");                   // (weights are read anew, not kept in registers)
    x.get(lo, hi);
    if (w.norm) {
      bool scaled = false;
      if (unknown || factor < 0.f) factor = norm_factor<HD>(lo, hi, w.eps, scaled);
      const float r = factor;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[j] *= r * weight[8 * l + j];
        hi[j] *= r * weight[HALF + 8 * l + j];
      }
      if (scaled) factor = -1.f;                       // (taken anew, with the elements' scaling)
    }
    if (w.theta) {
      if (t != turned_to) {
        if (kept) turns.from(&far[t / 8][8 * l], &near[t % 8][8 * l]);
        else turns.at(w.pos + t, w.theta + 8 * l);
      }
      turned_to = t;
#pragma unroll
      for (int j = 0; j < 8; ++j) turned(lo[j], hi[j], turns.c[j], turns.s[j]);
    }
  };
  auto search = [&](int h, const float (&lo)[8], const float (&hi)[8]) __attribute__((always_inline)) {
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fmaxf(finite_size(lo[j]), finite_size(hi[j])));
#pragma unroll
    for (int x = 1; x < L; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
    if (l == 0) atomicMax(&top[h], __float_as_uint(m));
  };
  auto round = [&](int t, int h, const float (&lo)[8], const float (&hi)[8])
                   __attribute__((always_inline)) {
    const float f = pow2(-now[h]);
    uint8_t* to = w.dst + (w.kept + t) * w.ps1 + h * w.ps2 + 8 * l;
    uint2 x, y;
    x.x = codes4(lo[0] * f, lo[1] * f, lo[2] * f, lo[3] * f);
    x.y = codes4(lo[4] * f, lo[5] * f, lo[6] * f, lo[7] * f);
    y.x = codes4(hi[0] * f, hi[1] * f, hi[2] * f, hi[3] * f);
    y.y = codes4(hi[4] * f, hi[5] * f, hi[6] * f, hi[7] * f);
    *(uint2*)to = x;
    *(uint2*)(to + HD / 2) = y;
  };

  Raw<TI> kept[E8_KEEP];
  const bool keep = items <= E8_KEEP;
  if (keep) {
#pragma unroll
    for (int i = 0; i < E8_KEEP; ++i) {
      int t, h;
      if (item(i, t, h)) kept[i].load(w.src + t * w.st0 + h * w.st1 + 8 * l, HD / 2);
    }
  }
  const int page = checked(a.pool, entry);
  if (page < 0) return;
  w.dst = (uint8_t*)(key ? a.pool.k : a.pool.v) + page * ps[0] + h0 * ps[2];
  int8_t* exps = (key ? a.exps.k : a.exps.v) + page * es[0] + h0 * es[1];
  for (int h = tid; h < w.heads; h += E8_THREADS) {
    top[h] = 0;
    top64[h] = 0;
    was[h] = held_exp(exps[h * es[1]]);
  }
  if (tid == 0) close = risen = 0;
  if (w.norm && tid < HD) weight[tid] = w.norm[tid];
  if (keep && w.theta) {
    const int eighths = (w.tokens + 7) / 8, all = eighths + min(8, w.tokens);
    for (int i = tid; i < all * HALF; i += E8_THREADS) {
      const int j = i % HALF, t = i / HALF;
      float2* to = t < eighths ? &far[t][j] : &near[t - eighths][j];
      turn_of(t < eighths ? w.pos + 8 * t : t - eighths, w.theta[j], to->x, to->y);
    }
  }
  __syncthreads();
  float factor[E8_KEEP];
  Turns turns;
  int turned_to = -1;
  float lo[8], hi[8];
  if (keep) {
#pragma unroll
    for (int i = 0; i < E8_KEEP; ++i) {
      int t, h;
      if (item(i, t, h)) {
        numbers_of(kept[i], t, turned_to, turns, true, true, factor[i], lo, hi);
        search(h, lo, hi);
      }
    }
  } else {
    for (int i = 0; i < items; ++i) {
      int t, h;
      if (!item(i, t, h)) continue;
      Raw<TI> x;
      x.load(w.src + t * w.st0 + h * w.st1 + 8 * l, HD / 2);
      numbers_of(x, t, turned_to, turns, false, true, factor[0], lo, hi);
      search(h, lo, hi);
    }
  }
  __syncthreads();
  // An exponent that the roundings of norm and rotation (2^-19 of a, at the most)
  // could change is taken from 64-bit numbers.
  for (int h = tid; h < w.heads; h += E8_THREADS) {
    const float m = __uint_as_float(top[h]);
    now[h] = exp_for(m);
    if ((w.norm || w.theta) && exp_for(m * (1.f - 0x1p-18f)) != exp_for(m * (1.f + 0x1p-18f)))
      close = 1;
  }
  __syncthreads();
  if (close) {
    exact_sizes<TI, HD>(w, top64);
    __syncthreads();
  }
  for (int h = tid; h < w.heads; h += E8_THREADS) {
    int e = close ? exp_for(__longlong_as_double((long long)top64[h])) : now[h];
    if (w.kept && was[h] > e) e = was[h];
    if (w.kept && e > was[h]) risen = 1;
    now[h] = e;
    exps[h * es[1]] = (int8_t)e;
  }
  __syncthreads();
  if (keep) {
#pragma unroll
    for (int i = 0; i < E8_KEEP; ++i) {
      int t, h;
      if (item(i, t, h)) {
        numbers_of(kept[i], t, turned_to, turns, true, false, factor[i], lo, hi);
        round(t, h, lo, hi);
      }
    }
  } else {
    for (int i = 0; i < items; ++i) {
      int t, h;
      if (!item(i, t, h)) continue;
      Raw<TI> x;
      x.load(w.src + t * w.st0 + h * w.st1 + 8 * l, HD / 2);
      numbers_of(x, t, turned_to, turns, false, true, factor[0], lo, hi);
      round(t, h, lo, hi);
    }
  }
  if (risen) {                    // the tokens before: their codes under the new scale
    constexpr int N = HD / 16;
    for (int i = tid; i < w.kept * w.heads * N; i += E8_THREADS) {
      const int c = i % N, h = i / N % w.heads, t = i / N / w.heads;
      if (now[h] == was[h]) continue;
      const float f = pow2(was[h] - now[h]);
      u4* at = (u4*)(w.dst + t * w.ps1 + h * w.ps2 + 16 * c);
      u4 x = *at;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const auto p = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[j], false);
        const auto q = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[j], true);
        x[j] = codes4(p[0] * f, p[1] * f, q[0] * f, q[1] * f);
      }
      *at = x;
    }
  }
}

// Queries: E8_ROWS tokens (or one), a row of lanes per head.  All their loads are
// on the way while the threads share the sines and cosines out among themselves.
constexpr int E8_ROWS = 4;

template <typename TI, typename TQ, int HD>
__device__ __forceinline__ void append_queries(const Append8Args& a, int64_t wg) {
  constexpr int L = HD / 16, RP = E8_THREADS / L, HALF = HD / 2;
  __shared__ float2 turns[E8_ROWS][HALF];
  const int tid = threadIdx.x, l = tid % L;
  const int per = (a.Hq + RP - 1) / RP;
  const int row0 = (int)(wg / per) * a.rows, h = (int)(wg % per) * RP + tid / L;
  const int rows = min(a.rows, a.T - row0);
  const bool mine = h < a.Hq;
  Raw<TI> x[E8_ROWS];
  int64_t pos[E8_ROWS];
#pragma unroll
  for (int i = 0; i < E8_ROWS; ++i)
    if (mine && i < rows)
      x[i].load((const TI*)a.q + (row0 + i) * a.qst[0] + h * a.qst[1] + 8 * l, HALF);
#pragma unroll
  for (int i = 0; i < E8_ROWS; ++i) {
    pos[i] = INT64_MIN;                                // a row of no sequence
    const int b = i < rows ? sequence_of(a.q_start, a.pool.B, row0 + i) : -1;
    if (b < 0) continue;
    int first, n;
    new_rows(a.q_start, b, a.T, first, n);
    pos[i] = (int64_t)a.seq_len[b] - n + (row0 + i - first);
  }
  if (a.theta) {
#pragma unroll
    for (int i = 0; i < E8_ROWS; ++i)                  // (HALF divides 256: a thread's pairs are all one)
      if (i % (E8_THREADS / HALF) == tid / HALF && pos[i] != INT64_MIN)
        turn_of(pos[i], a.theta[tid % HALF], turns[i][tid % HALF].x, turns[i][tid % HALF].y);
    __syncthreads();
  }
  if (!mine) return;
#pragma unroll
  for (int i = 0; i < E8_ROWS; ++i) {
    if (pos[i] == INT64_MIN) continue;
    float lo[8], hi[8];
    x[i].get(lo, hi);
    if (a.q_norm) {
      bool scaled;
      const float r = norm_factor<HD>(lo, hi, a.eps, scaled);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[j] *= r * a.q_norm[8 * l + j];
        hi[j] *= r * a.q_norm[HALF + 8 * l + j];
      }
    }
    if (a.theta) {
#pragma unroll
      for (int j = 0; j < 8; ++j) turned(lo[j], hi[j], turns[i][8 * l + j].x, turns[i][8 * l + j].y);
    }
    TQ* dst = (TQ*)a.q_out + ((int64_t)(row0 + i) * a.Hq + h) * HD + 8 * l;
    store8(dst, lo);
    store8(dst + HALF, hi);
  }
}

template <typename TI, typename TQ, int HD>
__global__ void __launch_bounds__(E8_THREADS, sizeof(TI) == 4 ? 3 : 4) cache8_append_kernel(Append8Args a) {
  if ((int64_t)blockIdx.x < a.page_wgs) append_page<TI, HD>(a, blockIdx.x);
  else append_queries<TI, TQ, HD>(a, (int64_t)blockIdx.x - a.page_wgs);
}

// --------------------------------------------------------------- attention

struct Pt8Args {
  PtArgs p;
  PageExps exps;
};

// Eight codes as numbers of the queries' type.
template <typename T>
__device__ __forceinline__ typename Vec<T>::v8 numbers(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ h8 numbers<_Float16>(uint32_t a, uint32_t b) {
  const auto x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, false);
  const auto y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, true);
  const auto z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, false);
  const auto w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, true);
  const auto lo = __builtin_shufflevector(x, y, 0, 1, 2, 3), hi = __builtin_shufflevector(z, w, 0, 1, 2, 3);
  return __builtin_bit_cast(h8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <> __device__ __forceinline__ b8 numbers<__bf16>(uint32_t a, uint32_t b) {
  const auto x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.f, false);
  const auto y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.f, true);
  const auto z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.f, false);
  const auto w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.f, true);
  return (b8){x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// 0xff in the bytes of a word that hold NaN codes.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) {
  return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu;
}
// Takes the NaN out of 16 codes; whether there were any.
__device__ __forceinline__ bool without_nan(u4& x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = nan_codes(x[i]);
    any |= m;
    x[i] &= ~m;
  }
  return any != 0;
}

// Places of a tile's 16-byte chunk c of row r in LDS, as codes: rows of a key
// tile are read 32 at a time at one chunk, rows of a value tile eight at a time
// at two neighbouring chunks, both without bank conflicts in these orders.
template <int HD> __device__ __forceinline__ int key_chunk8(int r, int c) {
  return c ^ (HD == 64 ? (r >> 2) & 3 : HD == 128 ? (r >> 1) & 7 : r & 15);
}
template <int HD> __device__ __forceinline__ int value_chunk8(int r, int c) {
  return c ^ 2 * (HD == 64    ? (r >> 3) & 1
                  : HD == 128 ? ((r >> 1) & 1) | ((r >> 2) & 2)
                              : (r & 3) | ((r >> 1) & 4));
}

// Scales of a tile's groups of eight keys, the same for the whole wave: the
// factor of a score (log2), and the values' exponent.
template <int NB> struct Groups {
  float ck[4 * NB], ev[4 * NB], iv[4 * NB];           // iv: 2^-ev
};

// The same, of one page, for the lane that looks it up.
struct PageScale {
  float ck;
  int ev;
};
__device__ __forceinline__ PageScale page_scale(const Pt8Args& a, int head, int page) {
  int k = 0, v = 0;
  if (page >= 0) {
    k = held_exp(a.exps.k[page * a.exps.ks[0] + head * a.exps.ks[1]]);
    v = held_exp(a.exps.v[page * a.exps.vs[0] + head * a.exps.vs[1]]);
  }
  // (a factor above zero: -inf times zero would be NaN)
  return {fmaxf(a.p.c * pow2(k), 1.17549435e-38f), v};
}
// Those of a tile whose first group lane `first` has looked up.
template <int NB>
__device__ __forceinline__ Groups<NB> groups_from(const PageScale& x, int first) {
  Groups<NB> g;
#pragma unroll
  for (int j = 0; j < 4 * NB; ++j) {
    const int ev = __builtin_amdgcn_readlane(x.ev, first + j);
    g.ck[j] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x.ck), first + j));
    g.ev[j] = (float)ev;
    g.iv[j] = pow2(-ev);
  }
  return g;
}

// The largest of four products' sums (as max16).
__device__ __forceinline__ float max4(float a, float b, float c, float d) {
  float r = __builtin_amdgcn_fmed3f(a, b, INFINITY);
  asm("v_max3_f32 %0, %0, %1, %2" : "+v"(r) : "v"(c), "v"(d));
  return r;
}

template <typename T, int HD> struct Columns8 : Columns<T, HD> {
  typedef Columns<T, HD> Base;
  typedef typename Base::v8 v8;
  using Base::DT;
  using Base::l;
  using Base::m;
  using Base::o;
  using Base::q;
  using Base::see_hi;
  using Base::see_lo;

  // Scores of NB blocks of 32 keys in LDS, as codes (queries PAIRED).
  template <int NB>
  __device__ __forceinline__ void scores8(const char* kt, f16v (&sc)[NB]) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 32; ++k)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int row = 32 * n + col;
        const u4 x = *(const u4*)(kt + row * HD + 16 * key_chunk8<HD>(row, 2 * k + half));
        sc[n] = Vec<T>::mfma(numbers<T>(x[0], x[1]), q[2 * k], sc[n]);
        sc[n] = Vec<T>::mfma(numbers<T>(x[2], x[3]), q[2 * k + 1], sc[n]);
      }
  }

  template <int NB>
  __device__ __forceinline__ void settle8(int t0, uint64_t absent, const Groups<NB>& g,
                                          f16v (&sc)[NB]) {
    this->template mask<NB>(t0, absent, sc);
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        top = fmaxf(top, fmaf(max4(sc[n][4 * j], sc[n][4 * j + 1], sc[n][4 * j + 2], sc[n][4 * j + 3]),
                              g.ck[4 * n + j], g.ev[4 * n + j]));
    const float2 tops = both_halves(top);
    top = fmaxf(tops.x, tops.y);
    const bool past = top > m + PT_HEADROOM;
    if (__any(past)) {
      const float f = past ? __builtin_amdgcn_exp2f(m - top) : 1.f;
      m = past ? top : m;
      l *= f;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= f;
    }
  }

  template <int NB>
  __device__ __forceinline__ void weights8(const Groups<NB>& g, const f16v (&sc)[NB],
                                           v8 (&p)[NB][2]) {
    const float sub = m == -INFINITY ? 0.f : PT_SHIFT - m;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float ck = g.ck[4 * n + j], ev = g.ev[4 * n + j], base = sub + ev;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(sc[n][4 * j + e], ck, base));
          p[n][j / 2][4 * (j % 2) + e] = (T)x[e];
        }
        l = fmaf((x[0] + x[1]) + (x[2] + x[3]), g.iv[4 * n + j], l);
      }
  }

  template <int NB>
  __device__ __forceinline__ void add_values8(const char* vt, const v8 (&p)[NB][2]) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] = Vec<T>::mfma(values8(vt, n, k, t), p[n][k], o[t]);
  }

  // V^T of 32 dimensions and the 16 tokens of weights [n][k], in their order:
  // each 16 lanes read eight rows of 16 codes and get a column each.
  static __device__ __forceinline__ v8 values8(const char* vt, int n, int k, int t) {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63, half = lane >> 5, e = (lane & 15) >> 1;
    const int row = 32 * n + 16 * k + 4 * half + (e & 3) + 8 * (e >> 2);
    const int ch = 2 * t + ((lane >> 4) & 1);
    const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (__attribute__((address_space(3))) v2i*)(lds_char*)(vt + row * HD +
                                                            16 * value_chunk8<HD>(row, ch) +
                                                            8 * (lane & 1)));
    return numbers<T>((uint32_t)x[0], (uint32_t)x[1]);
  }

  // NaN among the values of `rows` keys every `step` from `from` to `to`, for
  // the queries that see them (without_nan() has taken them out).
  __device__ __forceinline__ void see_nan(const Pt8Args& a, int b, int head, int from, int to,
                                          int step, int rows) {
    const PagePool& pool = a.p.pool;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const auto value = [&](int page, int j) __attribute__((always_inline)) {
      return (const uint8_t*)pool.v + page * pool.vs[0] +
             (int64_t)(j & ((1 << pool.shift) - 1)) * pool.vs[1] + head * pool.vs[2];
    };
    for (int t0 = from; t0 <= to; t0 += step) {
      // one key a lane: whether it holds any
      const int mine = lane < rows ? page_of(pool, b, t0 + lane) : -1;
      bool odd = false;
      if (mine >= 0) {
        const uint8_t* v = value(mine, t0 + lane);
#pragma unroll 4
        for (int c = 0; c < HD / 16; ++c) {
          u4 x = *(const u4*)(v + 16 * c);
          odd = without_nan(x) || odd;
        }
      }
      for (uint64_t todo = __ballot(odd); todo; todo &= todo - 1) {
        const int j = t0 + __builtin_ctzll(todo);
        const uint8_t* v = value(__builtin_amdgcn_readlane(mine, j - t0), j) + 4 * half;
        const bool seen = j < see_hi && j >= see_lo;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = nan_codes(*(const uint32_t*)(v + 32 * t + 8 * i));
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[t][4 * i + e] += seen && (x >> (8 * e) & 1u) ? NAN : 0.f;
          }
      }
    }
  }
};

// Where a lane's token lies from its head's first key (or value) on (bytes); an
// absent page counts as the pool's first, which nobody looks at.
__device__ __forceinline__ uint64_t token_offset8(const PagePool& p, const int64_t (&st)[3],
                                                  int page, int t) {
  const uint32_t in = page < 0 ? 0 : t & ((1 << p.shift) - 1);
  return (uint64_t)(uint32_t)(page < 0 ? 0 : page) * (uint32_t)st[0] +
         (uint64_t)in * (uint32_t)st[1];
}

// The 64 HD / 16 rows of a wave's load, a lane its row and 16-byte chunk, from
// the offset that lane `row` holds: eight rows lie in one page, and where the
// load has 16 (heads of 64) the lane `next` holds that of the other eight.
template <int HD>
__device__ __forceinline__ const char* row_of_load(const char* base, uint64_t offset, int row,
                                                   int next, uint32_t within) {
  const char* at = rows_at(base, offset, row);
  if (HD == 64) {
    const char* second = rows_at(base, offset, next);
    at = threadIdx.x & 32 ? second : at;
  }
  return at + within;
}

// The rows of a tile that are not there: by groups of eight (bits of `groups`),
// and behind the `left` that it has.
template <int ROWS> __device__ __forceinline__ uint64_t gone_rows(uint32_t groups, int left) {
  uint64_t held = ((groups & 15u) * 0x00204081u & 0x01010101u) * 0xffu;
  if (ROWS == 64) held |= (uint64_t)((((groups >> 4) & 15u) * 0x00204081u & 0x01010101u) * 0xffu) << 32;
  const uint64_t behind = left >= ROWS ? 0ull : left <= 0 ? ~0ull : ~0ull << left;
  return (~held | behind) & (~0ull >> (64 - ROWS));
}

// As load_to_lds(), from an address of the lane's own, and past the caches: keys and
// values of few rows are read once (8 sequences of <= 32768 tokens, 32 / 8 heads of
// 128: 92 us a call, 102 with cached loads; of 256: 167 and 182).  Not so with heads of
// 64, whose row is half a cache line and the other half another workgroup's: there
// cached loads are the faster (54 us, 61 so).  Sixteen sequences that share the pages
// of 16000 tokens: the same with heads of 128 (67 us and 67) and of 64 (55 and 55).
__device__ __forceinline__ void load_lane_to_lds(const char* at, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off nt"
      :
      : "v"(at), "s"(to)
      : "memory", "m0");
}

template <int HD> struct Pt8Cfg {
  static constexpr int TN = PtCfg<HD>::TN;             // keys per tile of the `many` kind
  static constexpr int BYTES = PtCfg<HD>::BYTES;       // of a tile as numbers
  static constexpr int CH = HD / 16;                   // 16-byte chunks of codes per row
  static constexpr int RL = 64 / CH;                   // rows of one load of a wave
  static constexpr int PER = TN * CH / PT_THREADS;     // chunks per thread (many)
  // 32 keys per tile of the `few` kind (64: 108 us against 106 for one token each
  // over 8 x <= 32768, 38 against 33 for 16 x 5 drafts in a window of 4096)
  static constexpr int NB = 1;
  static constexpr int FEW_N = 32 * NB;
  static constexpr int UNIT = FEW_N * PT_WAVES;        // keys of one round of its waves
  static constexpr int FEW_BYTES = FEW_N * HD;
  static constexpr int FEW_PER = FEW_N * CH / 64;      // loads of a tile
  static constexpr int FEW_TILES = PT_WAVES * 2 * FEW_BYTES, FEW_SUMS = PT_WAVES * PT_FEW * HD * 4;
  static constexpr int FEW_LDS = FEW_TILES > FEW_SUMS ? FEW_TILES : FEW_SUMS;
  static constexpr int MANY_LDS = 4 * BYTES + 32;
  static constexpr int LDS = FEW_LDS > MANY_LDS ? FEW_LDS : MANY_LDS;
};

// 128 queries of one sequence and key head, 32 a wave, and a piece of the keys.
// Tiles become numbers on their way to LDS, once for the four waves: where each
// wave converts what it reads (codes in LDS, half its traffic), vector
// instructions bound it: 874 us against 838 for 1024 tokens over 40000.
template <typename T, int HD>
__device__ __forceinline__ void many8(const Pt8Args& a8, char* lds, int block) {
  typedef Pt8Cfg<HD> C;
  const PtArgs& a = a8.p;
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
  Columns8<T, HD> c;
  c.start(a, s, head, r);
  int* odd_tiles = (int*)(lds + 4 * C::BYTES);         // first and last tile with NaN among the values
  if (tid == 0) {
    odd_tiles[0] = INT32_MAX;
    odd_tiles[1] = -1;
  }

  // Pages and scales are looked up for several tiles at once, one group of 8
  // tokens (which lie in one page) a lane, lane GP (tile mod TILES) + group: a
  // lookup per tile takes as many instructions as a quarter of its weights (838
  // us against 748 for 1024 tokens over 40000).
  constexpr int NB = C::TN / 32, GP = 4 * NB, TILES = 64 / GP;
  const int lrow = lane / C::CH, lch = lane % C::CH;
  const char* const kbase = a.pool.k + head * a.pool.ks[2];
  const char* const vbase = a.pool.v + head * a.pool.vs[2];
  uint64_t k_at = 0, v_at = 0, there = 0;              // offsets; lanes whose page is there
  PageScale scale = {1.f, 0};
  auto token_of = [&](int i) { return begin + i * C::TN + 8 * lane; };
  int entry = entry_of(a.pool, b, token_of(0));
  auto look_up = [&](int i) __attribute__((always_inline)) {
    const int t = token_of(i), page = t < end ? checked(a.pool, entry) : -1;
    k_at = token_offset8(a.pool, a.pool.ks, page, t);
    v_at = token_offset8(a.pool, a.pool.vs, page, t);
    there = __ballot(page >= 0);
    scale = page_scale(a8, head, page);
    if (begin + (i + TILES) * C::TN < end) entry = entry_of(a.pool, b, token_of(i + TILES));
  };
  auto gone = [&](int i) {
    return gone_rows<C::TN>((uint32_t)(there >> (GP * (i % TILES))), end - begin - i * C::TN);
  };
  auto fetch = [&](bool key, uint64_t at, int i, u4 (&raw)[C::PER]) __attribute__((always_inline)) {
    const int64_t (&st)[3] = key ? a.pool.ks : a.pool.vs;
#pragma unroll
    for (int u = 0; u < C::PER; ++u) {
      const int row = (u * PT_WAVES + wave) * C::RL, from = GP * (i % TILES) + row / 8;
      raw[u] = *(const u4*)row_of_load<HD>(key ? kbase : vbase, at, from, from + 1,
                                           (row % 8 + lrow % 8) * (uint32_t)st[1] + 16 * lch);
    }
  };
  auto put = [&](bool key, const u4 (&raw)[C::PER], char* at) __attribute__((always_inline)) {
    typedef typename Vec<T>::v8 v8;
#pragma unroll
    for (int u = 0; u < C::PER; ++u) {
      const int row = (u * PT_WAVES + wave) * C::RL + lrow;
      const int c0 = key ? key_at<HD>(row, 2 * lch) : value_at<HD>(row, 2 * lch);
      const int c1 = key ? key_at<HD>(row, 2 * lch + 1) : value_at<HD>(row, 2 * lch + 1);
      *(v8*)(at + c0) = numbers<T>(raw[u][0], raw[u][1]);
      *(v8*)(at + c1) = numbers<T>(raw[u][2], raw[u][3]);
    }
  };
  // Keys run one tile ahead of values, as over 16-bit pages; both are read one
  // tile before they go to LDS.
  char* const kt = lds;
  char* const vt = lds + 2 * C::BYTES;
  u4 rk[C::PER], rv[C::PER];
  look_up(0);
  fetch(true, k_at, 0, rk);
  uint64_t absent = gone(0);
  put(true, rk, kt);
  __syncthreads();                                     // (odd_tiles, too)
  fetch(false, v_at, 0, rv);
  fetch(true, k_at, 1, rk);
  f16v even_scores[NB], odd_scores[NB];
  Groups<NB> g = groups_from<NB>(scale, 0);
  c.template scores<NB>(kt, even_scores);
  c.template settle8<NB>(begin, absent, g, even_scores);
  auto step = [&](int i, int odd, f16v (&sc)[NB], f16v (&next)[NB]) __attribute__((always_inline)) {
    char* const v = vt + odd * C::BYTES;
    const int t0 = begin + i * C::TN;
    if (absent || t0 + C::TN > wg_hi || t0 < wg_lo) {
      // each thread looks at the values that it has loaded; rows of absent
      // pages become zeros
#pragma unroll
      for (int u = 0; u < C::PER; ++u) {
        const int row = (u * PT_WAVES + wave) * C::RL + lrow;
        if ((absent >> row) & 1) {
          rv[u] = (u4){0u, 0u, 0u, 0u};
        } else if (without_nan(rv[u])) {
          atomicMin(&odd_tiles[0], t0);
          atomicMax(&odd_tiles[1], t0);
        }
      }
    }
    put(false, rv, v);
    put(true, rk, kt + (odd ^ 1) * C::BYTES);
    __syncthreads();                                   // both are there, the other halves free
    absent = gone(i + 1);
    const Groups<NB> now = g;
    g = groups_from<NB>(scale, GP * ((i + 1) % TILES));
    if (t0 + C::TN < end) {
      fetch(false, v_at, i + 1, rv);
      if ((i + 2) % TILES == 0) look_up(i + 2);        // (what the tiles before want of it is taken)
      fetch(true, k_at, i + 2, rk);
    }
    // (past the last tile the scores are those of keys that nobody sees)
    typename Vec<T>::v8 p[NB][2];
    c.template scores<NB>(kt + (odd ^ 1) * C::BYTES, next);
    c.template weights8<NB>(now, sc, p);
    c.template add_values<NB>(v, p);
    // (one product of the scores, one key read, and a share of the weights in turn;
    // then the values, read two products ahead: 1024 tokens over 40000 778 us without
    // and 748 with it)
    constexpr int N = NB * (HD / 16), W = NB * 16;     // products, weights
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < N - 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 2 * W / N, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, W / N, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < N - 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    if (t0 + C::TN < end) c.template settle8<NB>(t0 + C::TN, absent, g, next);
  };
  for (int i = 0; begin + i * C::TN < end; i += 2) {
    step(i, 0, even_scores, odd_scores);
    if (begin + (i + 1) * C::TN >= end) break;
    step(i + 1, 1, odd_scores, even_scores);
  }
  __syncthreads();
  const float2 ls = both_halves(c.l);
  c.l = ls.x + ls.y;
  const int odd_from = __builtin_amdgcn_readfirstlane(odd_tiles[0]);
  const int odd_to = __builtin_amdgcn_readfirstlane(odd_tiles[1]);
  if (__builtin_expect(odd_from <= odd_to, 0))
    c.see_nan(a8, b, head, odd_from, odd_to, C::TN, C::TN);
  if (r >= s.n * a.GQ) return;
  const int tok = r / a.GQ, gq = r - tok * a.GQ;
  const int64_t orow = (int64_t)(s.first + tok) * a.Hq + head * a.GQ + gq;
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

// All queries (32 at most) of one sequence and key head, and a piece of the
// keys: each wave takes every fourth tile, and the waves' sums are joined in
// LDS.  Tiles stay codes in LDS; each wave converts what it reads, once.
template <typename T, int HD>
__device__ __forceinline__ void few8(const Pt8Args& a8, char* lds, int block) {
  typedef Pt8Cfg<HD> C;
  constexpr int NB = C::NB, GP = 4 * NB, TILES = 64 / GP;     // groups of a tile, tiles of a lookup
  const PtArgs& a = a8.p;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the heads of a piece's tokens, which lie side by side, 8 workgroups apart: on
  // one XCD, and at the same time (105.2 us against 106.1 for one token each over
  // 8 x <= 32768)
  const int Hkv = a.pool.Hkv, whole = a.pool.B * a.ns_few / 8 * 8 * Hkv;
  const int in = block < whole ? block % (8 * Hkv) : block - whole;
  const int head = block < whole ? in / 8 : in % Hkv;
  const int rest = block < whole ? block / (8 * Hkv) * 8 + in % 8 : whole / Hkv + in / Hkv;
  const int part = rest % a.ns_few, b = rest / a.ns_few;
  const Seq s = sequence(a, b);
  if (s.n == 0 || !is_few(a, s)) return;
  const Span w = span_of(a, s, 0, PT_FEW, C::UNIT, a.ns_few);
  if (part >= w.parts) return;
  const int begin = w.lo + part * w.step + C::FEW_N * wave;
  const int end = min(w.hi, w.lo + (part + 1) * w.step);
  char* kt = lds + wave * 2 * C::FEW_BYTES;
  char* vt = kt + C::FEW_BYTES;
  // Pages and scales are looked up for several tiles at once, one group of 8
  // tokens (which lie in one page) a lane, lane GP (tile mod TILES) + group.  The
  // table is read a lookup ahead, and the scales of its pages half a lookup:
  // waiting for either holds up all loads behind it.
  const int lrow = lane / C::CH, lch = lane % C::CH;
  const char* const kbase = a.pool.k + head * a.pool.ks[2];
  const char* const vbase = a.pool.v + head * a.pool.vs[2];
  auto token_of = [&](int i) { return begin + (i + lane / GP) * C::UNIT + 8 * (lane % GP); };
  auto page_at = [&](int i, int entry) {
    return token_of(i) < end ? checked(a.pool, entry) : -1;
  };
  int next_entry = entry_of(a.pool, b, token_of(0));
  Columns8<T, HD> c;
  c.template start<true>(a, s, head, lane & 31);
  // keys that every query of the sequence sees
  const int64_t q_hi = min((int64_t)s.keys, s.pos0 + 1);
  const int64_t q_lo = a.window ? s.pos0 + s.n - a.window : 0;
  uint64_t k_at = 0, v_at = 0, there = 0;              // offsets; lanes whose page is there
  PageScale scale = {1.f, 0}, next_scale = page_scale(a8, head, page_at(0, next_entry));
  auto look_up = [&](int i) __attribute__((always_inline)) {
    const int t = token_of(i), page = page_at(i, next_entry);
    k_at = token_offset8(a.pool, a.pool.ks, page, t);
    v_at = token_offset8(a.pool, a.pool.vs, page, t);
    there = __ballot(page >= 0);
    scale = next_scale;
    if (begin + (i + TILES) * C::UNIT < end)
      next_entry = entry_of(a.pool, b, token_of(i + TILES));
  };
  auto gone = [&](int i, int t0) {
    return gone_rows<C::FEW_N>((uint32_t)(there >> (GP * (i % TILES))), end - t0);
  };
  auto fetch = [&](bool key, int i, const char* to) __attribute__((always_inline)) {
    const int64_t (&st)[3] = key ? a.pool.ks : a.pool.vs;
#pragma unroll
    for (int u = 0; u < C::FEW_PER; ++u) {
      const int row = u * C::RL, in = row % 8, from = GP * (i % TILES) + row / 8;
      const int ch = key ? key_chunk8<HD>(row + lrow, lch) : value_chunk8<HD>(row + lrow, lch);
      load_lane_to_lds(row_of_load<HD>(key ? kbase : vbase, key ? k_at : v_at, from, from + 1,
                                       (in + lrow % 8) * (uint32_t)st[1] + 16 * ch),
                       lds_offset(to) + 1024 * u);
    }
  };
  auto groups_of = [&](int i) __attribute__((always_inline)) {
    return groups_from<NB>(scale, GP * (i % TILES));
  };
  int odd_from = INT32_MAX, odd_to = -1;               // tiles with NaN among the values
  // Keys and values have one tile's place each: while weights are computed
  // the values are on their way, and while these are added the next keys.
  uint64_t absent = 0;
  Groups<NB> g = {};
  if (begin < end) {
    look_up(0);
    absent = gone(0, begin);
    fetch(true, 0, kt);
    fetch(false, 0, vt);
    g = groups_of(0);
  }
  int i = 0;
  for (int t0 = begin; t0 < end; t0 += C::UNIT) {
    wait_loads<C::FEW_PER>();                          // the keys are there
    f16v sc[NB];
    typename Vec<T>::v8 p[NB][2];
    c.template scores8<NB>(kt, sc);
    c.template settle8<NB>(t0, absent, g, sc);
    c.template weights8<NB>(g, sc, p);
    wait_lds();                                        // the keys have been read
    ++i;
    if (i % TILES == TILES / 2 && t0 + (TILES / 2 + 1) * C::UNIT < end)
      next_scale = page_scale(a8, head, page_at(i + TILES / 2, next_entry));
    if (i % TILES == 0) look_up(i);
    fetch(true, i, kt);
    wait_loads<C::FEW_PER>();                          // the values are there
    if (absent || t0 + C::FEW_N > q_hi || t0 < q_lo) {
      bool odd = false;
      int me = lane;
      asm volatile("" : "+v"(me));
#pragma unroll
      for (int u = 0; u < C::FEW_PER; ++u) {
        u4* v = (u4*)(vt + 16 * (u * 64 + me));
        u4 x = *v;
        if ((absent >> ((u * 64 + me) / C::CH)) & 1) {
          *v = (u4){0u, 0u, 0u, 0u};
        } else if (without_nan(x)) {
          *v = x;
          odd = true;
        }
      }
      if (__any(odd)) {
        odd_from = min(odd_from, t0);
        odd_to = t0;
      }
    }
    c.template add_values8<NB>(vt, p);
    wait_lds();                                        // the values have been read
    fetch(false, i, vt);
    absent = gone(i, t0 + C::UNIT);
    g = groups_of(i);
  }
  wait_loads<0>();                                     // no load writes to LDS from here on
  if (__builtin_expect(odd_from <= odd_to, 0))
    c.see_nan(a8, b, head, odd_from, odd_to, C::UNIT, C::FEW_N);

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
    const int tok = r / a.GQ, gq = r - tok * a.GQ;
    const int64_t orow = (int64_t)(s.first + tok) * a.Hq + head * a.GQ + gq;
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

// (Two workgroups a CU also for heads of 64: in the registers of three, chunks
// spill; 1024 tokens over 30000 took 540 us against 437 with 32 / 8 heads, 289 against
// 228 with 16 / 16.)
template <typename T, int HD>
__global__ void __launch_bounds__(PT_THREADS, HD == 256 ? 1 : 2) cache8_attn_kernel(Pt8Args a) {
  __shared__ __align__(16) char lds[Pt8Cfg<HD>::LDS];
  const bool first = (int)blockIdx.x < a.p.first_blocks;
  const int block = first ? blockIdx.x : blockIdx.x - a.p.first_blocks;
  if (first == a.p.many_first) many8<T, HD>(a, lds, block);
  else few8<T, HD>(a, lds, block);
}

// --------------------------------------------------------------- host side

gsrq_status page_exps(const gsrq_page_exps* x, const gsrq_pages* pages, PageExps& o) {
  if (!x || !x->k || !x->v) return GSRQ_E_ARG;
  const int count[2] = {pages->pages, pages->Hkv};
  for (int i = 0; i < 2; ++i) {
    const int64_t least = count[i] > 1 ? 1 : 0;        // no two exponents in one place
    if (x->k_stride[i] < least || x->v_stride[i] < least) return GSRQ_E_ARG;
    o.ks[i] = x->k_stride[i];
    o.vs[i] = x->v_stride[i];
  }
  o.k = x->k;
  o.v = x->v;
  return GSRQ_OK;
}

template <typename TI, typename TQ>
gsrq_status append8_launch(const Append8Args& a, int hd, int64_t wgs, hipStream_t st) {
  TimedLaunch tl(GSRQ_KERNEL_APPEND, st);
  const unsigned n = (unsigned)wgs;
  if (hd == 64) cache8_append_kernel<TI, TQ, 64><<<n, E8_THREADS, 0, st>>>(a);
  else if (hd == 128) cache8_append_kernel<TI, TQ, 128><<<n, E8_THREADS, 0, st>>>(a);
  else cache8_append_kernel<TI, TQ, 256><<<n, E8_THREADS, 0, st>>>(a);
  return launch_ok();
}

template <typename TQ>
gsrq_status append8_from(const Append8Args& a, int hd, gsrq_dtype dtype, int64_t wgs,
                         hipStream_t st) {
  if (dtype == GSRQ_F32) return append8_launch<float, TQ>(a, hd, wgs, st);
  if (dtype == GSRQ_F16) return append8_launch<_Float16, TQ>(a, hd, wgs, st);
  return append8_launch<__bf16, TQ>(a, hd, wgs, st);
}

template <typename T, int HD>
gsrq_status pt8_launch(const Pt8Args& a, const PtPlan& p, hipStream_t st) {
  static_assert(Pt8Cfg<HD>::LDS <= 160 * 1024 - 2048, "LDS of a CU");
  TimedLaunch tl(GSRQ_KERNEL_ATTENTION, st);
  cache8_attn_kernel<T, HD><<<p.few_blocks + p.many_blocks, PT_THREADS, 0, st>>>(a);
  gsrq_status e = launch_ok();
  if (e || p.merge_few + p.merge_rows == 0) return e;
  paged_attn_merge_kernel<T, HD, Pt8Cfg<HD>::UNIT><<<p.merge_few + p.merge_rows, 256, 0, st>>>(a.p);
  return launch_ok();
}

gsrq_status pt8_plan(const gsrq_paged_attn* s, const gsrq_pages* pages, PtPlan& p) {
  return pt_plan(s, pages, true, Pt8Cfg<128>::UNIT, p);
}

}  // namespace

extern "C" {

gsrq_status gsrq_paged_append8(const gsrq_pages* pages, const gsrq_page_exps* exps, int64_t T,
                               const int32_t* q_start, const int32_t* seq_len,
                               const gsrq_heads* k, const gsrq_heads* v, const gsrq_heads* q,
                               int32_t Hq, gsrq_dtype dtype, const double* theta,
                               const float* k_norm, const float* q_norm, float eps, void* q_out,
                               gsrq_dtype q_dtype, void* stream) {
  Append8Args a;
  gsrq_status e = page_pool(pages, true, a.pool);
  if (e || (e = page_exps(exps, pages, a.exps))) return e;
  if (T < 1 || !q_start || !seq_len) return GSRQ_E_ARG;
  if (dtype != GSRQ_F32 && dtype != GSRQ_F16 && dtype != GSRQ_BF16) return GSRQ_E_ARG;
  const int64_t esz = dtype == GSRQ_F32 ? 4 : 2;
  if ((e = head_rows(k, esz)) || (e = head_rows(v, esz))) return e;
  if (q) {
    if ((e = head_rows(q, esz))) return e;
    if (Hq < 1 || !q_out || (uintptr_t)q_out % 16) return GSRQ_E_ARG;
    if (q_dtype != GSRQ_F16 && q_dtype != GSRQ_BF16) return GSRQ_E_ARG;
  } else if (q_norm || q_out) {
    return GSRQ_E_ARG;
  }
  if (!(eps >= 0.f) || !(eps < INFINITY)) return GSRQ_E_ARG;
  if ((uintptr_t)theta % 8) return GSRQ_E_ARG;
  if (T > MAX_BLOCKS || a.pool.B > (1 << 20)) return GSRQ_E_UNSUPPORTED;
  if (2ll * a.pool.Hkv + (q ? Hq : 0) > 65535) return GSRQ_E_UNSUPPORTED;
  const int hd = pages->head_dim, rows = E8_THREADS * 16 / hd;
  // (a page's codes are rounded again 16 bytes a thread, counted in 32 bits)
  if ((int64_t)pages->page_size * (a.pool.Hkv * (hd / 16)) > INT32_MAX - E8_THREADS)
    return GSRQ_E_UNSUPPORTED;
  // as many heads as E8_KEEP items a thread hold of a page's tokens; fewer where that
  // leaves less than 512 workgroups, but for sequences of one token each, whose
  // heads are few items (8 heads of 128, kernel times: 512 tokens of one sequence 9.8 us
  // with all, 7.7 so; 32 sequences of one token 5.6 and 7.0).  Sequences of a few drafts
  // are few items too, and lose by it: 32 of 5 tokens take 9.0 us, with all heads 6.4;
  // 128 of 5 11.3 and 8.4.
  const int tokens = (int)std::min<int64_t>(pages->page_size, T);
  const int most = tokens <= rows ? E8_KEEP * (rows / tokens) : E8_KEEP / ((tokens + rows - 1) / rows);
  const int64_t touched = (T >> a.pool.shift) + a.pool.B;
  const int64_t fill = T > a.pool.B ? 2 * touched * a.pool.Hkv / 512 : most;
  a.HG = (int)std::min<int64_t>(a.pool.Hkv, std::max<int64_t>(1, std::min<int64_t>(most, fill)));
  a.groups = (a.pool.Hkv + a.HG - 1) / a.HG;
  a.page_wgs = ((T >> a.pool.shift) + 2ll * a.pool.B) * 2 * a.groups;
  a.Hq = q ? Hq : 0;
  // (one token's queries a workgroup where the GPU holds them all at once)
  const int64_t wide = (a.Hq + rows - 1) / rows;
  a.rows = T * wide <= 1024 ? 1 : E8_ROWS;
  const int64_t wgs = a.page_wgs + (T + a.rows - 1) / a.rows * wide;
  if (wgs > MAX_BLOCKS) return GSRQ_E_UNSUPPORTED;
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
  a.eps = eps;
  hipStream_t st = (hipStream_t)stream;
  return q && q_dtype == GSRQ_F16 ? append8_from<_Float16>(a, hd, dtype, wgs, st)
                                  : append8_from<__bf16>(a, hd, dtype, wgs, st);
}

gsrq_status gsrq_attn_paged8_workspace_bytes(const gsrq_paged_attn* s, const gsrq_pages* pages,
                                             size_t* bytes) {
  if (!bytes) return GSRQ_E_ARG;
  PtPlan p;
  gsrq_status e = pt8_plan(s, pages, p);
  if (e) return e;
  *bytes = p.bytes;
  return GSRQ_OK;
}

gsrq_status gsrq_attn_paged8(const gsrq_paged_attn* s, const gsrq_pages* pages,
                             const gsrq_page_exps* exps, const int32_t* q_start,
                             const int32_t* seq_len, const gsrq_heads* q, gsrq_dtype q_dtype,
                             void* out, float* lse, void* workspace, size_t ws_bytes,
                             void* stream) {
  PtPlan p;
  Pt8Args a;
  gsrq_status e = pt8_plan(s, pages, p);
  if (e || (e = page_exps(exps, pages, a.exps))) return e;
  if (q_dtype != GSRQ_F16 && q_dtype != GSRQ_BF16) return GSRQ_E_ARG;
  if ((e = pt_args(s, pages, p, q_start, seq_len, q, out, lse, workspace, ws_bytes, a.p))) return e;
  hipStream_t st = (hipStream_t)stream;
  const int hd = pages->head_dim;
  if (q_dtype == GSRQ_F16) {
    if (hd == 64) return pt8_launch<_Float16, 64>(a, p, st);
    if (hd == 128) return pt8_launch<_Float16, 128>(a, p, st);
    return pt8_launch<_Float16, 256>(a, p, st);
  }
  if (hd == 64) return pt8_launch<__bf16, 64>(a, p, st);
  if (hd == 128) return pt8_launch<__bf16, 128>(a, p, st);
  return pt8_launch<__bf16, 256>(a, p, st);
}

}  // extern "C"
