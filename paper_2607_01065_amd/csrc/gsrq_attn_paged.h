// Private header of attention over a paged cache (gsrq_attn_paged.hip: 16-bit
// pages; gsrq_cache8.hip: 8-bit pages): the work's division among workgroups,
// one wave's queries and their sums, and the joining of pieces.
#ifndef GSRQ_ATTN_PAGED_H
#define GSRQ_ATTN_PAGED_H

#include <algorithm>

#include "gsrq_paged.h"

namespace {

constexpr int PT_THREADS = 256;
constexpr int PT_WAVES = PT_THREADS / 64;
constexpr int PT_ROWS = 32 * PT_WAVES;     // queries per workgroup of the `many` kind
constexpr int PT_FEW = 32;                 // queries per key head of the `few` kind, at most
constexpr int PT_FEW_UNIT = 32 * PT_WAVES; // keys of one round of its four waves
constexpr float PT_HEADROOM = 8.f;         // log2 by which a tile may exceed the maximum in use
constexpr float PT_SHIFT = 6.f;            // log2 of the largest weight at a fresh maximum
static_assert(PT_HEADROOM + PT_SHIFT < 16.f, "weights are float16 numbers");

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
  static constexpr uint32_t EXP = 0x7c007c00u;         // exponent bits of a pair
  static constexpr float MAX = 65504.f;
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
  static constexpr uint32_t EXP = 0x7f807f80u;
  static constexpr float MAX = 0x1.fep127f;
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
  // pieces: sums [record][HD] unscaled, [record][2] base and sum of weights;
  // records of the `few` kind [T][Hq][ns_few] or, where that is more,
  // [B][Hkv][32][ns_few], then of the `many` kind [T][Hq][ns_many]
  float *part, *part_ml;
  int64_t many0;                  // first record of the `many` kind
  int T, Hq, GQ, ns_few, ns_many, window, slots, first_blocks, merge_few;
  bool many_first, few_by_row, shared_few, shared_rows;
  float c;                        // scale * log2(e)
};

// Sequence b's new rows [first, first + n), keys [0, keys), and the position
// of its first new row.
struct Seq {
  int first, n, keys;
  int64_t pos0;
};

__device__ __forceinline__ Seq sequence(const PtArgs& a, int b) {
  Seq s;
  new_rows(a.q_start, b, a.T, s.first, s.n);
  const int len = max(a.seq_len[b], 0);
  const int64_t cap = (int64_t)a.pool.per << a.pool.shift;
  s.keys = len < cap ? len : (int)cap;
  s.pos0 = (int64_t)len - s.n;
  return s;
}

__device__ __forceinline__ bool is_few(const PtArgs& a, const Seq& s) {
  return s.n * a.GQ <= PT_FEW;                                  // (T GQ < 2^30)
}

// What queries r0 .. r0 + rows - 1 of a sequence read: keys lo .. hi - 1, in
// `parts` pieces of `step` keys, at most ns, cut at multiples of `unit`.
struct Span {
  int lo, hi, step, parts;
};

__device__ __forceinline__ Span span_of(const PtArgs& a, const Seq& s, int r0, int rows, int unit,
                                        int ns) {
  const uint32_t last = min(r0 + rows, s.n * a.GQ) - 1;        // (T GQ < 2^30)
  const int64_t top = s.pos0 + last / (uint32_t)a.GQ + 1;
  const int64_t bottom = a.window ? s.pos0 + (uint32_t)r0 / (uint32_t)a.GQ - a.window + 1 : 0;
  Span w;
  w.hi = (int)(top < s.keys ? top : s.keys);
  w.lo = bottom > 0 ? (int)(bottom < s.keys ? bottom : s.keys) / unit * unit : 0;
  const int units = w.hi > w.lo ? (w.hi - w.lo + unit - 1) / unit : 0;
  const int per = (units + ns - 1) / ns;
  w.step = per * unit;
  w.parts = units ? (units + per - 1) / per : 1;
  return w;
}

// Tile slot of the `many` kind: sequence b owns the slots from its first row's
// tile number on, one more than it can need at most.
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

// The largest of 16 products' sums, NaN left out: fmaxf() would quiet each
// operand first.  The first maximum is the compiler's own instruction, before
// which it waits for the matrix unit; for the others, which need its result,
// it would not.
__device__ __forceinline__ float max16(f16v x) {
  float r = __builtin_amdgcn_fmed3f(x[0], x[1], INFINITY);
  asm("v_max3_f32 %0, %0, %1, %2\n\t"
      "v_max3_f32 %0, %0, %3, %4\n\t"
      "v_max3_f32 %0, %0, %5, %6\n\t"
      "v_max3_f32 %0, %0, %7, %8\n\t"
      "v_max3_f32 %0, %0, %9, %10\n\t"
      "v_max3_f32 %0, %0, %11, %12\n\t"
      "v_max3_f32 %0, %0, %13, %14"
      : "+v"(r)
      : "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]), "v"(x[8]), "v"(x[9]),
        "v"(x[10]), "v"(x[11]), "v"(x[12]), "v"(x[13]), "v"(x[14]), "v"(x[15]));
  return r;
}

// Places of a tile's 16-byte chunk c of row r in LDS: rows of a key tile are
// read 32 at a time at one chunk, rows of a value tile four at a time at four
// chunks, both without bank conflicts in these orders.
template <int HD> __device__ __forceinline__ int key_chunk(int r, int c) {
  return c ^ (HD == 64 ? (r >> 1) & 7 : r & 15);
}
template <int HD> __device__ __forceinline__ int value_chunk(int r, int c) {
  return c ^ (4 * (HD == 64 ? (r >> 1) & 1 : r & 3));
}
template <int HD> __device__ __forceinline__ int key_at(int r, int c) {
  return r * (HD * 2) + (key_chunk<HD>(r, c) << 4);
}
template <int HD> __device__ __forceinline__ int value_at(int r, int c) {
  return r * (HD * 2) + (value_chunk<HD>(r, c) << 4);
}

template <int HD> struct PtCfg {
  static constexpr int TN = HD == 256 ? 32 : 64;       // keys per tile of the `many` kind
  static constexpr int CH = HD / 8;                    // 16-byte chunks per row
  static constexpr int BYTES = TN * HD * 2;
  static constexpr int PER = TN * CH / PT_THREADS;     // chunks per thread
  static constexpr int FEW_BYTES = 32 * HD * 2;        // a wave's tile of the `few` kind
  static constexpr int FEW_PER = 32 * CH / 64;         // chunks per lane
  // LDS of a workgroup: two key and two value tiles, and which tiles held
  // infinities or NaN; for `few` a key and a value tile a wave (where it also
  // joins its waves' sums)
  static constexpr int FEW_LDS = PT_WAVES * 2 * FEW_BYTES;
  static constexpr int MANY_LDS = 4 * BYTES + 32;
  static constexpr int LDS = FEW_LDS > MANY_LDS ? FEW_LDS : MANY_LDS;
};

// 16 bytes a lane from `base` + `offset` (bytes) to LDS, to `to` + 16 * lane;
// base and `to` the same for the whole wave.  Not waited for: a load that the
// compiler does not know of, so that it makes no LDS read wait for all loads
// in flight; wait_loads() does.  Every lane is active at every call (a load
// that no lane takes part in would be missing in the count of those in flight).
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(offset), "s"(base), "s"(to)
      : "memory", "m0");
}
// Until at most N of this wave's loads are in flight.
template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory");
}
// Until this wave's LDS accesses are done.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

__device__ __forceinline__ uint32_t lds_offset(const char* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const lds_char*)p);
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }

// o + f x for a factor f >= 0 that stands for a weight above zero, however
// small: an infinity stays one where f has come to zero.
__device__ __forceinline__ float add_weighted(float o, float f, float x) {
  return is_finite(x) ? fmaf(f, x, o) : o + x;
}

// An element of a result.  Weights are rounded and their sum is not, so a mean
// of values at the type's end can come out past it by a rounding (in float16
// 2^-11 of itself); it is held inside.
template <typename T> __device__ __forceinline__ T result(float x) {
  return (T)(is_finite(x) ? __builtin_amdgcn_fmed3f(x, -Vec<T>::MAX, Vec<T>::MAX) : x);
}

// Takes infinities and NaN out of eight values; whether there were any.
template <typename T> __device__ __forceinline__ bool finite_pairs(u4& x) {
  constexpr uint32_t HI = Vec<T>::EXP & 0xffff0000u, LO = Vec<T>::EXP & 0xffffu;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = x[i];
    if ((w & LO) == LO) w &= 0xffff0000u;
    if ((w & HI) == HI) w &= 0xffffu;
    any = any || w != x[i];
    x[i] = w;
  }
  return any;
}

// Takes infinities and NaN out of a 16-byte chunk of values in a tile where
// some query does not see every row (its weight of zero would make NaN of
// them); add_infinities() brings them to the queries that see them.  Whether
// there were any.
template <typename T> __device__ __forceinline__ bool without_infinities(u4* at) {
  u4 x = *at;
  const bool any = finite_pairs<T>(x);
  if (any) *at = x;
  return any;
}

// One wave's queries, as columns: the lane's query, and its part of the sums.
template <typename T, int HD> struct Columns {
  typedef typename Vec<T>::v8 v8;
  typedef typename Vec<T>::v4 v4;
  static constexpr int KS = HD / 16, DT = HD / 32;
  v8 q[KS];
  f16v o[DT];
  float m, l;                     // maximum in use (of scaled scores, log2), sum of weights
  int see_lo, see_hi;             // keys that the query sees
  int all_lo, all_hi;             // keys that every query of the wave sees

  // Query r of the sequence.  Rows past the last are copies of row 0 that see
  // everything, so that they ask for no masks; what they come to (weights of
  // zero, or NaN) is not used.
  // PAIRED: dimensions in the order of 16-byte rows of codes (a lane's 16 are
  // those of two products).
  template <bool PAIRED = false>
  __device__ __forceinline__ void start(const PtArgs& a, const Seq& s, int head, int r) {
    const int half = (threadIdx.x >> 5) & 1;
    const bool real = r < s.n * a.GQ;
    const int tok = real ? (uint32_t)r / (uint32_t)a.GQ : 0, g = real ? r - tok * a.GQ : 0;
    const int64_t pos = s.pos0 + tok;
    const int64_t from = a.window ? pos - a.window + 1 : 0;
    see_hi = pos + 1 < s.keys ? (pos + 1 > 0 ? (int)(pos + 1) : 0) : s.keys;
    see_lo = from > 0 ? (from < s.keys ? (int)from : s.keys) : 0;
    if (!real) {
      see_hi = INT32_MAX;
      see_lo = 0;
    }
    const T* qp = (const T*)a.q + (int64_t)(s.first + tok) * a.qst[0] +
                  (int64_t)(head * a.GQ + g) * a.qst[1] + 8 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k)
      q[k] = *(const v8*)(qp + (PAIRED ? 8 * half + 32 * (k / 2) + 8 * (k % 2) : 16 * k));
    // (waited for here: the compiler does not count load_to_lds(), and would
    // wait for those in flight too inside the loop)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" : "+v"(q[k]));
    all_hi = see_hi;
    all_lo = see_lo;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      all_hi = min(all_hi, __shfl_xor(all_hi, x));
      all_lo = max(all_lo, __shfl_xor(all_lo, x));
    }
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    m = real ? -INFINITY : INFINITY;                   // (a copy's maximum is never raised)
    l = 0.f;
  }

  // Scores of NB blocks of 32 keys in LDS.
  template <int NB>
  __device__ __forceinline__ void scores(const char* kt, f16v (&sc)[NB]) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const v8 kf = *(const v8*)(kt + key_at<HD>(32 * n + col, 2 * k + half));
        sc[n] = Vec<T>::mfma(kf, q[k], sc[n]);
      }
  }

  // Masks the scores of the keys from t0 on (absent: rows that nobody sees).
  template <int NB>
  __device__ __forceinline__ void mask(int t0, uint64_t absent, f16v (&sc)[NB]) {
    if (absent || t0 + 32 * NB > all_hi || t0 < all_lo) {
      // (bounds moved to the lane's first row, so that each element compares
      // with a constant)
      const int half = (threadIdx.x >> 5) & 1;
      const int hi = see_hi - t0 - 4 * half, lo = see_lo - t0 - 4 * half;
      const uint64_t gone = absent >> (4 * half);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = 32 * n + 8 * (i / 4) + i % 4;
          const bool seen = row < hi && row >= lo && !((gone >> row) & 1);
          sc[n][i] = seen ? sc[n][i] : -INFINITY;
        }
    }
  }

  // The same, and raises the maximum in use where they exceed it.
  template <int NB>
  __device__ __forceinline__ void settle(const PtArgs& a, int t0, uint64_t absent,
                                         f16v (&sc)[NB]) {
    mask<NB>(t0, absent, sc);
    float top = max16(sc[0]);
    if (NB > 1) top = fmaxf(top, max16(sc[NB - 1]));
    const float2 tops = both_halves(top);
    top = fmaxf(tops.x, tops.y) * a.c;
    // (each query by itself: what another one sees changes no bit of its result;
    // one that has seen nothing keeps -inf)
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

  // Weights of settled scores.
  template <int NB>
  __device__ __forceinline__ void weights(const PtArgs& a, const f16v (&sc)[NB],
                                          v8 (&p)[NB][2]) {
    const float sub = m == -INFINITY ? 0.f : PT_SHIFT - m;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float x = __builtin_amdgcn_exp2f(fmaf(sc[n][8 * k + e], a.c, sub));
          const float y = __builtin_amdgcn_exp2f(fmaf(sc[n][8 * k + e + 1], a.c, sub));
          p[n][k][e] = (T)x;
          p[n][k][e + 1] = (T)y;
          l += x + y;
        }
  }

  // Adds their values, from LDS.
  template <int NB>
  __device__ __forceinline__ void add_values(const char* vt, const v8 (&p)[NB][2]) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] = Vec<T>::mfma(values(vt, n, k, t), p[n][k], o[t]);
  }

  // V^T of 32 dimensions and the 16 tokens of weights [n][k], in their order.
  static __device__ __forceinline__ v8 values(const char* vt, int n, int k, int t) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int row = 32 * n + 16 * k + 4 * half + ((lane & 15) >> 2);
    const int ch = 4 * t + ((lane >> 3) & 2) + ((lane & 3) >> 1), in = 8 * (lane & 1);
    const v4 lo = Vec<T>::read_tr((lds_char*)(vt + value_at<HD>(row, ch) + in));
    const v4 hi = Vec<T>::read_tr((lds_char*)(vt + value_at<HD>(row + 8, ch) + in));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }

  // Adds the infinities and NaN among the values of `rows` keys every `step`
  // from `from` to `to`, for the queries that see them.  A weight above zero
  // leaves them what they are, and adding one twice changes nothing.
  __device__ __forceinline__ void see_infinities(const PtArgs& a, int b, int head, int from, int to,
                                                 int step, int rows) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const auto value = [&](int page, int j) __attribute__((always_inline)) {
      return (const T*)a.pool.v + page * a.pool.vs[0] +
             (int64_t)(j & ((1 << a.pool.shift) - 1)) * a.pool.vs[1] + head * a.pool.vs[2];
    };
    for (int t0 = from; t0 <= to; t0 += step) {
      // one key a lane: whether it holds any
      const int mine = lane < rows ? page_of(a.pool, b, t0 + lane) : -1;
      bool odd = false;
      if (mine >= 0) {
        const T* v = value(mine, t0 + lane);
#pragma unroll 4
        for (int c = 0; c < HD / 8; ++c) {
          u4 x = *(const u4*)(v + 8 * c);
          odd = finite_pairs<T>(x) || odd;
        }
      }
      for (uint64_t todo = __ballot(odd); todo; todo &= todo - 1) {
        const int j = t0 + __builtin_ctzll(todo);
        const T* v = value(__builtin_amdgcn_readlane(mine, j - t0), j) + 4 * half;
        const bool seen = j < see_hi && j >= see_lo;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const v4 x = *(const v4*)(v + 32 * t + 8 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float y = (float)x[e];
              o[t][4 * i + e] += seen && !is_finite(y) ? y : 0.f;
            }
          }
      }
    }
  }

  // After the last tile, l joined: the infinities and NaN that the sums lack.
  // They are those that without_infinities() took out, in the tiles from
  // `odd_from` to `odd_to`; and where a sum is NaN though no score was (`real`:
  // the lane's query is one), any of the piece's, whose tiles start at `begin`
  // and end before `end`: a weight that is zero in the pages' type, or that a
  // later maximum made zero, has made NaN of an infinity that the query sees.
  __device__ __forceinline__ void add_infinities(const PtArgs& a, int b, int head, bool real,
                                                 int odd_from, int odd_to, int begin, int end,
                                                 int step, int rows) {
    // (NaN if any of them is; infinities of both signs look the same, and change nothing)
    f16v sum = o[0];
#pragma unroll
    for (int t = 1; t < DT; ++t) sum += o[t];
#pragma unroll
    for (int i = 2; i < 16; ++i) sum[i & 1] += sum[i];
    const float all = sum[0] + sum[1];
    const bool again = __any(all != all && real && l == l);
    // (rare: what follows lies apart from the code of every call)
    if (__builtin_expect(!again && odd_from > odd_to, 1)) return;
    uint32_t nan[(DT + 1) / 2] = {};
    if (again) {
      odd_from = begin;
      odd_to = end - 1;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool is = o[t][i] != o[t][i];
          nan[t / 2] |= is ? 1u << (16 * (t & 1) + i) : 0u;
          o[t][i] = is ? 0.f : o[t][i];
        }
    }
    see_infinities(a, b, head, odd_from, odd_to, step, rows);
    if (again) {                                       // NaN of another cause stays
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool was = (nan[t / 2] >> (16 * (t & 1) + i)) & 1u;
          o[t][i] = was && is_finite(o[t][i]) ? NAN : o[t][i];
        }
    }
  }
};

// Where a lane's token lies from its head's first key (or value) on, in bytes;
// an absent page counts as the pool's first, which nobody looks at.  Taken one
// token a lane, so that a load of several rows needs two lane reads and an
// addition, not their products: pages hold at least 8 tokens, and a wave's
// load of 64 / CH <= 8 rows lies in one.
__device__ __forceinline__ uint64_t token_offset(const PagePool& p, const int64_t (&st)[3], int page,
                                                 int t) {
  const uint32_t in = page < 0 ? 0 : t & ((1 << p.shift) - 1);
  return 2 * ((uint64_t)(uint32_t)(page < 0 ? 0 : page) * (uint32_t)st[0] +
              (uint64_t)in * (uint32_t)st[1]);
}
// base + the offset that lane `row` holds.
__device__ __forceinline__ const char* rows_at(const char* base, uint64_t offset, int row) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)offset, row);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(offset >> 32), row);
  return base + ((uint64_t)hi << 32 | lo);
}

// A row's result, from its lane's part of the sums (both halves of l joined).
template <typename T, int HD>
__device__ __forceinline__ void put_row(const PtArgs& a, const Columns<T, HD>& c, int64_t orow) {
  typedef typename Vec<T>::v4 v4;
  const int half = (threadIdx.x >> 5) & 1;
  const float inv = c.l == 0.f ? 0.f : 1.f / c.l;
  T* dst = (T*)a.out + orow * HD + 4 * half;
#pragma unroll
  for (int t = 0; t < HD / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = result<T>(c.o[t][4 * i + e] * inv);
      *(v4*)(dst + 32 * t + 8 * i) = x;
    }
  if (a.lse && half == 0)
    a.lse[orow] = c.l == 0.f ? -INFINITY
                             : (c.m - PT_SHIFT + log2f(c.l)) * 0.69314718055994531f;
}

// Joins the pieces of a row whose keys were cut: by one wave, or (`shared`) by
// four that take a quarter of the records each.  The first loads (N sums)
// start on construction, before it is known how many pieces there are: what
// lies past the row's last one is anything, and not used.
template <typename T, int HD, int N> struct Pieces {
  static constexpr int E = HD / 64;
  typedef float vec __attribute__((ext_vector_type(E)));
  static __device__ __forceinline__ void add_sums(vec& o, float f, vec x) {
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = add_weighted(o[e], f, x[e]);
  }
  static __device__ __forceinline__ bool any_nan(vec o) {
    bool nan = false;
#pragma unroll
    for (int e = 0; e < E; ++e) nan = nan || o[e] != o[e];
    return __any(nan);
  }
  const float2* mls;
  const float* sums;
  float2 ml;
  vec first[N];
  int from, most;                 // the wave's first record, and how many it has at most
  bool shared;

  __device__ __forceinline__ Pieces(const PtArgs& a, int64_t rec, int ns, bool four)
      : shared(four) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = (ns + 3) / 4;
    from = shared ? min(wave * quarter, ns) : 0;
    most = shared ? min(quarter, ns - from) : ns;
    const int64_t at = rec + min(from, ns - 1);
    mls = (const float2*)a.part_ml + at;
    sums = a.part + at * HD + lane * E;
    ml = mls[lane < most ? lane : 0];
#pragma unroll
    for (int x = 0; x < N; ++x) first[x] = *(const vec*)(sums + (x < most ? x : 0) * HD);
  }

  __device__ __forceinline__ void join(const PtArgs& a, int all, int64_t orow) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int parts = max(0, min(all - from, most));
    // 64 pieces at a time, one a lane; then their sums
    float top = -INFINITY, l = 0.f;
    vec o = {};
    for (int i0 = 0; i0 < parts; i0 += 64) {
      const int count = min(64, parts - i0);
      if (i0) ml = mls[i0 + (lane < count ? lane : 0)];
      if (lane >= count) ml = make_float2(-INFINITY, 0.f);
      float now = ml.x;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) now = fmaxf(now, __shfl_xor(now, x));
      now = fmaxf(now, top);
      const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - now);
      float sum = f * ml.y;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
      top = now;
      l = l * old + sum;
      o *= old;
      auto factor = [&](int x) {
        return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), x));
      };
      if (i0 == 0) {
#pragma unroll
        for (int x = 0; x < N; ++x)
          if (x < count) o += factor(x) * first[x];
      }
#pragma unroll 8
      for (int x = i0 ? 0 : N; x < count; ++x)
        o += factor(x) * *(const vec*)(sums + (int64_t)(i0 + x) * HD);
    }
    if (__builtin_expect(any_nan(o), 0)) {             // a factor of zero, perhaps: once more
      o = (vec){};
      for (int x = 0; x < parts; ++x) {
        const float m = mls[x].x;
        add_sums(o, m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top),
                 *(const vec*)(sums + (int64_t)x * HD));
      }
    }
    if (shared) {
      __shared__ float2 wave_ml[4];
      __shared__ vec wave_o[4][64];
      if (lane == 0) wave_ml[wave] = make_float2(top, l);
      wave_o[wave][lane] = o;
      __syncthreads();
      if (wave) return;
      const float own = top;
#pragma unroll
      for (int x = 1; x < 4; ++x) top = fmaxf(top, wave_ml[x].x);
      const float f0 = own == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(own - top);
      l *= f0;
      o *= f0;
#pragma unroll
      for (int x = 1; x < 4; ++x) {
        const float m = wave_ml[x].x;
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l += f * wave_ml[x].y;
        o += f * wave_o[x][lane];
      }
      if (__builtin_expect(any_nan(o), 0)) {
        o = (vec){};
        for (int x = 0; x < 4; ++x) {
          const float m = wave_ml[x].x;
          add_sums(o, m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), wave_o[x][lane]);
        }
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) ((T*)a.out)[orow * HD + lane * E + e] = result<T>(o[e] * inv);
    if (a.lse && lane == 0)
      a.lse[orow] = l == 0.f ? -INFINITY : (top - PT_SHIFT + log2f(l)) * 0.69314718055994531f;
  }
};

template <int UNIT> __device__ __forceinline__ int few_parts(const PtArgs& a, const Seq& s) {
  return span_of(a, s, 0, PT_FEW, UNIT, a.ns_few).parts;
}

// One wave (shared: one workgroup) per row and head (and, where the records of
// the `few` kind are laid out by sequence, one per such record).  A row's
// records are found without its sequence, so their first loads are on their
// way while the sequence is looked up, not after three round trips to memory
// one after the other (one token's rows: 3.9 us).
template <typename T, int HD, int UNIT>     // UNIT: keys of one round of a `few` workgroup
__global__ void __launch_bounds__(256) paged_attn_merge_kernel(PtArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < a.merge_few) {
    const int i = a.shared_few ? blockIdx.x : blockIdx.x * 4 + wave;     // [B][Hkv][32]
    Pieces<T, HD, 8> p(a, (int64_t)i * a.ns_few, a.ns_few, a.shared_few);
    const int r = i % PT_FEW, head = i / PT_FEW % a.pool.Hkv, b = i / PT_FEW / a.pool.Hkv;
    const Seq s = sequence(a, b);
    if (!is_few(a, s) || r >= s.n * a.GQ) return;
    const int parts = few_parts<UNIT>(a, s), tok = r / a.GQ;
    if (parts < 2) return;
    p.join(a, parts, (int64_t)(s.first + tok) * a.Hq + head * a.GQ + r - tok * a.GQ);
    return;
  }
  const int64_t block = (int64_t)blockIdx.x - a.merge_few;
  const int64_t orow = a.shared_rows ? block : block * 4 + wave;
  if (orow >= (int64_t)a.T * a.Hq) return;
  const int row = (int)(orow / a.Hq), head = (int)(orow - (int64_t)row * a.Hq);
  auto look_up = [&](Seq& s) {
    const int b = sequence_of(a.q_start, a.pool.B, row);
    if (b >= 0) s = sequence(a, b);
    return b >= 0;
  };
  auto many_parts = [&](const Seq& s) {
    const int r = (row - s.first) * a.GQ + head % a.GQ;
    return span_of(a, s, r / PT_ROWS * PT_ROWS, PT_ROWS, PtCfg<HD>::TN, a.ns_many).parts;
  };
  Seq s;
  if (a.few_by_row && a.ns_few > 1) {
    Pieces<T, HD, 8> p(a, orow * a.ns_few, a.ns_few, a.shared_rows);
    if (!look_up(s)) return;
    if (is_few(a, s)) {
      const int parts = few_parts<UNIT>(a, s);
      if (parts > 1) p.join(a, parts, orow);
      return;
    }
    if (a.ns_many < 2) return;
    const int parts = many_parts(s);
    if (parts < 2) return;
    Pieces<T, HD, 2> q(a, a.many0 + orow * a.ns_many, a.ns_many, a.shared_rows);
    q.join(a, parts, orow);
    return;
  }
  Pieces<T, HD, 2> p(a, a.many0 + orow * a.ns_many, a.ns_many, a.shared_rows);
  if (!look_up(s) || is_few(a, s)) return;
  const int parts = many_parts(s);
  if (parts > 1) p.join(a, parts, orow);
}

// --------------------------------------------------------------- host side

struct PtPlan {
  PagePool pool;
  int64_t slots, many0;
  int ns_few, ns_many, few_blocks, many_blocks, merge_few, merge_rows;
  bool few_by_row, shared_few, shared_rows;
  size_t off_ml, bytes;
};

inline gsrq_status pt_plan(const gsrq_paged_attn* s, const gsrq_pages* pages, bool eight, int unit,
                           PtPlan& p) {
  gsrq_status e = page_pool(pages, eight, p.pool);
  if (e) return e;
  if (!s || s->T < 1 || s->Hq < 1 || s->Hq % pages->Hkv || s->window < 0 || s->flags)
    return GSRQ_E_ARG;
  if (!(s->scale > 0.f) || !(s->scale < INFINITY)) return GSRQ_E_ARG;
  const int64_t GQ = s->Hq / pages->Hkv;
  // (T by itself first: its product with GQ is taken in 64 bits)
  if (s->T > INT32_MAX / 2 || s->T * GQ > INT32_MAX / 2 || pages->B > (1 << 20))
    return GSRQ_E_UNSUPPORTED;
  const int64_t Hkv = pages->Hkv, B = pages->B, held = (int64_t)pages->per * pages->page_size;
  // (8-bit pages: a sequence's few rows see no more than the window and themselves;
  // pieces by the table's length took 33 us for 16 x 5 drafts in a window of 4096,
  // by the window 26)
  const int64_t cap = eight && s->window ? std::min<int64_t>(held, (int64_t)s->window + PT_FEW) : held;
  // `few`: pieces that give every CU two workgroups, and where they stay longer
  // than 512 keys twice as many (lengths differ); of one round of the four waves
  // at the least.  More, shorter ones cost their starts: 8 sequences of 2048
  // tokens took 25 us in 1024 workgroups, 19 in 512.  Four pieces at the
  // least where the sequences alone would fill the GPU: one of them may be much
  // longer than the others (128 sequences of 8 heads, one of 20000 tokens among
  // 500s: 146 us with one piece, 99 with four, 104 with 16).  A fixed number
  // cannot follow every batch: one of 100000 among 31 of 1000 takes 296 us in
  // these four and 123 in 16, 32 of 4000 take 101 and 117.  None where the table
  // holds 256 tokens at most: 8 us a call against 10 with the joining launch; at
  // 700 tokens 16 against 11.
  int64_t few = 1;
  if (cap > 256) {
    const int64_t once = (512 + B * Hkv - 1) / (B * Hkv);
    few = std::min(2 * once, std::max(once, cap / 512));
    few = std::min(std::max<int64_t>(4, few), (cap + unit - 1) / unit);
  }
  // `many`: none where no sequence can have more than 32 queries; cut until
  // the launch's tiles (not counting the slots that hold none) give every CU two
  // workgroups, into pieces of 256 keys at the least, and no more than 1024
  // workgroups in all (of which those of empty slots, and of sequences that
  // prove to bring few queries, end at once)
  p.slots = s->T * GQ > PT_FEW ? s->T * GQ / PT_ROWS + B : 0;
  int64_t many = 1;
  if (p.slots) {
    const int64_t tiles = (s->T * GQ + PT_ROWS - 1) / PT_ROWS * Hkv;
    many = std::min((512 + tiles - 1) / tiles, (cap + 255) / 256);
    many = std::max<int64_t>(1, std::min(many, 1024 / (p.slots * Hkv)));
  }
  const int64_t few_blocks = B * Hkv * few, many_blocks = p.slots * Hkv * many;
  p.few_by_row = s->T * GQ <= PT_FEW * B;
  const int64_t few_rows = p.few_by_row ? s->T * s->Hq : B * Hkv * PT_FEW;
  // four waves join a row of more than 32 pieces (128 pieces: 137 us a call of
  // one token over 131072 with one wave, 113 with four)
  p.shared_few = few > 32;
  p.shared_rows = many > 32 || (p.few_by_row && few > 32);
  const int64_t merge_few = few > 1 && !p.few_by_row ? few_rows / (p.shared_few ? 1 : 4) : 0;
  const bool by_row = (few > 1 && p.few_by_row) || (p.slots && many > 1);
  const int64_t merge_rows = !by_row ? 0 : p.shared_rows ? s->T * s->Hq : (s->T * s->Hq + 3) / 4;
  if (few_blocks + many_blocks > MAX_BLOCKS || merge_few + merge_rows > MAX_BLOCKS)
    return GSRQ_E_UNSUPPORTED;
  p.ns_few = (int)few;
  p.ns_many = (int)many;
  p.few_blocks = (int)few_blocks;
  p.many_blocks = (int)many_blocks;
  p.merge_few = (int)merge_few;
  p.merge_rows = (int)merge_rows;
  p.many0 = few > 1 ? few_rows * few : 0;
  const size_t rows = (size_t)p.many0 + (p.slots && many > 1 ? (size_t)(s->T * s->Hq * many) : 0);
  p.off_ml = align256(rows * pages->head_dim * sizeof(float));
  p.bytes = p.off_ml + align256(rows * 2 * sizeof(float));
  return GSRQ_OK;
}

// Host checks of a call's other arguments, and the kernels' arguments.
inline gsrq_status pt_args(const gsrq_paged_attn* s, const gsrq_pages* pages, const PtPlan& p,
                           const int32_t* q_start, const int32_t* seq_len, const gsrq_heads* q,
                           void* out, float* lse, void* workspace, size_t ws_bytes, PtArgs& a) {
  gsrq_status e;
  if (!q_start || !seq_len || !out || (uintptr_t)out % 16) return GSRQ_E_ARG;
  if ((e = head_rows(q, 2))) return e;
  if (p.bytes && (!workspace || (uintptr_t)workspace % 256)) return GSRQ_E_ARG;
  if (ws_bytes < p.bytes) return GSRQ_E_WORKSPACE;
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
  a.ns_few = p.ns_few;
  a.ns_many = p.ns_many;
  // the longer workgroups first: those of chunks among single tokens, unless
  // the sequences bring few rows on average
  a.many_first = !p.few_by_row;
  a.few_by_row = p.few_by_row;
  a.shared_few = p.shared_few;
  a.shared_rows = p.shared_rows;
  a.first_blocks = a.many_first ? p.many_blocks : p.few_blocks;
  a.merge_few = p.merge_few;
  a.many0 = p.many0;
  a.window = s->window;
  a.slots = (int)p.slots;
  a.c = (float)((double)s->scale * 1.4426950408889634);
  return GSRQ_OK;
}

}  // namespace

#endif  // GSRQ_ATTN_PAGED_H
