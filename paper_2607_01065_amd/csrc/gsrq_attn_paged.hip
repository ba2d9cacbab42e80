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
    for (int k = 0; k < KS; ++k) q[k] = *(const v8*)(qp + 16 * k);
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

  // Masks the scores of the keys from t0 on (absent: rows that nobody sees)
  // and raises the maximum in use where they exceed it.
  template <int NB>
  __device__ __forceinline__ void settle(const PtArgs& a, int t0, uint64_t absent,
                                         f16v (&sc)[NB]) {
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

__device__ __forceinline__ int few_parts(const PtArgs& a, const Seq& s) {
  return span_of(a, s, 0, PT_FEW, PT_FEW_UNIT, a.ns_few).parts;
}

// One wave (shared: one workgroup) per row and head (and, where the records of
// the `few` kind are laid out by sequence, one per such record).  A row's
// records are found without its sequence, so their first loads are on their
// way while the sequence is looked up, not after three round trips to memory
// one after the other (one token's rows: 3.9 us).
template <typename T, int HD>
__global__ void __launch_bounds__(256) paged_attn_merge_kernel(PtArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < a.merge_few) {
    const int i = a.shared_few ? blockIdx.x : blockIdx.x * 4 + wave;     // [B][Hkv][32]
    Pieces<T, HD, 8> p(a, (int64_t)i * a.ns_few, a.ns_few, a.shared_few);
    const int r = i % PT_FEW, head = i / PT_FEW % a.pool.Hkv, b = i / PT_FEW / a.pool.Hkv;
    const Seq s = sequence(a, b);
    if (!is_few(a, s) || r >= s.n * a.GQ) return;
    const int parts = few_parts(a, s), tok = r / a.GQ;
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
      const int parts = few_parts(a, s);
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

gsrq_status pt_plan(const gsrq_paged_attn* s, const gsrq_pages* pages, PtPlan& p) {
  gsrq_status e = page_pool(pages, p.pool);
  if (e) return e;
  if (!s || s->T < 1 || s->Hq < 1 || s->Hq % pages->Hkv || s->window < 0 || s->flags)
    return GSRQ_E_ARG;
  if (!(s->scale > 0.f) || !(s->scale < INFINITY)) return GSRQ_E_ARG;
  const int64_t GQ = s->Hq / pages->Hkv;
  // (T by itself first: its product with GQ is taken in 64 bits)
  if (s->T > INT32_MAX / 2 || s->T * GQ > INT32_MAX / 2 || pages->B > (1 << 20))
    return GSRQ_E_UNSUPPORTED;
  const int64_t Hkv = pages->Hkv, B = pages->B, cap = (int64_t)pages->per * pages->page_size;
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
    few = std::min(std::max<int64_t>(4, few), (cap + PT_FEW_UNIT - 1) / PT_FEW_UNIT);
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

template <typename T, int HD>
gsrq_status pt_launch(const PtArgs& a, const PtPlan& p, hipStream_t st) {
  static_assert(PtCfg<HD>::LDS <= 160 * 1024 - 2048, "LDS of a CU");
  TimedLaunch tl(GSRQ_KERNEL_ATTENTION, st);
  paged_attn_kernel<T, HD><<<p.few_blocks + p.many_blocks, PT_THREADS, 0, st>>>(a);
  gsrq_status e = launch_ok();
  if (e || p.merge_few + p.merge_rows == 0) return e;
  paged_attn_merge_kernel<T, HD><<<p.merge_few + p.merge_rows, 256, 0, st>>>(a);
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
