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
// keys then turned in float32 at the token's position.  A workgroup owns 64
// or 128 dimensions of one head, half of them turned with the other half, of the
// keys or of the values, and holds a stage's codewords there as K rows in LDS.
#include <algorithm>

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

// Where a row's code of stage m and subspace g lies.  Codes of 1, 2, 4, 8 or 16
// bits never cross words; for others the next word, where there is one, comes
// along.  Reading and extracting are apart so that many codes can be on their
// way at once, without a branch between them.
struct CodeBits {
  int64_t word;
  int shift;
};
template <bool V> struct Bool { static constexpr bool value = V; };

__device__ __forceinline__ CodeBits code_bits(const RestoreArgs& a, int m, int g) {
  const int64_t bit = ((int64_t)m * a.G + g) * a.b;
  return {bit >> 5, (int)(bit & 31)};
}
// Calls f with whether codes cross words, the same for a whole launch.
template <typename F> __device__ __forceinline__ void by_crossing(const RestoreArgs& a, F f) {
  if (32 % a.b) f(Bool<true>());
  else f(Bool<false>());
}
template <bool CROSS>
__device__ __forceinline__ uint32_t read_code(const RestoreArgs& a, const uint32_t* row,
                                              const CodeBits& c) {
  const uint32_t lo = row[c.word];
  if (!CROSS) return lo;
  const uint32_t hi = row[c.word + 1 < a.words ? c.word + 1 : c.word];
  return (uint32_t)(((uint64_t)hi << 32 | lo) >> c.shift);
}
__device__ __forceinline__ int code_of(const RestoreArgs& a, uint32_t v, const CodeBits& c) {
  return (int)(v >> (32 % a.b ? 0 : c.shift) & ((1u << a.b) - 1u));
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
    const CodeBits at = code_bits(a, m, g);
    int k = 0;
    by_crossing(a, [&](auto cross) {
      k = code_of(a, read_code<decltype(cross)::value>(a, codes, at), at);
    });
    const float gk = gain[cb * a.K + k];
    float s[8];
    load8(shape + (cb * a.K + k) * a.d + (e - g * a.d), s);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += gk * s[j];
  }
}

// One workgroup's share of a restored cache: HALF dimensions of one head's keys
// or values and the HALF they are turned with.
struct Slice {
  const uint32_t* codes;
  const float *gain, *shape;
  char* base;
  uint32_t st0, st1;              // page, token (elements)
  bool turn;
  int lo, hi;                     // first elements of the halves in a row of D
  int first;                      // of the lower half in the head
};

template <typename TP, int HALF>
__device__ __forceinline__ Slice slice_of(const RestoreArgs& a, int sub) {
  // (a head's slices 2 Hkv workgroups apart, as a rule on one XCD: its L2
  // joins their 64-byte pieces of a line)
  const bool key = !(sub & 1);
  const int head = (sub >> 1) % a.pool.Hkv, slice = (sub >> 1) / a.pool.Hkv;
  const int64_t* st = key ? a.pool.ks : a.pool.vs;
  Slice s;
  s.codes = key ? a.k_codes : a.v_codes;
  s.gain = key ? a.k_gain : a.v_gain;
  s.shape = key ? a.k_shape : a.v_shape;
  s.first = HALF * slice;
  s.base = (key ? a.pool.k : a.pool.v) + (head * st[2] + s.first) * (int64_t)sizeof(TP);
  s.st0 = (uint32_t)st[0];
  s.st1 = (uint32_t)st[1];
  s.turn = key && a.theta;
  s.lo = head * a.hd + s.first;
  s.hi = s.lo + a.hd / 2;
  return s;
}

// Four elements from element e on of codeword k of a stage, rounded to float32
// before any sum.
__device__ __forceinline__ f4 codeword4(const RestoreArgs& a, const Slice& s, int m, int k, int e) {
#pragma clang fp contract(off)
  const int g = e / a.d;
  const int64_t cb = ((int64_t)m * a.G + g) * a.K + k;
  const f4 v = *(const f4*)(s.shape + cb * a.d + (e - g * a.d));
  const float gk = s.gain[cb];
  return (f4){gk * v[0], gk * v[1], gk * v[2], gk * v[3]};
}

// Where a token's slice goes; null: its page is not there.  (Strides fit 32
// bits in elements: one multiply-add each, where 64-bit products take three.)
__device__ __forceinline__ char* token_at(const RestoreArgs& a, const Slice& s, int page, int t) {
  const uint32_t in = t & ((1 << a.pool.shift) - 1);
  const uint64_t at = (uint64_t)(uint32_t)page * s.st0 + (uint64_t)in * s.st1;
  return page < 0 ? nullptr : s.base + 2 * at;
}

// All stages' codewords of the slice in LDS (M K rows of 64 L bytes), kept while
// the workgroup goes through chunks of the tokens, its own of the launch's
// `ranges`.  L lanes share a token, each with 8 dimensions of the lower half
// and the 8 they are turned with: two codes and four 16-byte gathers a stage.
// L = 8 for heads of 128 and more, so that a workgroup writes whole 128-byte
// lines (L = 4, 64-byte pieces of a line from two workgroups: 182 us against
// 129 for 4 x <= 32768 tokens x 1024 of 1 bit, of which 67 without the
// stores).  The four groups of columns of an LDS row are permuted by the
// codeword's index, so that tokens' gathers, which want the same columns, meet
// less in a bank.  Angles: position = chunk + 128 slot + row; the row's rotation
// stays in registers, the chunk's slots' go through LDS, so that a sine is
// computed per 128 tokens; c and s carry 15 roundings.
constexpr int PR_ROWS = 128;
constexpr int PR_SLOTS = 4;
constexpr int PR_CHUNK = PR_ROWS * PR_SLOTS;
constexpr int PR_TABLE = 128 * 1024;        // bytes of codewords, at most

template <typename TP, int M, int L>
__global__ void __launch_bounds__(PR_ROWS* L, M == 1 ? 4 : 2)
    paged_decode_lds_kernel(RestoreArgs a, int nsub, int ranges) {
  constexpr int THREADS = PR_ROWS * L, HALF = 8 * L, COLS = 4 * L;
  extern __shared__ __align__(16) f4 tab[];                 // [M][K][COLS]
  __shared__ float2 turns[2][PR_SLOTS][HALF];
  const int tid = threadIdx.x, l = tid % L, rg = tid / L;
  const Slice s = slice_of<TP, HALF>(a, blockIdx.x % nsub);
  const int per = (a.cap + PR_CHUNK - 1) / PR_CHUNK;
  CodeBits bx[M], by[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    bx[m] = code_bits(a, m, (s.lo + 8 * l) / a.d);
    by[m] = code_bits(a, m, (s.hi + 8 * l) / a.d);
  }
  // the next chunk with tokens from chunk c on, and what it needs from memory,
  // which is read while the one before is at work: pages and codes (of the
  // lower and of the upper half)
  const int64_t end = (int64_t)per * a.pool.B;
  int64_t c = blockIdx.x / nsub;
  int next_t0 = 0, next_len = 0, next_entry[PR_SLOTS];
  uint32_t next_x[PR_SLOTS][M], next_y[PR_SLOTS][M];
  auto read = [&]() __attribute__((always_inline)) {
    int b = 0;
    for (; c < end; c += ranges) {
      b = (int)(c / per);
      next_t0 = (int)(c - (int64_t)b * per) * PR_CHUNK;
      next_len = min(a.seq_len[b], a.cap);
      if (next_t0 < next_len) break;
    }
    if (c >= end) return;
    const uint32_t* rows = s.codes + ((int64_t)b * a.cap + next_t0) * a.words;
    by_crossing(a, [&](auto cross) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < PR_SLOTS; ++u) {
        const int r = min(PR_ROWS * u + rg, next_len - 1 - next_t0);
        next_entry[u] = entry_of(a.pool, b, next_t0 + r);
        const uint32_t* row = rows + (uint32_t)r * (uint32_t)a.words;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          next_x[u][m] = read_code<decltype(cross)::value>(a, row, bx[m]);
          next_y[u][m] = read_code<decltype(cross)::value>(a, row, by[m]);
        }
      }
    });
  };
  read();
  if (c >= end) return;
  for (int i = tid; i < M * a.K * COLS; i += THREADS) {
    const int m = i / COLS / a.K, k = i / COLS - m * a.K, col = i % COLS;
    const int q = col / L ^ (k & 3);                        // lower 0, 1, upper 2, 3
    tab[i] = codeword4(a, s, m, k, (q < 2 ? s.lo : s.hi) + 8 * (col % L) + 4 * (q & 1));
  }
  float cr[8], sr[8];
  if (s.turn) {
#pragma unroll
    for (int j = 0; j < 8; ++j) turn_of(rg, a.theta[s.first + 8 * l + j], cr[j], sr[j]);
  }
  __syncthreads();
  for (int buf = 0; c < end; buf ^= 1) {
    const int t0 = next_t0, len = next_len;
    int entry[PR_SLOTS];
    uint32_t cx[PR_SLOTS][M], cy[PR_SLOTS][M];
#pragma unroll
    for (int u = 0; u < PR_SLOTS; ++u) {
      entry[u] = next_entry[u];
#pragma unroll
      for (int m = 0; m < M; ++m) {
        cx[u][m] = next_x[u][m];
        cy[u][m] = next_y[u][m];
      }
    }
    if (s.turn) {
      if (tid < HALF * PR_SLOTS) {
        float2 x;
        turn_of(t0 + PR_ROWS * (tid / HALF), a.theta[s.first + tid % HALF], x.x, x.y);
        turns[buf][tid / HALF][tid % HALF] = x;
      }
      __syncthreads();
    }
    c += ranges;
    read();
#pragma unroll
    for (int u = 0; u < PR_SLOTS; ++u) {
      const int t = t0 + PR_ROWS * u + rg;
      float x[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = y[j] = 0.f;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int kx = code_of(a, cx[u][m], bx[m]), ky = code_of(a, cy[u][m], by[m]);
        const f4* tx = tab + (m * a.K + kx) * COLS + l;
        const f4* ty = tab + (m * a.K + ky) * COLS + l;
        const f4 x0 = tx[L * (kx & 3)], x1 = tx[L * ((kx & 3) ^ 1)];
        const f4 y0 = ty[L * ((ky & 3) ^ 2)], y1 = ty[L * ((ky & 3) ^ 3)];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] += x0[j];
          x[4 + j] += x1[j];
          y[j] += y0[j];
          y[4 + j] += y1[j];
        }
      }
      if (s.turn) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 w = turns[buf][u][8 * l + j];
          const float cc = cr[j] * w.x - sr[j] * w.y, ss = sr[j] * w.x + cr[j] * w.y;
          const float v = x[j], z = y[j];
          x[j] = v * cc - z * ss;
          y[j] = z * cc + v * ss;
        }
      }
      const bool held = t < len && in_table(a.pool, t);
      char* dst = token_at(a, s, held ? checked(a.pool, entry[u]) : -1, t);
      if (dst) {
        store8((TP*)dst + 8 * l, x);
        store8((TP*)dst + a.hd / 2 + 8 * l, y);
      }
    }
  }
}

// More stages than LDS holds: a chunk of 64 S tokens keeps its sums in
// registers and goes through the stages; a stage's codewords (64 dimensions)
// are written to one LDS buffer while the tokens gather from the other.
// Sixteen lanes share a token, four dimensions each (the first eight the lower
// half), so that a gather touches every bank once, whatever the codes: with
// eight lanes a token and slices of 32 dimensions the gathers alone took 85 us
// for 3 x <= 10007 tokens x 1024 of 12 stages.  SHARE lanes have one code (4
// where d >= 16, all 16 where the slice lies in one subspace): each of them
// holds that of one stage of SHARE, which a DPP broadcast hands out when its
// turn comes, so that codes, whose loads are waited for, are read once in
// SHARE stages (12 stages: 127 us with 4 lanes, 115 with 16).
constexpr int PS_THREADS = 1024;
constexpr int PS_ROWS = PS_THREADS / 16;
constexpr int PS_K = 256;
constexpr int PS_BUF = PS_K * 16;           // f4 per buffer

template <typename TP, int S, int SHARE>
__global__ void __launch_bounds__(PS_THREADS) paged_row_decode_stages_kernel(RestoreArgs a,
                                                                             int nsub) {
  __shared__ __align__(16) f4 tab[2][PS_BUF];
  __shared__ float2 slot_turn[S][32], row_turn[PS_ROWS][32];
  const int tid = threadIdx.x, l = tid & 15, rg = tid >> 4;
  const int per = (a.cap + PS_ROWS * S - 1) / (PS_ROWS * S);
  const Slice s = slice_of<TP, 32>(a, blockIdx.x % nsub);
  const int chunk = blockIdx.x / nsub;
  const int b = chunk / per, t0 = (chunk - b * per) * PS_ROWS * S;
  const int len = min(a.seq_len[b], a.cap);
  if (t0 >= len) return;
  // (of this chunk alone: all that are left times their words would not fit
  // 32 bits in long contexts)
  const int nrows = min(len - t0, PS_ROWS * S);
  const int e = (l < 8 ? s.lo : s.hi - 32) + 4 * l, g = e / a.d;
  constexpr int PER = PS_BUF / PS_THREADS;
  f4 v[PER];
  float gk[PER];
  auto load = [&](int m) __attribute__((always_inline)) {
    const float* gb = s.gain + ((int64_t)m * a.G + g) * a.K;
    const float* sb = s.shape + ((int64_t)m * a.G + g) * a.K * a.d + (e - g * a.d);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const uint32_t k = (uint32_t)min(u * PS_ROWS + rg, a.K - 1);
      gk[u] = gb[k];
      v[u] = *(const f4*)(sb + k * (uint32_t)a.d);
    }
  };
  f4 acc[S];
#pragma unroll
  for (int u = 0; u < S; ++u) acc[u] = (f4){0.f, 0.f, 0.f, 0.f};
  int code[S];
  const uint32_t* rows = s.codes + ((int64_t)b * a.cap + t0) * a.words;
  const uint32_t words = (uint32_t)a.words, last_word = (nrows - 1) * words;
  load(0);
  if (s.turn) {
    for (int i = tid; i < 32 * (S + PS_ROWS); i += PS_THREADS) {
      const bool slot = i < 32 * S;
      const int r = slot ? i >> 5 : (i >> 5) - S;
      float2 x;
      turn_of(slot ? t0 + PS_ROWS * r : r, a.theta[s.first + (i & 31)], x.x, x.y);
      (slot ? slot_turn[r] : row_turn[r])[i & 31] = x;
    }
  }
  for (int m = 0; m < a.M; ++m) {
    f4* from = tab[m & 1];
    if (m % SHARE == 0) {
      // (the row opaque: addresses are formed here, not kept across stages)
      uint32_t first_word = rg * words;
      asm volatile("" : "+v"(first_word));
      const int mm = min(m + l % SHARE, a.M - 1);
      const int64_t bit = ((int64_t)mm * a.G + g) * a.b;
      const CodeBits at = {bit >> 5, (int)(bit & 31)};
      by_crossing(a, [&](auto cross) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < S; ++u)
          code[u] = (int)read_code<decltype(cross)::value>(
              a, rows + min(first_word + u * PS_ROWS * words, last_word), at);
      });
#pragma unroll
      for (int u = 0; u < S; ++u) code[u] = code_of(a, (uint32_t)code[u], at) * 256;
    }
    {
#pragma clang fp contract(off)
#pragma unroll
      for (int u = 0; u < PER; ++u) from[u * PS_THREADS + tid] = gk[u] * v[u];
    }
    if (m + 1 < a.M) load(m + 1);
    // one barrier a stage: who writes stage m + 2 over this buffer has passed
    // stage m + 1's, which all reach only after their gathers of stage m
    __syncthreads();
    const char* const mine = (const char*)(from + l);
#pragma unroll
    for (int u = 0; u < S; ++u) {
      int k = code[u];                    // in bytes
      // the first of the lanes' codes, and on by one
      if (SHARE == 4) {
        k = __builtin_amdgcn_update_dpp(0, code[u], 0x00, 0xf, 0xf, true);
        code[u] = __builtin_amdgcn_update_dpp(0, code[u], 0x39, 0xf, 0xf, true);
      } else if (SHARE == 16) {
        k = __builtin_amdgcn_update_dpp(0, code[u], 0x150, 0xf, 0xf, true);
        code[u] = __builtin_amdgcn_update_dpp(0, code[u], 0x12f, 0xf, 0xf, true);
      }
      acc[u] += *(const f4*)(mine + k);
    }
  }
  int entry[S];                           // all read at once
#pragma unroll
  for (int u = 0; u < S; ++u) entry[u] = entry_of(a.pool, b, t0 + min(u * PS_ROWS + rg, nrows - 1));
  float cr[4], sr[4];
  if (s.turn) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 w = row_turn[rg][4 * (l & 7) + j];
      cr[j] = w.x;
      sr[j] = w.y;
    }
  }
#pragma unroll
  for (int u = 0; u < S; ++u) {
    const int t = t0 + u * PS_ROWS + rg;
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = acc[u][j];
    if (s.turn) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // the element that this one is turned with: eight lanes on
        const float z = __uint_as_float(
            __builtin_amdgcn_update_dpp(0u, __float_as_uint(acc[u][j]), 0x128, 0xf, 0xf, true));
        const float2 w = slot_turn[u][4 * (l & 7) + j];
        const float cc = cr[j] * w.x - sr[j] * w.y, ss = sr[j] * w.x + cr[j] * w.y;
        x[j] = x[j] * cc + (l < 8 ? -z : z) * ss;
      }
    }
    char* dst = token_at(a, s, t < len && in_table(a.pool, t) ? checked(a.pool, entry[u]) : -1, t);
    if (!dst) continue;
    typedef TP v4 __attribute__((ext_vector_type(4)));
    v4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (TP)x[j];
    *(v4*)((TP*)dst + (l < 8 ? 0 : a.hd / 2 - 32) + 4 * l) = r;
  }
}

// Codebooks of more codewords than the kernels above hold in LDS: a lane per 16
// elements of a head of one token's key or value row, codewords from memory.
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

template <typename TP, int M, int L>
gsrq_status restore_resident(const RestoreArgs& a, hipStream_t st) {
  const int64_t B = a.pool.B, nsub = 2ll * a.pool.Hkv * (a.hd / (16 * L));
  const int64_t table = (int64_t)M * a.K * 64 * L;
  // two workgroups per CU where two tables fit, each with its share of the chunks
  const int64_t chunks = B * ((a.cap + PR_CHUNK - 1) / PR_CHUNK);
  const int64_t wgs = table <= PR_TABLE / 2 ? 512 : 256;
  const int64_t ranges = std::max<int64_t>(1, std::min(wgs / nsub, chunks));
  if (nsub * ranges > (1 << 22) - 1) return GSRQ_E_UNSUPPORTED;   // of up to 1024 threads
  auto kern = paged_decode_lds_kernel<TP, M, L>;
  if (table > 65536 - 4096 &&
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)table) != hipSuccess)
    return GSRQ_E_HIP;
  kern<<<(unsigned)(nsub * ranges), PR_ROWS * L, (size_t)table, st>>>(a, (int)nsub, (int)ranges);
  return launch_ok();
}

template <typename TP> gsrq_status restore_launch(const RestoreArgs& a, hipStream_t st) {
  const int64_t B = a.pool.B, nsub = 2ll * a.pool.Hkv * (a.hd / 64);
  const int L = a.hd == 64 ? 4 : 8;
  // (rows of codes so long that a chunk's do not fit 32 bits: from memory)
  const bool near = a.words <= 1 << 20;
  if (near && a.M <= (L == 4 ? 2 : 1) && (int64_t)a.M * a.K * 64 * L <= PR_TABLE) {
    if (L == 8) return restore_resident<TP, 1, 8>(a, st);
    return a.M == 1 ? restore_resident<TP, 1, 4>(a, st) : restore_resident<TP, 2, 4>(a, st);
  }
  if (near && a.K <= PS_K) {
    // chunks of 640 tokens (fewer fills of the stages' buffers) where they
    // give every CU a workgroup, else of 128, which start more workgroups on few
    // tokens.  One sequence, 8 heads of 128, 12 stages, chunks of 128 against
    // 640: 600 tokens 14 us and 20, 1280 tokens 27 and 21, 5100 tokens (256 long
    // chunks) 61 and 22.  Long chunks win before that where the cache is full,
    // but `cap` is all that is known here: three sequences of 460 to 1387
    // tokens, 2 heads, took 14 us and 20.
    constexpr int LONG = 10, SHORT = 2;
    const int64_t longs = nsub * B * ((a.cap + PS_ROWS * LONG - 1) / (PS_ROWS * LONG));
    const int64_t shorts = nsub * B * ((a.cap + PS_ROWS * SHORT - 1) / (PS_ROWS * SHORT));
    const bool is_long = longs >= 256;
    const int64_t blocks = is_long ? longs : shorts;
    if (blocks > (1 << 22) - 1) return GSRQ_E_UNSUPPORTED;
    const unsigned n = (unsigned)blocks;
    const int i = (int)nsub;
    auto launch = [&](auto kern) { kern<<<n, PS_THREADS, 0, st>>>(a, i); };
    if (is_long) {
      if (a.d >= a.hd) launch(paged_row_decode_stages_kernel<TP, LONG, 16>);
      else if (a.d >= 16) launch(paged_row_decode_stages_kernel<TP, LONG, 4>);
      else launch(paged_row_decode_stages_kernel<TP, LONG, 1>);
    } else {
      if (a.d >= a.hd) launch(paged_row_decode_stages_kernel<TP, SHORT, 16>);
      else if (a.d >= 16) launch(paged_row_decode_stages_kernel<TP, SHORT, 4>);
      else launch(paged_row_decode_stages_kernel<TP, SHORT, 1>);
    }
    return launch_ok();
  }
  const int64_t items = (int64_t)a.cap * a.pool.Hkv * (a.hd / 16);
  const int64_t blocks = (items + PA_THREADS - 1) / PA_THREADS;
  if (blocks > MAX_BLOCKS || B > 65535) return GSRQ_E_UNSUPPORTED;
  paged_row_decode_kernel<TP>
      <<<dim3((unsigned)blocks, 2, (unsigned)B), PA_THREADS, 0, st>>>(a);
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
  if (cap > 1 << 30) return GSRQ_E_UNSUPPORTED;       // (no table holds more)
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
  hipStream_t st = (hipStream_t)stream;
  TimedLaunch tl(GSRQ_KERNEL_DECODE, st);
  return pages->dtype == GSRQ_F16 ? restore_launch<_Float16>(a, st) : restore_launch<__bf16>(a, st);
}

}  // extern "C"
