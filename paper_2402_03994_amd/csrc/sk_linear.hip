// sk_linear.hip -- log-probabilities of tokens from hidden states and the output
// matrix, with both gradients, over pieces of the vocabulary (C ABI of
// include/sketch_train.h).
//
// Logits x = H W^T are formed tile by tile in the matrix cores' accumulators and
// never kept.  Forward: each tile leaves its (m, z) (largest logit, sum of
// exp(scale (x - m))) per token, k_join joins them.  Gradient: the logits of a
// piece of the vocabulary are formed again, become
// G = dlogp scale (onehot - p) in the tile's epilogue, and the piece adds G W to
// dH and gives its rows G^T H of dW:
//   8 n V d operations for n tokens, of which 2 n V d are the second forming.
// Rows whose target is masked are left out of everything: k_front (k_live, of many
// rows) lists the live ones, each example's padded with empty rows to a multiple of 16.
//
// All three products are one kernel core, C[m][n] = sum_k A[m][k] B[n][k], which
// takes its operands as they lie, with K along their rows or across them (Side
// and Core below).  16-bit operands, fp32 sums.
//   bf16 inputs are used as they are, and G is rounded to bf16, once, like any
//   entry of a bf16 gradient (of few rows it takes two bf16: kPairRows).  What the
//   rounding of a target's entry, most of its row of G, has left is returned to
//   both gradients.
//   fp32 inputs are split, x = hi + lo in two fp16 numbers (22 bits) under a power
//   of two that brings the largest to 2^13, and each product is the three hi lo,
//   lo hi, hi hi: a large library product reaches 153 TFLOP/s in fp32, 1256 in
//   fp16.  What lo cannot hold is below 2^-38 of the largest entry of the row.  G
//   is split under powers of two of its own for each of its products (Powers
//   below), so that a vocabulary entry that no token finds likely, and an example
//   whose factors are small, keep their bits.
//
// What bounds it: the products, at the rate that their operands leave the caches
// (the figures are at Tiling); below some hundred rows the reads of W; below those
// the launches.  One MI355X, both calls: 4096 x 50257 x 768 bf16 (40% masked) 884 us,
// 8192 x 128256 x 4096 19.5 ms (790 TFLOP/s of the 6 n V d, 1060 with the logits
// that are formed again); 8 examples of 257 x 50257 x 768 fp32 1680 us.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "sk_train.h"

using namespace sk;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;   // K a stage
constexpr int kPad = 16;    // an example's rows in the list come in multiples of it
constexpr int kTop = 13;    // split operands lie below 2^(kTop + 1)
[[maybe_unused]] constexpr int kNone = INT_MIN / 2;  // the exponent of nothing
// Split entries of G lie below 2^(kTopG + 1), in a product below 2^(kTopG + 1 + kSlack)
[[maybe_unused]] constexpr int kTopG = 12, kSlack = 2;

// What the kernels of a call share in its workspace.
struct Meta {
  int np;  // listed rows
};

// A listed row in the gradient: G = one [v = target] + w exp(scale (x - m)).  A row that only fills the list, or has no logit
// above -inf, has m = inf, w = one = 0.
struct RowPrm {
  float m, w, one;  // fp32: without the factor dlogp scale, which is in cs
};

__device__ __forceinline__ int exponent_of(uint32_t bits) { return (int)((bits >> 23) & 255) - 127; }
__device__ __forceinline__ int exponent_of(float x) { return exponent_of(__float_as_uint(x)); }

// What the operands of a product are: bf16; G in two bf16, beside bf16; all in two fp16.
enum Mode { kBf16, kPair, kSplit };
// G of bf16 inputs takes two numbers up to so many rows, where the reads of W count and not the products; and where dW is
// wanted in fp32, up to so many rows of an example, whatever the others: there few tokens make a row of dW, and what their
// number costs in precision would show (gradients of 16 examples of 200 x 50257 x 768 868 us, 1225 us so; of 8 of 250 x 32000
// x 2048 816 and 1274 us).
constexpr int kPairRows = 256;

// hi (low half) and lo of x (kSplit: |x| < 2^15)
template <Mode M>
__device__ __forceinline__ uint32_t split(float x) {
  if (M != kSplit) {
    const uint32_t h = bf16_bits(x);
    if (M == kBf16) return h;
    const float r = x - to_f32(bf16{(uint16_t)h});
    return h | bf16_bits(r == r ? r : 0.0f) << 16;  // of an infinity hi is all
  }
  const _Float16 h = (_Float16)x;
  const float r = x - (float)h;
  const _Float16 l = (_Float16)(r == r ? r : 0.0f);
  return (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
}
// plane p of two of them, side by side
template <Mode M>
__device__ __forceinline__ uint32_t two(float a, float b, int p) {
  return __builtin_amdgcn_perm(split<M>(b), split<M>(a), p ? 0x07060302 : 0x05040100);
}

// Split operands keep 32 hi and the 32 lo that belong to them side by side, a line of 128 bytes: the place of number p of
// column k in a row.
__device__ __forceinline__ int64_t split_at(int64_t k, int p) { return (k >> 5) * 64 + p * 32 + (k & 31); }

// Powers of two of a split G.  The other operand's row at column k has left its own power to the entries of that column.
//   kRows (dW): G's entries may be anything from 1 down.  16 columns (tokens of one example: they come in multiples of 16)
//   of a row (an entry of the vocabulary) share the power of the largest of them; the product brings each group to that of
//   the largest that its row has had.  What is lost lies below 2^-37 of the row's largest entry.
//   kBlocks (dH): G is a fixed-point number beside 1; 64 columns (entries of the vocabulary) of all rows share the power of
//   the largest row of W among them, in steps of 2^4, so that the powers of most weights are all the same.
enum Scaling { kPlain, kRows, kBlocks };
struct Powers {
  const int *p;  // exponents [K / 16][rows], [K / 64]
  int64_t ld;
};
[[maybe_unused]] constexpr int kCoarse = 4;
// What the rounding of the targets' entries of G in bf16 has left, as another term of dW: rest[k] stands in the row of entry
// tgt[k] of the vocabulary.  marks, [rows / 64][K / 32], say where there is one: few stages of a tile.
struct Rest {
  const int *tgt;
  const float *rest;
  const uint8_t *marks;  // of the tile's first row and the matrix's first k
  int64_t ld;
  int first, k0;  // entry of the vocabulary and k that the tile begins with
};

// N elements of a row from column k on, zeros past the width
template <int N, typename T>
__device__ __forceinline__ void row_part(const T *row, int k, int width, float *f) {
  if (k + N <= width) {
#pragma unroll
    for (int i = 0; i < N; i += Vec<T>::N) {
      const u32x4 v = Vec<T>::load(row + k + i);
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) f[i + e] = Vec<T>::get(v, e);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = k + i < width ? to_f32(row[k + i]) : 0.0f;
  }
}

// --- the list of rows ---------------------------------------------------------------------------------------
// a wave's largest finite |x| of a row, as its exponent
template <typename T>
__device__ __forceinline__ int row_exponent(const T *row, int width) {
  const int lane = threadIdx.x & 63;
  float big = 0.0f;
  for (int k = lane * 8; k < width; k += 1024) {
    float f[8], g[8];
    row_part<8>(row, k, width, f);
    row_part<8>(row, k + 512, width, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      big = fmaxf(big, fabsf(f[i]) < INFINITY ? fabsf(f[i]) : 0.0f);
      big = fmaxf(big, fabsf(g[i]) < INFINITY ? fabsf(g[i]) : 0.0f);
    }
  }
  return exponent_of(wave_all(big, OpMax()));
}

struct Live {
  const void *targets;
  const float *dlogp;  // NULL: forward
  int32_t index, vocab, n, batch;
  int *list, *pos, *tgt, *seg, *cnt;
  Meta *meta;
  float *logp;
  float2 *stats;
};

__device__ __forceinline__ int wave_scan(int v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}

// the row (-1: none) and target (-1: masked) of this lane in chunk c; an example has `per` of them
__device__ __forceinline__ void fetch(const Live &a, int per, int chunks, int c, int &t, int &v) {
  const int i = c % per * 64 + (threadIdx.x & 63);
  t = c < chunks && i < a.n ? c / per * a.n + i : -1;
  int64_t id = -1;
  float d = 1.0f;
  if (t >= 0) {
    id = a.index == SK_I64 ? ((const int64_t *)a.targets)[t] : ((const int32_t *)a.targets)[t];
    if (a.dlogp) d = a.dlogp[t];
  }
  v = id >= 0 && id < a.vocab && d != 0.0f ? (int)id : -1;
}

__device__ __forceinline__ void masked(const Live &a, int row) {
  a.pos[row] = -1;
  if (a.logp) {
    a.logp[row] = 0.0f;
    if (a.stats) a.stats[row] = float2{0.0f, 0.0f};
  }
}

// Counts of 64 rows each, their sums within the examples, the examples' starts, the list.  A wave has four chunks of 64 rows
// under way (8192 rows: 17 us one after another, 14.5 us so).
__global__ __launch_bounds__(1024) void k_live(Live a) {
  constexpr int U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (a.n + 63) / 64, chunks = per * a.batch;
  for (int c0 = wave * U; c0 < chunks; c0 += 16 * U) {
    int t[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(a, per, chunks, c0 + u, t[u], v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint64_t live = __ballot(v[u] >= 0);
      if (lane == 0 && c0 + u < chunks) a.cnt[c0 + u] = __popcll(live);
    }
  }
  __syncthreads();
  for (int b = wave; b < a.batch; b += 16) {
    int sum = 0;
    for (int i = 0; i < per; i += 64) {
      int *p = a.cnt + b * per + i + lane;
      const int v = i + lane < per ? *p : 0, s = wave_scan(v, lane);
      if (i + lane < per) *p = sum + s - v;
      sum += __shfl(s, 63, 64);
    }
    if (lane == 0) a.seg[b + 1] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    int sum = 0;
    for (int b = 0; b < a.batch; b += 64) {
      const int v = b + lane < a.batch ? (a.seg[b + 1 + lane] + kPad - 1) / kPad * kPad : 0;
      const int s = wave_scan(v, lane) + sum;
      if (b + lane < a.batch) a.seg[b + 1 + lane] = s;
      sum = __shfl(s, 63, 64);
    }
    if (lane == 0) {
      a.seg[0] = 0;
      a.meta->np = sum;
    }
  }
  __syncthreads();
  for (int c0 = wave * U; c0 < chunks; c0 += 16 * U) {
    int t[U], v[U], at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fetch(a, per, chunks, c0 + u, t[u], v[u]);
      at[u] = c0 + u < chunks ? a.seg[(c0 + u) / per] + a.cnt[c0 + u] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint64_t live = __ballot(v[u] >= 0);
      if (v[u] >= 0) {
        const int p = at[u] + __popcll(live & ((1ull << lane) - 1));
        a.list[p] = t[u];
        a.tgt[p] = v[u];
        a.pos[t[u]] = p;
      } else if (t[u] >= 0) {
        masked(a, t[u]);
      }
      if (c0 + u < chunks && (c0 + u) % per == per - 1)
        for (int p = at[u] + __popcll(live) + lane; p < a.seg[(c0 + u) / per + 1]; p += 64) a.list[p] = a.tgt[p] = -1;
    }
  }
}

// --- operands -----------------------------------------------------------------------------------------------
struct Gather {
  const void *hidden;
  int64_t ld;
  int width, kp;
  const int *list;
  Meta *meta;
  uint16_t *hc;
  int *eh;
  // gradient only
  const float2 *stats;
  const float *dlogp;
  float scale;
  RowPrm *prm;
  float *cs;
};

// Row t of H at place n of the list (t < 0: a row of zeros), zeros to a width of kp, by a wave.  fp32: the row's exponent,
// its split; in the gradient what that needs to know of it.
template <typename T>
__device__ __forceinline__ void gather(const Gather &a, int n, int t) {
  const int lane = threadIdx.x & 63;
  const T *row = (const T *)a.hidden + (int64_t)(t < 0 ? 0 : t) * a.ld;
  const int width = t < 0 ? 0 : a.width;
  uint16_t *hc = a.hc + (int64_t)n * a.kp * (sizeof(T) == 4 ? 2 : 1);
  int e = 0;
  if (sizeof(T) == 4) {
    e = row_exponent(row, width);
    if (lane == 0) a.eh[n] = e;
  }
  for (int k = lane * 8; k < a.kp; k += 512) {
    float f[8];
    row_part<8>(row, k, width, f);
    if (sizeof(T) == 4) {
      u32x4 h, l;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = ldexpf(f[i], kTop - e);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = two<kSplit>(f[2 * i], f[2 * i + 1], 0);
        l[i] = two<kSplit>(f[2 * i], f[2 * i + 1], 1);
      }
      *(u32x4 *)(hc + split_at(k, 0)) = h;
      *(u32x4 *)(hc + split_at(k, 1)) = l;
    } else {
      *(u32x4 *)(hc + k) = Vec<bf16>::pack(f);
    }
  }
  if (!a.prm) return;
  RowPrm p{INFINITY, 0.0f, 0.0f};
  float c = 0.0f;
  if (t >= 0) {
    const float2 s = a.stats[t];
    if (s.y != 0.0f) {
      c = a.dlogp[t] * a.scale;
      p.m = s.x;
      p.one = sizeof(T) == 4 ? 1.0f : c;
      p.w = -p.one / s.y;
    }
  }
  if (lane == 0) {
    if (sizeof(T) == 4) a.cs[n] = c;
    a.prm[n] = p;
  }
}

// a wave a row
template <typename T>
__global__ __launch_bounds__(256) void k_gather(Gather a) {
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.meta->np) return;
  gather<T>(a, n, a.list[n]);
}

struct Prep {
  const void *src;
  int64_t ld;
  int rows, width, kp;  // what there is, zeros up to kp columns
  int *ev;  // W in fp32: exponents of its rows, which bring their own powers of two
  uint16_t *out;  // [..][kp] numbers
};

// Rows of W as an operand takes them: padded with zeros to kp columns, fp32 split.  A wave a row, up to a multiple of 64 rows;
// `block` counts groups of WAVES rows.
template <typename T, int WAVES>
__device__ __forceinline__ void prep(const Prep &a, int block) {
  constexpr int P = sizeof(T) == 4 ? 2 : 1;
  const int r = block * WAVES + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= (a.rows + 63) / 64 * 64) return;
  const T *row = (const T *)a.src + (r < a.rows ? r : 0) * a.ld;
  const int width = r < a.rows ? a.width : 0;
  int e = 0;
  if (P == 2) {
    e = row_exponent(row, width);
    if (lane == 0) a.ev[r] = e;
  }
  uint16_t *out = a.out + (int64_t)r * a.kp * P;
  for (int k = lane * 8; k < a.kp; k += 512) {
    float f[8];
    row_part<8>(row, k, width, f);
    if (P == 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = ldexpf(f[i], kTop - e);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      u32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = two<P == 2 ? kSplit : kBf16>(f[2 * i], f[2 * i + 1], p);
      *(u32x4 *)(out + (P == 2 ? split_at(k, p) : k)) = v;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_prep(Prep a) {
  prep<T, 4>(a, blockIdx.x);
}

// The list, H's rows and W's in one launch, for up to 64 chunks of 64 rows: each workgroup counts the live rows by itself and
// takes 16 rows of a chunk, a wave each.  `blocks` of those; the workgroups behind them prepare W.  Beside k_live, k_gather and
// k_prep one after another: 61 x 8000 x 250 fp32 with gradients 78.7 us, 68.1 us so; 2000 x 50257 x 768 fp32 345 and 329 us;
// 4096 x 50257 x 768 bf16 with gradients 868 and 855 us.
struct Front {
  Live l;
  Gather g;
  Prep w;
  int blocks;
};
constexpr int kFrontChunks = 64;

template <typename T>
__global__ __launch_bounds__(1024) void k_front(Front a) {
  __shared__ int cnt[kFrontChunks], ids[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x >= a.blocks) {
    prep<T, 16>(a.w, blockIdx.x - a.blocks);
    return;
  }
  constexpr int U = kFrontChunks / 16;
  const int per = (a.l.n + 63) / 64, chunks = per * a.l.batch, mine = blockIdx.x >> 2;
  int t[U], v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) fetch(a.l, per, chunks, wave * U + u, t[u], v[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = wave * U + u;
    const uint64_t live = __ballot(v[u] >= 0);
    if (lane == 0) cnt[c] = __popcll(live);
    if (c == mine) ids[lane] = v[u];
  }
  __syncthreads();
  // lane c: live rows before the end of chunk c; lane b: places before the end of example b
  const int sum = wave_scan(cnt[lane], lane), before = sum - cnt[lane];
  const int all = __shfl(sum, min(lane * per + per - 1, 63), 64) - __shfl(before, min(lane * per, 63), 64);
  const int ends = wave_scan(lane < a.l.batch ? (all + kPad - 1) / kPad * kPad : 0, lane);
  const int ex = mine / per, end = __shfl(ends, ex, 64);
  const int at = (ex ? __shfl(ends, ex - 1, 64) : 0) + __shfl(before, mine, 64) - __shfl(before, ex * per, 64);
  if (blockIdx.x == 0 && wave == 0) {
    if (lane < a.l.batch) a.l.seg[lane + 1] = ends;
    if (lane == 0) a.l.seg[0] = 0;
    if (lane == 63) a.l.meta->np = ends;
  }
  const int r = (blockIdx.x & 3) * 16 + wave, i = mine % per * 64 + r;
  const uint64_t live = __ballot(ids[lane] >= 0);
  if (i < a.l.n) {
    const int row = ex * a.l.n + i, target = ids[r];
    if (target >= 0) {
      const int p = at + __popcll(live & ((1ull << r) - 1));
      if (lane == 0) {
        a.l.list[p] = row;
        a.l.tgt[p] = target;
        a.l.pos[row] = p;
      }
      gather<T>(a.g, p, row);
    } else if (lane == 0) {
      masked(a.l, row);
    }
  }
  if ((int)blockIdx.x % (4 * per) == 4 * per - 1) {  // an example's last: the rows that only fill the list
    const int p = at + __popcll(live) + wave;
    if (p < end) {
      if (lane == 0) a.l.list[p] = a.l.tgt[p] = -1;
      gather<T>(a.g, p, -1);
    }
  }
}

// --- the product --------------------------------------------------------------------------------------------
// Rows of an operand, K or the operand's rows contiguous; kPair: G's lo in a matrix of its own.
struct Operand {
  const uint16_t *p[2];
  int64_t ld;  // 16-bit numbers
};

// A BM x BN tile by WM x WN waves, each (BM / WM) x (BN / WN) in 32 x 32 accumulators of v_mfma_f32_32x32x16.  Stages of
// 64 of K go straight from memory to LDS, 16 bytes a lane, two stages deep: the loads of the next one are issued
// behind the barrier that frees its buffer and have the products of a whole stage to arrive.  Two workgroups share a
// CU, so that one's epilogue lies beside the other's products.  Alone (8192^3, and 16384 x 2560 x 768, bf16): 128 x 192
// 1150 and 803 TFLOP/s, 128 x 128 1108 and 773, one 256 x 256 a CU 1240 and 729, the library's 1290 and 817.  In the
// operators (4096 x 50257 x 768 and 8192 x 128256 x 4096): log-probabilities 225 us and 4.47 ms with 128 x 192, 243 us and
// 5.0 ms with 128 x 128, 226 us and 4.5 ms with 256 x 256.  Up to 1024 rows the smaller tiles fill the chip better
// (gradients of 200 x 50257 x 768: 134 us, 146 with the larger ones; 1000: 301 and 299).
template <int BM_, int BN_, int WM_, int WN_>
struct Tiling {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NW = WM * WN, TH = NW * 64;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static constexpr int LDS = 2 * (BM + BN) * kStep * 2;
};
using Large = Tiling<128, 192, 2, 2>;
using Small = Tiling<128, 128, 2, 2>;
using Narrow = Tiling<128, 64, 2, 2>;  // logits of up to 64 rows (61 x 8000 x 250 fp32, both calls: 67.2 us with Small, 62.4 us so)
using Huge = Tiling<256, 256, 2, 4>;
constexpr int64_t kSmallRows = 1024;  // rows up to which the smaller tiles are taken
// Where the gradients' products have both rows and tiles in plenty, one 256 x 256 tile a CU asks for 0.6 times as much
// of the caches (which the products miss by the distance their tiles drift apart: 5 TB/s at 8192 x 128256 x 4096): 15.1
// ms, 14.1 ms there; 4096 x 50257 x 4096 3.09 and 2.87 ms; 8000 x 32000 x 5000 fp32 14.6 and 13.8 ms.  With fewer tiles
// than four rounds of the chip, or short sums, it loses as much (16384 x 50257 x 1024: 3.53 and 3.95 ms; four examples
// of 512 x 50257 x 4096 2.12 and 2.35 ms).
constexpr int64_t kHugeRows = 4096, kHugeTiles = 1024;

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((address_space(3))) void *lds_ptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

// Four columns of 16 lanes, transposed.  __restrict__ tells the compiler that the loads to LDS that are under way write
// elsewhere (the barriers see to that): without it it waits for them before each read (8192 x 128256 x 4096 bf16: 20.6 ms,
// 19.7 ms so).
__device__ __forceinline__ s16x4 read_tr(const lds_s16x4 __restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }

// One operand of a tile, N of its rows, by TH threads of which a wave multiplies N / W rows.  A stage is 64 numbers of each
// row: 64 of K, or (P = 2, split operands) hi and lo of 32 of K.
// KM false: K contiguous.  A stage is N rows of 128 bytes, whose 16-byte chunks are exchanged by row / 2 so that 16 rows
// that are read in a cycle fill the 256 bytes of the banks (exchanged by the row: 8192^3 bf16, 256 x 256, 957 us, 887 us
// so).
// KM true: the matrix has K for its rows and the operand's rows for its columns.  A stage is 64 rows of N columns (32 of
// hi, 32 of lo), which ds_read_b64_tr_b16 transposes: of 16 lanes, lane 4 r + q gives the address of four columns 4 q of row
// r, and lane i gets column i of the four rows.  Chunks are exchanged so that the eight rows of 64 bytes that a wave reads
// at a time fill the banks twice over: rows lie 256 bytes (N = 128), 384 (192) or 512 (256) apart.
template <int N, int W, int TH, bool KM, int P>
struct Side {
  static constexpr int KS = kStep / P;                   // K of a stage
  static constexpr int CH = KM ? N / 8 : kStep / 8;      // chunks of an LDS row
  static constexpr int PASS = KM ? P : 1;                // hi's and lo's rows are loaded apart
  static constexpr int L = N * kStep / 8 / TH / PASS;    // loads of a thread, pass and stage
  static constexpr int T = N / W / 32, LO = N * KS * 2;  // 32 x 32 blocks of a wave; where lo's rows begin (KM)
  static_assert(!KM || N == 128 || N == 192 || N == 256, "exchanges are worked out for these");
  int off[L], ld, depth;

  static __device__ __forceinline__ int swz(int row) {
    return !KM ? (row >> 1) & 7 : N != 192 ? (row & 3) * 4 : ((row >> 1) & 1) * 4;
  }
  // rows: how many there are from the tile's first on (those behind repeat one of them; a multiple of 8 with KM); k: K rows
  // that there are (KM; those behind count as zeros)
  __device__ __forceinline__ void init(const Operand &o, int rows, int k) {
    ld = (int)(o.ld * 2);
    depth = k;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int c = i * TH + threadIdx.x, r = c / CH, s = (c % CH) ^ swz(r);
      if (KM) {
        const int col = min(s * 8, rows - 8);
        off[i] = r * ld + (int)(P == 2 ? split_at(col, 0) : col) * 2;
      } else {
        off[i] = min(r, rows - 1) * ld + s * 16;
      }
    }
  }
  // stage k to LDS; none: zeros (K contiguous)
  __device__ __forceinline__ void load(char *lds, const uint16_t *from, int k, bool none = false) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const char *base = (const char *)from + (KM ? (int64_t)k * ld * KS + p * 64 : (int64_t)k * kStep * 2);
      // K rows that there are not lie past the buffer's end, where loads give zeros
      const int there = KM ? min(depth - k * KS, KS) * ld : __builtin_amdgcn_readfirstlane(none ? 0 : -1);
      const auto m = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, there, 0x00020000);
#pragma unroll
      for (int i = 0; i < L; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(m, (lds_ptr)(lds + p * LO + (i * (TH / 64) + wave) * 1024), 16, off[i], 0, 0, 0);
    }
  }
  // operands of step ks of a stage, number p: rows w N / W + 32 i + lane % 32, K 16 ks + 8 (lane / 32) and on
  __device__ __forceinline__ void read(const char *lds, int w, int ks, int p, u32x4 *f) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < T; ++i) {
      if constexpr (KM) {
        const int r = (lane & 15) >> 2, col = w * (N / W) + i * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        const char *at = lds + p * LO + (ks * 16 + (lane >> 5) * 8 + r) * (N * 2) + ((col >> 3) ^ swz(r)) * 16 + (col & 4) * 2;
        union {
          s16x4 h[2];
          u32x4 v;
        } u;
        u.h[0] = read_tr((lds_s16x4)at);
        u.h[1] = read_tr((lds_s16x4)(at + 4 * N * 2));
        f[i] = u.v;
      } else {
        const int r = lane & 31;
        f[i] = *(const u32x4 *)(lds + (w * (N / W) + i * 32 + r) * 128 + ((p * 4 + ks * 2 + (lane >> 5)) ^ swz(r)) * 16);
      }
    }
  }
};

// the largest of 16 lanes', in each of them
__device__ __forceinline__ int most16(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, true));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, true));
  return max(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, true));
}

// G's entries in a block lie below 2^(kTopG + kCoarse), 2^15
static_assert(kTopG + 1 + kSlack <= 15 && kTopG - 1 + kCoarse <= 15, "fp16");
__device__ __forceinline__ int coarse_of(int e) { return e & ~(kCoarse - 1); }

// eight fp16 numbers times 2^d, d <= 15 (0 below 2^-24)
__device__ __forceinline__ u32x4 times_power(u32x4 v, int d) {
  const _Float16 f = __builtin_amdgcn_ldexph((_Float16)1.0f, d);
  return __builtin_bit_cast(u32x4, __builtin_bit_cast(f16x8, v) * f16x8{f, f, f, f, f, f, f, f});
}

template <typename C, Mode M>
struct Core {
  f32x16 acc[C::TM][C::TN];
  int top[C::TM];  // kRows: the exponent of row 32 i + lane % 32 in the sums so far; kBlocks: top[0] that of all rows
  int wm, wn, fr, fk;

  __device__ __forceinline__ Core() {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave % C::WM;
    wn = wave / C::WM;
    fr = threadIdx.x & 31;
    fk = (threadIdx.x & 63) >> 5;
  }
  // the tile's row of accumulator entry (i, e) of this lane, and its column of (j)
  __device__ __forceinline__ int row(int i, int e) const { return wm * (C::BM / C::WM) + i * 32 + (e >> 2) * 8 + fk * 4 + (e & 3); }
  __device__ __forceinline__ int col(int j) const { return wn * (C::BN / C::WN) + j * 32 + fr; }
  // what lane `row % 32` of the 32 x 32 accumulators holds, for entry e's row
  template <typename T>
  __device__ __forceinline__ T of_row(T v, int e) const {
    return __shfl(v, (e >> 2) * 8 + fk * 4 + (e & 3), 64);
  }

  // The sums of block i come down to the power of t.
  __device__ __forceinline__ void come_down(int i, int t) {
    const float down = ldexpf(1.0f, max(top[i] - t, -300));
    top[i] = t;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float g = of_row(down, q);
#pragma unroll
      for (int j = 0; j < C::TN; ++j) acc[i][j][q] *= g;
    }
  }

  // The sums as they are, without the powers that their operands had.
  __device__ __forceinline__ void level() {
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int power = of_row(top[i], q) - kTopG - kTop;
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j][q] = ldexpf(acc[i][j][q], power);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The products of a stage.  TIMES: a's blocks times 2^(d[ks][i]), in one or two factors (below 2^-38 nothing is left of them).
  template <int TIMES, int KSTEPS, int P, typename A, typename B>
  __device__ __forceinline__ void stage(const char *at, const char *bt, const A &sa, const B &sb, const int (&d)[KSTEPS][C::TM]) {
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      u32x4 fa[P][C::TM], fb[P][C::TN];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        sa.read(at, wm, ks, p, fa[p]);
        sb.read(bt, wn, ks, p, fb[p]);
      }
      if (TIMES > 0) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
          const int first = max(d[ks][i], -14);
#pragma unroll
          for (int p = 0; p < P; ++p) {
            fa[p][i] = times_power(fa[p][i], first);
            if (TIMES > 1) fa[p][i] = times_power(fa[p][i], max(d[ks][i] - first, -25));
          }
        }
      }
      if (P == 2) {
        multiply(fa[0], fb[P - 1]);
        multiply(fa[P - 1], fb[0]);
      }
      multiply(fa[0], fb[0]);
      if (TIMES > 0 && ks + 1 < KSTEPS) __builtin_amdgcn_sched_barrier(0);
    }
  }

  __device__ __forceinline__ void multiply_row(int i, const u32x4 &fa, const u32x4 *fb) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      if (M == kSplit)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, fa), __builtin_bit_cast(f16x8, fb[j]),
                                                           acc[i][j], 0, 0, 0);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa), __builtin_bit_cast(bf16x8, fb[j]),
                                                            acc[i][j], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void multiply(const u32x4 *fa, const u32x4 *fb) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i) multiply_row(i, fa[i], fb);
  }

  // acc = sum over `depth` of K from a and b on, a multiple of 64 (of 16 with KA); b has depth_b rows where they are K,
  // some in every stage.
  // kSplit: both numbers of both operands are in a stage, each is read once for hi lo, lo hi and hi hi (one stage for each
  // of the three: gradients of 8 x 257 x 50257 x 768, each example's, 1774 us with the log-probabilities, 1659 us so).
  // kPair: all of K with a's lo, then with its hi.
  // kRows: each row begins at the largest of its first 256 columns (one trip to the caches), so that few groups bring the sums
  // down; what a stage's blocks are times is settled a stage before, since the products would wait for it.
  // REST: the rows of a marked stage once more with the rest (4096 x 50257 x 768 bf16 855 us without it, 879 us so; as stages of
  // their own at the end 911 us; 8192 x 128256 x 4096 19.2 and 19.8 ms).
  template <bool KA, bool KB, Scaling S = kPlain, bool REST = false>
  __device__ __forceinline__ void run(char *lds, const Operand &a, const Operand &b, int rows_a, int rows_b, int depth,
                                      int depth_b, Powers pw = Powers{}, Rest r = Rest{}) {
    constexpr int P = M == kSplit ? 2 : 1, HALF = C::BM * kStep * 2, STAGE = HALF + C::BN * kStep * 2;
    using A = Side<C::BM, C::WM, C::TH, KA, P>;
    using B = Side<C::BN, C::WN, C::TH, KB, P>;
    A sa;
    B sb;
    const int steps = (depth + A::KS - 1) / A::KS;
    sa.init(a, rows_a, depth);
    sb.init(b, rows_b, depth_b);
    int part = 0, k = 0;  // of the next stage to load
    auto load = [&](int st, bool none = false) {
      sa.load(lds + st * STAGE, a.p[M == kPair && part == 0], k, none);
      sb.load(lds + st * STAGE + HALF, b.p[0], k);
      if (++k == steps) {
        k = 0;
        ++part;
      }
    };
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int all = steps * (M == kPair ? 2 : 1);
    // REST: target and number of row `lane` of the next stage, where that is marked
    int next_target = -1, chunk = r.k0 >> 5;
    float next_rest = 0.0f;
    uint64_t marks = 0;  // of 64 blocks of 32 rows from `chunk` on
    auto read_marks = [&]() {
      constexpr int V = C::BM / C::WM / 64;
      const int b = chunk + (threadIdx.x & 63), last = (r.k0 + depth - 1) >> 5;
      int m = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) m |= r.marks[(wm * V + v) * r.ld + min(b, last)];
      marks = __ballot(b <= last && m);
    };
    auto read_rest = [&](int s) {
      if (((r.k0 + s * kStep) >> 5) - chunk > 61) {
        chunk = (r.k0 + s * kStep) >> 5;
        read_marks();
      }
      next_target = -1;
      if (!(marks >> (((r.k0 + s * kStep) >> 5) - chunk) & (r.k0 & 31 ? 7 : 3))) return;
      const int k = s * kStep + (threadIdx.x & 63), at = min(k, depth - 1);
      if (k < depth) next_target = r.tgt[at] - r.first - wm * (C::BM / C::WM);
      next_rest = r.rest[at];
    };
    if (all > 0) load(0);
    if (REST && all > 0) {
      read_marks();
      read_rest(0);
    }
    constexpr int G = A::KS / 16;  // groups of a stage
    const int groups = depth / 16;
    int next[G][C::TM], d[G][C::TM];  // kRows: powers of the stage behind the next one; what this stage's blocks are times
    auto powers = [&](int k) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
          next[g][i] = pw.p[min(k * G + g, groups - 1) * pw.ld + wm * (C::BM / C::WM) + i * 32 + fr];
    };
    // kBlocks: the powers of the stage whose loads are under way and of the one behind it, the largest so far.  The sums go from
    // block to block's power, up to 2^60 above what they are under the largest; blocks below that count as zeros.
    int block = 0, behind = 0, most = 0;
    if (S == kRows) {
#pragma unroll
      for (int i = 0; i < C::TM; ++i) {
        top[i] = kNone;
        for (int g = 0; g < min(groups, 16); g += 4)
#pragma unroll
          for (int h = 0; h < 4; ++h)
            top[i] = max(top[i], pw.p[min(g + h, groups - 1) * pw.ld + wm * (C::BM / C::WM) + i * 32 + fr]);
      }
      if (groups) {
        powers(0);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int i = 0; i < C::TM; ++i) d[g][i] = next[g][i] - top[i];
        powers(1);
      }
    } else if (S == kBlocks) {
      top[0] = kNone;
      if (all > 0) block = most = top[0] = __builtin_amdgcn_readfirstlane(pw.p[0]);
      if (all > 1) behind = pw.p[A::KS / 64];
    }
    for (int s = 0; s < all; ++s) {
      // the loads of this stage, and the reads of the buffer that the next one gets
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      int to[C::TM], then[G][C::TM];
      bool up = false;
      if (S == kRows) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            then[g][i] = next[g][i];
            asm volatile("" : "+v"(then[g][i]));  // they have arrived: not waited for behind the loads that follow
          }
          to[i] = then[0][i];
#pragma unroll
          for (int g = 1; g < G; ++g) to[i] = max(to[i], then[g][i]);
          up = up || to[i] > top[i] + kSlack;
          to[i] = to[i] > top[i] + kSlack ? to[i] : top[i];
        }
        up = __any(up);
        if (s + 2 < all) powers(s + 2);
      }
      int target = next_target;
      float left = next_rest;
      if (REST) {
        asm volatile("" : "+v"(target), "+v"(left));
        if (s + 1 < all) read_rest(s + 1);
      }
      const int e = block;
      if (S == kBlocks) {
        asm volatile("" : "+v"(behind));
        const int b = __builtin_amdgcn_readfirstlane(behind);
        most = max(most, b);
        block = max(b, most - 60);
        if (s + 2 < all) behind = pw.p[(s + 2) * A::KS / 64];
        if (s + 1 < all) load((s + 1) & 1, b < most - 60);
      } else if (s + 1 < all) {
        load((s + 1) & 1);
      }
      const char *at = lds + (s & 1) * STAGE, *bt = at + HALF;
      if constexpr (S == kRows) {
        stage<2, G, P>(at, bt, sa, sb, d);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int i = 0; i < C::TM; ++i) d[g][i] = then[g][i] - to[i];
        if (up)
#pragma unroll
          for (int i = 0; i < C::TM; ++i) come_down(i, to[i]);
      } else if constexpr (S == kBlocks) {
        if (e != top[0]) {
          const float f = ldexpf(1.0f, max(top[0] - e, -300));
          top[0] = e;
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
              for (int q = 0; q < 16; ++q) acc[i][j][q] *= f;
        }
        stage<0, G, P>(at, bt, sa, sb, d);
      } else {
        stage<0, G, P>(at, bt, sa, sb, d);
      }
      if constexpr (REST) {
        // few stages have a row whose target is among the wave's: their 16 rows once more, a made in registers
        const uint32_t place = (unsigned)target < (unsigned)(C::BM / C::WM) ? target : 0xFFFF;
        const uint32_t word = place << 16 | bf16_bits(left);
        uint64_t hit[C::TM], any = 0;
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
          hit[i] = __ballot(place >> 5 == i);
          any |= hit[i];
        }
        if (any) {
#pragma unroll 1
          for (int ks = 0; ks < kStep / 16; ++ks) {
            if (!(any >> (ks * 16) & 0xFFFF)) continue;
            u32x4 fa[C::TM], fb[C::TN];
            uint32_t w[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) w[q] = __shfl(word, ks * 16 + fk * 8 + q, 64);
            sb.read(bt, wn, ks, 0, fb);
#pragma unroll
            for (int i = 0; i < C::TM; ++i) {
              if (!(hit[i] >> (ks * 16) & 0xFFFF)) continue;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t lo = w[2 * q] >> 16 == i * 32 + fr ? w[2 * q] & 0xFFFF : 0;
                const uint32_t hi = w[2 * q + 1] >> 16 == i * 32 + fr ? w[2 * q + 1] << 16 : 0;
                fa[i][q] = lo | hi;
              }
              multiply_row(i, fa[i], fb);
            }
          }
        }
      }
    }
  }
};
#endif

// from a row, and a column that is a multiple of 32, on
template <Mode M>
__device__ __forceinline__ Operand at_row(Operand a, int64_t row, int64_t k = 0) {
  a.p[0] += row * a.ld + (M == kSplit ? 2 * k : k);
  a.p[1] += row * a.ld + (M == kSplit ? 2 * k : k);
  return a;
}

// the place of number p of G's entry (n, v)
template <Mode M>
__device__ __forceinline__ int64_t g_at(int64_t plane, int64_t piece, int64_t n, int64_t v, int p) {
  return M == kSplit ? n * piece * 2 + split_at(v, p) : p * plane + n * piece + v;
}

#if defined(__HIP_DEVICE_COMPILE__)
// Tile number b of mt x nt: workgroups go to the eight XCDs in turn, and each XCD takes a run of tiles, in groups of
// eight of m, so that its L2 holds the rows that its CUs share.
__device__ __forceinline__ void tile_of(int b, int mt, int nt, int &tm, int &tn) {
  const int total = mt * nt, q = total / 8, r = total % 8, x = b & 7;
  b = x * q + (x < r ? x : r) + (b >> 3);
  const int per = 8 * nt, g = b / per, gm = min(8, mt - g * 8);
  tm = g * 8 + (b - g * per) % gm;
  tn = (b - g * per) / gm;
}
#endif

struct Logit {
  Operand w, h;
  int v0, valid, kp;  // the piece: its first row of the vocabulary and how many there are
  const Meta *meta;
  const int *tgt, *eh, *ev;
  float scale;
  // forward
  float2 *part;  // [piece / 64][tcap]
  float *xt;
  int64_t tcap;
  // gradient
  const RowPrm *prm;
  uint16_t *g;  // [tcap][piece] entries
  float *rest;     // [tcap], bf16: what the rounding of the target's entry has left
  uint8_t *marks;  // [piece / 64][tcap / 32], bf16: whether a row of the 32 has its target among the 64 entries
  int64_t gplane, piece;
  // fp32: G for dH without the rows' factors cs (g; NULL if not wanted) and for dW (gw), under the powers ph and pw
  uint16_t *gw;
  int *ph, *pw;  // [piece / 64], [tcap / 16][piece]
  const float *cs;
};

template <typename C, Mode M, bool GRAD>
__global__ __launch_bounds__(C::TH, 2) void k_logits(Logit a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool F16 = M == kSplit;
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int np = a.meta->np, mt = (a.valid + C::BM - 1) / C::BM, nt = (np + C::BN - 1) / C::BN;
  if ((int)blockIdx.x >= mt * nt) return;
  int tm, tn;
  tile_of(blockIdx.x, mt, nt, tm, tn);
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  Core<C, F16 ? kSplit : kBf16> c;  // H and W have one number or two
  c.template run<false, false>(lds, at_row<M>(a.w, m0), at_row<M>(a.h, n0), a.valid - m0, np - n0, a.kp, 0);
  const bool whole = m0 + C::BM <= a.valid;
  int ev[C::TM][16];
  if (F16) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const i32x4 v = *(const i32x4 *)(a.ev + m0 + c.row(i, e));
#pragma unroll
        for (int q = 0; q < 4; ++q) ev[i][e + q] = v[q];
      }
  }
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = n0 + c.col(j);
    const bool in = n < np;
    const int ex = F16 && in ? a.eh[n] - 2 * kTop : 0;
    if (GRAD) {
      const RowPrm p = in ? a.prm[n] : RowPrm{INFINITY, 0.0f, 0.0f};
      const int tv = in ? a.tgt[n] - a.v0 - m0 - c.wm * (C::BM / C::WM) : -1;
      const Power pw = power_of(a.scale);
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = c.acc[i][j][e];
          if (F16) x = ldexpf(x, ev[i][e] + ex);
          c.acc[i][j][e] = p.w * (F16 ? entry_exp<float>(x - p.m, pw) : entry_exp<bf16>(x - p.m, pw));
        }
      const bool any = __any(tv >= 0 && tv < C::BM / C::WM);
      if (M == kBf16 && (threadIdx.x & 63) == 0 && in) {
        static_assert(C::BM / C::WM == 64, "a row of marks");
        a.marks[((m0 >> 6) + c.wm) * (a.tcap >> 5) + (n >> 5)] = any;
      }
      if (any) {  // few tiles have one of their rows' targets
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (c.row(i, e) - c.wm * (C::BM / C::WM) == tv) {
              const float g = c.acc[i][j][e] + p.one;
              c.acc[i][j][e] = g;
              if (M == kBf16) a.rest[n] = g - to_f32(bf16{(uint16_t)bf16_bits(g)});
            }
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (m0 + c.row(i, e) >= a.valid) c.acc[i][j][e] = 0.0f;
      }
      // the one or two numbers of an entry, as bits
      if (!F16)
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) c.acc[i][j][e] = __uint_as_float(split<M>(c.acc[i][j][e]));
    } else {
      const float k2 = power_of(a.scale).k;
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = c.acc[i][j][e];
          if (F16) x = ldexpf(x, ev[i][e] + ex);
          if (!whole && m0 + c.row(i, e) >= a.valid) x = -INFINITY;
          c.acc[i][j][e] = x;
          m = fmaxf(m, x);
        }
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const float base = m == -INFINITY ? 0.0f : m;
      float z = 0.0f;
#pragma unroll
      for (int i = 0; i < C::TM; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f((c.acc[i][j][e] - base) * k2);
        z += s;
      }
      z += __shfl_xor(z, 32, 64);
      if (in) {
        const int64_t unit = m0 / (C::BM / C::WM) + c.wm;
        if (c.fk == 0) a.part[unit * a.tcap + n] = float2{m, z};
        const int tv = a.tgt[n] - a.v0 - m0 - c.wm * (C::BM / C::WM);
        if (tv >= 0 && tv < C::BM / C::WM) {
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (c.row(i, e) - c.wm * (C::BM / C::WM) == tv) a.xt[n] = c.acc[i][j][e];
        }
      }
    }
  }
  if (!GRAD) return;
  // G's rows leave through LDS, in whole lines (chunks of 16 bytes exchanged by the row, so that the lanes of a write meet
  // different banks).
  if constexpr (F16) {  // hi and lo of 32 columns of the waves' accumulators at a time, in two places by turns
    constexpr int RW = C::BM * 4, CH = RW / 16, ROWS = 32 * C::WN;
    static_assert(ROWS * RW <= C::LDS, "a turn fits");
    constexpr int PLACES = 2 * ROWS * RW <= C::LDS ? 2 : 1;
    int turn = 0;
    auto leave = [&](int j, const uint32_t (&bits)[C::TM][16], uint16_t *to) {
      char *at = lds + (turn % PLACES) * ROWS * RW;
      if (PLACES == 1 || turn == 0) __syncthreads();
      ++turn;
      const int n = c.wn * 32 + c.fr;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int m = c.row(i, e), ch = (m >> 5) * 8 + p * 4 + ((m & 31) >> 3);
            const uint32_t sel = p ? 0x07060302 : 0x05040100;
            const u32x2 v{__builtin_amdgcn_perm(bits[i][e + 1], bits[i][e], sel),
                          __builtin_amdgcn_perm(bits[i][e + 3], bits[i][e + 2], sel)};
            *(u32x2 *)(at + n * RW + (ch ^ (n & 31)) * 16 + (m & 4) * 2) = v;
          }
      __syncthreads();
#pragma unroll 4
      for (int k = threadIdx.x; k < ROWS * CH; k += C::TH) {
        const int r = k / CH, ch = k % CH, row = n0 + (r >> 5) * (C::BN / C::WN) + j * 32 + (r & 31);
        if (row < np)
          *(u32x4 *)(to + (int64_t)row * a.piece * 2 + m0 * 2 + ch * 8) = *(const u32x4 *)(at + r * RW + (ch ^ (r & 31)) * 16);
      }
    };
    int coarse = kNone;  // the wave's 64 entries of the vocabulary
    if (a.g) {
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) coarse = max(coarse, ev[i][e]);
      static_assert(C::BM / C::WM == 64, "a block of kBlocks");
      coarse = coarse_of(max(coarse, __shfl_xor(coarse, 32, 64)));
      if (tn == 0) a.ph[(m0 >> 6) + c.wm] = coarse;
    }
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      uint32_t bits[C::TM][16];
      if (a.g) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) bits[i][e] = split<M>(ldexpf(c.acc[i][j][e], ev[i][e] + kTopG - coarse));
        leave(j, bits, a.g);
      }
      if (a.gw) {
        const int n = n0 + c.col(j), eh = n < np ? a.eh[n] : 0;
        const float f = n < np ? a.cs[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
          int mine = kNone;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = c.acc[i][j][e] * f;
            const int most = most16(exponent_of(y) + eh);
            bits[i][e] = split<M>(ldexpf(y, eh + kTopG - most));
            if ((c.fr & 15) == e) mine = most;
          }
          if (n < np) a.pw[(int64_t)(n >> 4) * a.piece + m0 + c.row(i, c.fr & 15)] = mine;
        }
        leave(j, bits, a.gw);
      }
    }
    return;
  }
#pragma unroll
  for (int plane = 0; plane < (M == kBf16 ? 1 : 2); ++plane) {
    constexpr int CH = C::BM / 8;
    auto pair = [&](int i, int j, int e) {
      return __builtin_amdgcn_perm(__float_as_uint(c.acc[i][j][e + 1]), __float_as_uint(c.acc[i][j][e]),
                                   plane ? 0x07060302 : 0x05040100);
    };
    __syncthreads();
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      const int n = c.col(j);
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int m = c.row(i, e);
          const u32x2 v{pair(i, j, e), pair(i, j, e + 2)};
          *(u32x2 *)(lds + n * (C::BM * 2) + ((m >> 3) ^ (n & (CH - 1))) * 16 + (m & 4) * 2) = v;
        }
    }
    __syncthreads();
#pragma unroll 4
    for (int k = threadIdx.x; k < C::BN * CH; k += C::TH) {
      const int n = k / CH, m = k % CH;
      if (n0 + n < np)
        *(u32x4 *)(a.g + g_at<M>(a.gplane, a.piece, n0 + n, m0 + m * 8, plane)) =
            *(const u32x4 *)(lds + n * (C::BM * 2) + (m ^ (n & (CH - 1))) * 16);
    }
  }
#endif
}

// --- few rows -----------------------------------------------------------------------------------------------
constexpr int kFew = 16;        // rows up to which W goes straight from memory into the matrix cores, once
constexpr int kFewUnit = 64;    // vocabulary rows of a workgroup

__device__ __forceinline__ int target_of(const void *targets, int index, int64_t t, int vocab) {
  const int64_t v = index == SK_I64 ? ((const int64_t *)targets)[t] : ((const int32_t *)targets)[t];
  return v >= 0 && v < vocab ? (int)v : -1;
}

struct Few {
  const void *hidden, *weight, *targets;
  int64_t ld_hidden, ld_weight;
  int rows, vocab, width, index;
  float scale;
  float2 *part;  // [kFew][units]
  float *xt;     // [kFew]
  int units;
  float *logp;
  float2 *stats;
  // gradient: G of a piece
  int v0, valid;
  const Meta *meta;
  const int *pos, *list;
  const RowPrm *prm;
  uint16_t *g;
  int64_t gplane, piece;
  uint16_t *gw;  // fp32, as in Logit
  int *ph, *pw;
  const int *eh, *ev;
  const float *cs;
};

// Logits of up to 16 rows by 16 entries of the vocabulary a wave.  Lane l holds row l % 16 of both operands; its eight
// (fp32: four) columns from 8 (l / 16) on are one operand of v_mfma_f32_16x16x32_bf16 (element i of each lane one of
// v_mfma_f32_16x16x4_f32, in which fp32 stays fp32).  Bound by reading W: 50257 x 768 bf16
// 19 us, 4.1 TB/s.  GRAD: G from the same logits to the bit, so that a small 1 - p of the target keeps what it has (logits of
// the split product beside these statistics were off by 5e-6 of it where p = 0.9).  A logit is eight sums (bf16: four), since
// one of 4096 products in a row rounds to 8e-6 at random (log p of 16 x 20000 x 4096 fp32, relative: 1.3e-6 with one, 4.4e-7
// with four, 1.7e-7 with eight; sixteen take 60 us instead of 47 for 1 x 50257 x 768).
template <typename T, bool GRAD>
__global__ __launch_bounds__(256) void k_few(Few a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int N = Vec<T>::N, K = 4 * N, U = 4;  // columns of a lane, of a step, steps whose loads are under way together
  __shared__ float2 lds[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
  const int v0 = a.v0 + blockIdx.x * kFewUnit + wave * 16, v = v0 + r;
  const int n = GRAD && r < a.rows ? a.pos[r] : -1;
  const int target = r < a.rows && (!GRAD || n >= 0) ? target_of(a.targets, a.index, r, a.vocab) : -1;
  const T *w = (const T *)a.weight + (int64_t)(v < a.vocab ? v : a.vocab - 1) * a.ld_weight;
  const T *h = (const T *)a.hidden + (int64_t)(target >= 0 ? r : 0) * a.ld_hidden;
  const int hw = target >= 0 ? a.width : 0;  // masked rows are not read
  constexpr int S = sizeof(T) == 2 ? U : 8;  // sums, joined at the end
  f32x4 sum[S] = {};
  for (int k0 = q * N; k0 - q * N < a.width; k0 += K * U) {
    u32x4 fw[U], fh[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * K;
      auto part = [&](const T *row, int width) {
        if (k + N <= width) return Vec<T>::load(row + k);
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = k + i < width ? to_f32(row[k + i]) : 0.0f;
        return Vec<T>::pack(f);
      };
      fw[u] = part(w, a.width);
      fh[u] = part(h, hw);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (sizeof(T) == 2) {
        sum[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[u]), __builtin_bit_cast(bf16x8, fh[u]),
                                                         sum[u], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[(u * 4 + i) % S] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(fw[u][i]), __uint_as_float(fh[u][i]),
                                                                      sum[(u * 4 + i) % S], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int n = S / 2; n >= 1; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) sum[i] += sum[i + n];
  f32x4 acc = sum[0];
  // this lane: entries v0 + 4 q + e of row r
  if constexpr (GRAD) {
    constexpr Mode M = sizeof(T) == 4 ? kSplit : kPair;
    const int at = v0 - a.v0 + q * 4;
    float g[4] = {};
    auto leave = [&](uint16_t *to, const float *x) {
#pragma unroll
      for (int plane = 0; plane < 2; ++plane)
        *(u32x2 *)(to + g_at<M>(a.gplane, a.piece, n, at, plane)) = u32x2{two<M>(x[0], x[1], plane), two<M>(x[2], x[3], plane)};
    };
    if (n >= 0) {
      const RowPrm p = a.prm[n];
      const Power pw = power_of(a.scale);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[e] = p.w * entry_exp<T>(acc[e] - p.m, pw);
        if (v0 + q * 4 + e == target) g[e] += p.one;
        if (at + e >= a.valid) g[e] = 0.0f;
      }
    }
    if (M != kSplit && n >= 0) leave(a.g, g);
    if (M == kSplit && a.g) {
      int coarse = a.ev[blockIdx.x * kFewUnit + lane];
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) coarse = max(coarse, __shfl_xor(coarse, d, 64));
      coarse = coarse_of(coarse);
      if (threadIdx.x == 0) a.ph[blockIdx.x] = coarse;
      if (n >= 0) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ldexpf(g[e], a.ev[at + e] + kTopG - coarse);
        leave(a.g, x);
      }
    }
    const int np = a.meta->np;
    if (M == kSplit && a.gw) {  // up to 16 groups of rows, by the unit's entries of the vocabulary
      __shared__ int most[kFew][kFewUnit];
      for (int i = threadIdx.x; i < kFew * kFewUnit; i += 256) (&most[0][0])[i] = kNone;
      __syncthreads();
      const int eh = n >= 0 ? a.eh[n] : 0;
      const float f = n >= 0 ? a.cs[n] : 0.0f;
      int *mine = &most[n >= 0 ? n >> 4 : 0][wave * 16 + q * 4];
      if (n >= 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[e] *= f;
          atomicMax(mine + e, exponent_of(g[e]) + eh);
        }
      __syncthreads();
      if (n >= 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = ldexpf(g[e], eh + kTopG - mine[e]);
        leave(a.gw, g);
      }
      for (int i = threadIdx.x; i < np / 16 * kFewUnit; i += 256)
        a.pw[(int64_t)(i / kFewUnit) * a.piece + blockIdx.x * kFewUnit + i % kFewUnit] = most[i / kFewUnit][i % kFewUnit];
    }
    // rows that only fill the list
    for (int i = threadIdx.x >> 3; i < np; i += 32)
      if (a.list[i] < 0)
#pragma unroll
        for (int plane = 0; plane < 2; ++plane) {
          const int64_t to = g_at<M>(a.gplane, a.piece, i, blockIdx.x * kFewUnit + (threadIdx.x & 7) * 8, plane);
          if (a.g) *(u32x4 *)(a.g + to) = u32x4{0, 0, 0, 0};
          if (M == kSplit && a.gw) *(u32x4 *)(a.gw + to) = u32x4{0, 0, 0, 0};
        }
    return;
  }
  const float k2 = power_of(a.scale).k;
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int u = v0 + q * 4 + e;
    if (u >= a.vocab) acc[e] = -INFINITY;
    if (u == target) a.xt[r] = acc[e];
    m = fmaxf(m, acc[e]);
  }
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  if (q == 0) lds[wave][r].x = m;
  __syncthreads();
  m = fmaxf(fmaxf(lds[0][r].x, lds[1][r].x), fmaxf(lds[2][r].x, lds[3][r].x));
  const float base = m == -INFINITY ? 0.0f : m;
  float z = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) z += __builtin_amdgcn_exp2f((acc[e] - base) * k2);
  z += __shfl_xor(z, 16, 64);
  z += __shfl_xor(z, 32, 64);
  if (q == 0) lds[wave][r].y = z;
  __syncthreads();
  if (threadIdx.x < (unsigned)a.rows)
    a.part[threadIdx.x * (int64_t)a.units + blockIdx.x] = float2{m, lds[0][r].y + lds[1][r].y + lds[2][r].y + lds[3][r].y};
#endif
}

// A workgroup a row: its (m, z) and log-probability from the units'.
__global__ __launch_bounds__(512) void k_few_join(Few a) {
  __shared__ float big[8];
  __shared__ double sum[8];
  const int t = blockIdx.x, target = target_of(a.targets, a.index, t, a.vocab);
  Stats s{0.0f, 0.0f};
  float lp = 0.0f;
  if (target >= 0) {  // the same for all threads
    const float2 *part = a.part + (int64_t)t * a.units;
    const float k2 = power_of(a.scale).k;
    float m = -INFINITY;
    for (int u = threadIdx.x; u < a.units; u += 512) m = fmaxf(m, part[u].x);
    m = block_all<8>(m, OpMax(), big);
    if (m == -INFINITY) m = 0.0f;
    double z = 0.0;
    for (int u = threadIdx.x; u < a.units; u += 512) {
      const float2 p = part[u];
      if (p.y != 0.0f) z += (double)(p.y * __builtin_amdgcn_exp2f((p.x - m) * k2));
    }
    s = Stats{m, (float)block_all<8>(z, OpAdd(), sum)};
    lp = logp_of(a.xt[t], s, a.scale);
  }
  if (threadIdx.x == 0) {
    a.logp[t] = lp;
    if (a.stats) a.stats[t] = float2{s.m, s.z};
  }
}

// (m, z) of the listed rows from those of a piece's units and of the pieces before, at the end their log-probabilities; 16
// rows a workgroup, whose lanes share the units (64 rows a workgroup: 4096 x 50257 23 us, 8 us so).
struct Join {
  const Meta *meta;
  const int *list;
  const float2 *part;
  const float *xt;
  int64_t tcap;
  int units;
  float scale;
  bool first, last;
  float2 *run;  // [tcap]
  float *logp;
  float2 *stats;
};
__global__ __launch_bounds__(1024) void k_join(Join a) {
  __shared__ float2 lds[16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 16 + (lane & 15);
  if ((int)blockIdx.x * 16 >= a.meta->np) return;  // np is a multiple of 16
  const float k2 = power_of(a.scale).k;
  auto join = [&](float2 p, float2 q) {
    const float m = fmaxf(p.x, q.x), base = m == -INFINITY ? 0.0f : m;
    // a sum of nothing is left out: its exponent may be a NaN
    return float2{m, (p.y == 0.0f ? 0.0f : p.y * __builtin_amdgcn_exp2f((p.x - base) * k2)) +
                         (q.y == 0.0f ? 0.0f : q.y * __builtin_amdgcn_exp2f((q.x - base) * k2))};
  };
  float2 s{-INFINITY, 0.0f};
  constexpr int U = 4;
  for (int u = wave * 4 + (lane >> 4); u < a.units; u += 64 * U) {
    float2 p[U];
#pragma unroll
    for (int i = 0; i < U; ++i) p[i] = u + i * 64 < a.units ? a.part[(u + i * 64) * a.tcap + n] : float2{-INFINITY, 0.0f};
#pragma unroll
    for (int i = 0; i < U; ++i) s = join(s, p[i]);
  }
#pragma unroll
  for (int d = 16; d < 64; d <<= 1) s = join(s, float2{__shfl_xor(s.x, d, 64), __shfl_xor(s.y, d, 64)});
  if (lane < 16) lds[wave][lane] = s;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  s = lds[0][lane];
  for (int w = 1; w < 16; ++w) s = join(s, lds[w][lane]);
  if (!a.first) s = join(a.run[n], s);
  if (!a.last) {
    a.run[n] = s;
    return;
  }
  const int t = a.list[n];
  if (t < 0) return;
  if (s.x == -INFINITY) s.x = 0.0f;
  a.logp[t] = logp_of(a.xt[n], Stats{s.x, s.y}, a.scale);
  if (a.stats) a.stats[t] = s;
}

// What a piece adds to dH, and its rows of dW.
struct Back {
  int width;
  const Meta *meta;
  const int *seg;
  int64_t tcap;
  // dH: acc[split] (+)= G W
  Operand g, w;
  int steps, per, splits;  // stages of the piece, of a split
  int blocks;              // workgroups at most, a multiple of 8 (0: not wanted)
  bool first;
  float *acc;     // [splits][tcap][kp]
  int kp;
  const int *ph;  // fp32
  // dW = G^T H (fp32: of its own G)
  Operand gw, h;
  Powers pw;
  const int *tgt;     // bf16, one number, as in Rest
  const float *rest;
  const uint8_t *marks;
  int v0, valid, b0;  // the piece's first row and how many, the launch's first example
  void *out;      // rows from the piece's first on
  int64_t vocab;  // rows from example to example
  bool accumulate;
  bool past;  // dW is stored past the caches, which hold G and W (each example's of 8 x 257 x 50257 x 768 fp32: 1300, 1171 us)
};

// Both products of a piece in one launch: neither fills a whole number of rounds of the chip, and the longer ones (dH, K
// is the piece) come first.  Accumulator rows are tokens (vocabulary entries), columns features, so that a store is 32
// features of a row.
template <typename C, Mode M, typename TO>
__global__ __launch_bounds__(C::TH, 2) void k_back(Back a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool F16 = M == kSplit;
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const bool hidden = (int)blockIdx.x < a.blocks;
  const int np = a.meta->np, rows = hidden ? np : a.valid, mt = (rows + C::BM - 1) / C::BM, nt = (a.width + C::BN - 1) / C::BN;
  const int tiles = mt * nt, b = hidden ? blockIdx.x : blockIdx.x - a.blocks;
  if (hidden && b >= tiles * a.splits) return;
  const int part = b / tiles;  // split, or example
  int tm, tn;
  tile_of(b - part * tiles, mt, nt, tm, tn);
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  const int k0 = hidden ? part * a.per * kStep : a.seg[a.b0 + part];
  const int depth = hidden ? max(0, min(a.per, a.steps - part * a.per)) * kStep : a.seg[a.b0 + part + 1] - k0;
  Core<C, M> c;
  // split weights bring rows of zeros up to a multiple of 64
  if (hidden) {
    c.template run<false, true, F16 ? kBlocks : kPlain>(lds, at_row<M>(a.g, m0, k0), at_row<M>(a.w, k0, n0), np - m0,
                                                        a.kp - n0, depth, F16 ? a.steps * kStep - k0 : a.valid - k0,
                                                        Powers{a.ph + k0 / 64, 0});
  } else {
    const Powers pw{a.pw.p + k0 / 16 * a.pw.ld + m0, a.pw.ld};
    const int64_t blocks = a.tcap >> 5;
    const Rest rest{a.tgt + k0, a.rest + k0, a.marks + (m0 >> 6) * blocks, blocks, a.v0 + m0, k0};
    c.template run<true, true, F16 ? kRows : kPlain, M == kBf16>(lds, at_row<M>(a.gw, k0, m0), at_row<M>(a.h, k0, n0), C::BM,
                                                                 a.kp - n0, depth, depth, pw, rest);
  }
  if (hidden) {
    float *to = a.acc + (part * a.tcap + m0) * a.kp + n0;
    const int power = c.top[0] - kTopG - kTop;  // kBlocks: the same for all rows
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      if (n0 + c.col(j) >= a.kp) continue;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int m = c.row(i, e);
          if (m0 + m >= np) continue;
          float *p = to + (int64_t)m * a.kp + c.col(j);
          const float v = F16 ? ldexpf(c.acc[i][j][e], power) : c.acc[i][j][e];
          *p = a.first ? v : *p + v;
        }
    }
  } else {
    if constexpr (F16) c.level();
    TO *to = (TO *)a.out + ((a.b0 + part) * a.vocab + m0) * a.width + n0;
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      if (n0 + c.col(j) >= a.width) continue;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int m = c.row(i, e);
          if (m0 + m >= a.valid) continue;
          TO *p = to + (int64_t)m * a.width + c.col(j);
          const float v = c.acc[i][j][e];
          const TO r = from_f32<TO>(a.accumulate ? v + to_f32(*p) : v);
          if (a.past) {
            asm volatile("");  // or the compiler makes one ordinary store of the two
            if constexpr (sizeof(TO) == 4)
              __builtin_nontemporal_store(r, p);
            else
              __builtin_nontemporal_store(r.u, &p->u);
            asm volatile("");
          } else {
            *p = r;
          }
        }
    }
  }
#endif
}

// dH: the splits' sums in order; zeros for masked rows.  fp32: times the row's factor.  bf16: with what the rounding of the
// target's entry of G has left, since that entry is most of a row (errors of dH against 64 bits, of which 0.0017 are its
// own rounding: 0.0022 to 0.0026 without it, 0.0017 to 0.0019 with it).
struct DHidden {
  const int *pos, *tgt;
  const float *cs, *rest;
  const float *acc;
  int64_t tcap;
  int kp, splits, rows, width;
  const void *w;
  int64_t ldw;
  void *out;
  int64_t ld;
};
template <typename T>
__global__ __launch_bounds__(256) void k_dhidden_out(DHidden a) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= a.rows) return;
  const int p = a.pos[t];
  T *o = (T *)a.out + t * a.ld;
  const float f = p >= 0 ? (sizeof(T) == 4 ? a.cs[p] : a.rest ? a.rest[p] : 0.0f) : 0.0f;
  const T *w = (const T *)a.w + (sizeof(T) == 2 && p >= 0 ? a.tgt[p] : 0) * a.ldw;
  for (int k = lane * 8; k < a.width; k += 512) {
    float v[8] = {};
    if (p >= 0) {
      const float *x = a.acc + (int64_t)p * a.kp + k;
#pragma unroll 4
      for (int s = 0; s < a.splits; ++s, x += a.tcap * a.kp) {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const f32x4 y = *(const f32x4 *)(x + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[i + q] += y[q];
        }
      }
      float r[8];
      if (sizeof(T) == 2 && a.rest) row_part<8>(w, k, a.width, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = sizeof(T) == 4 ? v[i] * f : a.rest ? v[i] + f * r[i] : v[i];
    }
    if (k + 8 <= a.width) {
#pragma unroll
      for (int i = 0; i < 8; i += Vec<T>::N) Vec<T>::store(o + k + i, Vec<T>::pack(v + i));
    } else {
      for (int i = 0; k + i < a.width; ++i) o[k + i] = from_f32<T>(v[i]);
    }
  }
}

// --- host ---------------------------------------------------------------------------------------------------
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// How a call is cut, and where its parts lie in the workspace.
struct Plan {
  bool f16, grad, few, pair, copy, large, huge, front;
  int64_t batch, n, chunks, tcap, kp, piece, pieces, units, splits, planes, gplanes;  // numbers of an operand's entry, of G's
  int64_t list, pos, tgt, seg, cnt, meta, hc, eh, ev, part, xt, run, prm, cs, rest, marks, wc, g, gw, ph, pw, acc, bytes;
};

// single: dW in fp32
Plan plan_of(const sk_linear *x, int64_t batch, bool grad, bool dhidden, bool dweight, bool single) {
  Plan p{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t r = at;
    at += up(bytes, 256);
    return r;
  };
  p.f16 = x->dtype == SK_F32;
  p.grad = grad;
  p.units = (x->vocab + kFewUnit - 1) / kFewUnit;
  p.few = !grad && x->rows <= kFew;
  if (p.few) {
    p.part = take(8 * p.units * kFew);
    p.xt = take(4 * kFew);
    p.bytes = at;
    return p;
  }
  p.planes = p.f16 ? 2 : 1;
  p.batch = batch;
  p.n = x->rows / batch;
  p.pair = !p.f16 && (x->rows <= kPairRows || (single && p.n <= kPairRows));
  p.gplanes = p.f16 || p.pair ? 2 : 1;
  p.tcap = up(batch * up(p.n, kPad), 256);
  p.tcap = std::max<int64_t>(p.tcap, 256);
  p.chunks = batch * ((p.n + 63) / 64);
  p.front = p.chunks >= 1 && p.chunks <= kFrontChunks;
  p.kp = up(x->width, kStep);
  // rows that 16-byte loads in whole stages read as they lie
  p.copy = p.f16 || x->width % kStep || x->ld_weight % 8 || (uintptr_t)x->weight % 16 || x->ld_weight > (1 << 20);
  // a piece: G in 256 MB (a launch more for each halving), a copy of W in 256 MB.  fp32 has G twice where both gradients are
  // wanted: in 256 MB together up to a width of 1024 (4096 x 50257 x 768 2867 us, 2725 us so), in twice as much above, where
  // more pieces cost more sums of dH (4 examples of 512 x 32000 x 2048 2336 us, 2396 us; 8000 x 32000 x 5000 18.5 and 19.1 ms).
  int64_t most = x->vocab;
  const int64_t copies = p.f16 && dhidden && dweight && x->width <= 1024 ? 2 : 1;
  if (grad) most = std::min(most, ((int64_t)1 << 27) / (p.tcap * p.gplanes * copies));
  if (grad || p.copy) most = std::min(most, ((int64_t)1 << 27) / (p.kp * p.planes));
  // the tiles' (m, z) in 256 MB; grids below 2^32 threads
  if (!grad) most = std::min(most, ((int64_t)1 << 31) / p.tcap);
  most = std::min(most, ((int64_t)1 << 23) / (p.tcap / 128) * 128);
  if (most < x->vocab) most = std::max<int64_t>(most / 256 * 256, 256);
  p.pieces = (x->vocab + most - 1) / most;
  p.piece = up((x->vocab + p.pieces - 1) / p.pieces, 256);
  p.units = p.piece / 64;
  p.large = x->rows > kSmallRows;
  p.huge = p.n >= kHugeRows && (p.tcap / 256 + batch * (p.piece / 256)) * (up(x->width, 256) / 256) >= kHugeTiles;
  p.splits = 1;
  if (grad) {
    // dH has few tiles with all of the piece to sum up, dW many with the rows: a part of a dH tile takes half of what each
    // of the chip's 512 places has to do in all (4096 x 50257 x 768 bf16: 1271, 902, 819, 868, 979 us with 1, 2, 4, 8, 16
    // parts; 17 x 50257 x 768: 590, 203, 119, 123, 144 us with 1, 4, 16, 32, 64)
    const int64_t bn = p.large ? Large::BN : Small::BN, nt = up(x->width, bn) / bn, steps = p.piece / kStep;
    const int64_t all = up(p.tcap, 128) / 128 * nt * steps + batch * (p.piece / 128) * nt * (up(p.n, kStep) / kStep);
    p.splits = std::max<int64_t>(1, std::min<int64_t>({(768 * steps + all / 2) / all, 32, steps / 4}));
  }
  p.list = take(4 * p.tcap);
  p.pos = take(4 * x->rows);
  p.tgt = take(4 * p.tcap);
  p.seg = take(4 * (batch + 1));
  p.cnt = take(4 * p.chunks);
  p.meta = take(sizeof(Meta));
  p.hc = take(2 * p.planes * p.tcap * p.kp);
  p.eh = take(4 * p.tcap);
  if (p.f16) p.ev = take(4 * p.piece);
  if (p.copy) p.wc = take(2 * p.planes * p.piece * p.kp);
  if (!grad) {
    p.part = take(8 * p.units * p.tcap);
    p.xt = take(4 * p.tcap);
    p.run = take(8 * p.tcap);
  } else {
    p.prm = take(sizeof(RowPrm) * p.tcap);
    p.cs = take(4 * p.tcap);
    p.rest = take(4 * p.tcap);
    if (!p.f16 && !p.pair) p.marks = take(p.piece / 64 * (p.tcap / 32));
    if (dhidden || !p.f16) p.g = take(2 * p.gplanes * p.tcap * p.piece);
    if (dhidden && p.f16) p.ph = take(4 * (p.piece / 64));
    if (dweight && p.f16) {
      p.gw = take(2 * p.gplanes * p.tcap * p.piece);
      p.pw = take(4 * (p.tcap / 16) * p.piece);
    }
    if (dhidden) p.acc = take(4 * p.splits * p.tcap * p.kp);
  }
  p.bytes = at;
  return p;
}

int check_linear(const sk_linear *x) {
  if (!x) return train_fail(SK_EINVAL, "NULL argument");
  if (x->dtype != SK_F32 && x->dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (x->index != SK_I32 && x->index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (x->rows < 0 || x->vocab < 1 || x->width < 1 || x->ld_hidden < x->width || x->ld_weight < x->width)
    return train_fail(SK_EINVAL, "need rows >= 0, vocab >= 1, width >= 1 and row strides >= width");
  if (!(x->scale >= 0x1p-120f && x->scale <= 0x1p127f))
    return train_fail(SK_EINVAL, "scale must be in [2^-120, 2^127]");
  if (x->rows > (1 << 20) || x->vocab > (1 << 22) || x->width > (1 << 16))
    return train_fail(SK_EUNSUPPORTED, "more than 2^20 rows, 2^22 entries of the vocabulary or 2^16 features");
  if (!x->weight || (x->rows && (!x->hidden || !x->targets))) return train_fail(SK_EINVAL, "NULL argument");
  return SK_OK;
}
int check_batch(const sk_linear *x, int64_t batch) {
  if (batch < 1 || x->rows % batch) return train_fail(SK_EINVAL, "rows must be a multiple of batch >= 1");
  if (batch > (1 << 14)) return train_fail(SK_EUNSUPPORTED, "more than 2^14 examples");
  return SK_OK;
}

template <typename T>
T *ptr(void *work, int64_t at) {
  return (T *)((char *)work + at);
}


// W's rows from v0 on, as prep() takes them
Prep weights_of(const sk_linear *x, const Plan &p, int64_t v0, int64_t valid, void *work) {
  Prep a{};
  a.src = (const char *)x->weight + v0 * x->ld_weight * (p.f16 ? 4 : 2);
  a.ld = x->ld_weight;
  a.rows = (int)valid;
  a.width = (int)x->width;
  a.kp = (int)p.kp;
  if (p.f16) a.ev = ptr<int>(work, p.ev);
  a.out = ptr<uint16_t>(work, p.wc);
  return a;
}

// whether W's first piece is prepared by the launch that begins
bool in_front(const Plan &p) { return p.front && p.copy; }

// list, rows of H: what both directions begin with
void begin(const sk_linear *x, const Plan &p, const float *dlogp, const float *stats_in, float *logp, float *stats, void *work,
           hipStream_t st) {
  Meta *meta = ptr<Meta>(work, p.meta);
  int *list = ptr<int>(work, p.list);
  const Live l{x->targets, dlogp, (int32_t)x->index, (int32_t)x->vocab, (int32_t)p.n, (int32_t)p.batch, list,
               ptr<int>(work, p.pos), ptr<int>(work, p.tgt), ptr<int>(work, p.seg), ptr<int>(work, p.cnt), meta, logp,
               (float2 *)stats};
  const Gather g{x->hidden, x->ld_hidden, (int)x->width, (int)p.kp, list, meta, ptr<uint16_t>(work, p.hc),
                 ptr<int>(work, p.eh), (const float2 *)stats_in, dlogp, x->scale,
                 p.grad ? ptr<RowPrm>(work, p.prm) : nullptr, ptr<float>(work, p.cs)};
  if (p.front) {
    const int64_t valid = std::min(p.piece, x->vocab);
    const Front f{l, g, weights_of(x, p, 0, valid, work), (int)p.chunks * 4};
    const dim3 grid((unsigned)(f.blocks + (in_front(p) ? up(valid, 64) / 16 : 0))), block(1024);
    if (p.f16)
      hipLaunchKernelGGL(k_front<float>, grid, block, 0, st, f);
    else
      hipLaunchKernelGGL(k_front<bf16>, grid, block, 0, st, f);
    return;
  }
  hipLaunchKernelGGL(k_live, dim3(1), dim3(1024), 0, st, l);
  if (p.f16)
    hipLaunchKernelGGL(k_gather<float>, dim3((unsigned)(p.tcap / 4)), dim3(256), 0, st, g);
  else
    hipLaunchKernelGGL(k_gather<bf16>, dim3((unsigned)(p.tcap / 4)), dim3(256), 0, st, g);
}

// W's rows from v0 on as an operand
Operand weights(const sk_linear *x, const Plan &p, int64_t v0, int64_t valid, void *work, hipStream_t st) {
  Prep a = weights_of(x, p, v0, valid, work);
  if (!p.copy) return Operand{{(const uint16_t *)a.src, (const uint16_t *)a.src}, x->ld_weight};
  const Operand o{{a.out, a.out}, p.kp * p.planes};
  if (v0 == 0 && in_front(p)) return o;
  const dim3 grid((unsigned)(up(valid, 64) / 4));
  if (p.f16)
    hipLaunchKernelGGL(k_prep<float>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_prep<bf16>, grid, dim3(256), 0, st, a);
  return o;
}

Logit logit_of(const sk_linear *x, const Plan &p, int64_t v0, int64_t valid, Operand w, void *work) {
  Logit a{};
  a.w = w;
  const uint16_t *h = ptr<uint16_t>(work, p.hc);
  a.h = Operand{{h, h}, p.kp * p.planes};
  a.v0 = (int)v0;
  a.valid = (int)valid;
  a.kp = (int)p.kp;
  a.meta = ptr<Meta>(work, p.meta);
  a.tgt = ptr<int>(work, p.tgt);
  a.eh = ptr<int>(work, p.eh);
  a.ev = ptr<int>(work, p.ev);
  a.scale = x->scale;
  a.tcap = p.tcap;
  return a;
}

template <typename C, Mode M, bool GRAD>
void launch_logits(const Logit &a, int64_t rows, hipStream_t st) {
  const unsigned blocks = (unsigned)(((a.valid + C::BM - 1) / C::BM) * ((rows + C::BN - 1) / C::BN));
  hipLaunchKernelGGL((k_logits<C, M, GRAD>), dim3(blocks), dim3(C::TH), 0, st, a);
}
template <typename C, bool GRAD>
void run_logits_in(const Plan &p, const Logit &a, int64_t rows, hipStream_t st) {
  if (p.f16) return launch_logits<C, kSplit, GRAD>(a, rows, st);
  if constexpr (GRAD)
    if (p.pair) return launch_logits<C, kPair, GRAD>(a, rows, st);
  launch_logits<C, kBf16, GRAD>(a, rows, st);
}
template <bool GRAD>
void run_logits(const Plan &p, const Logit &a, hipStream_t st) {
  const int64_t rows = p.batch * up(p.n, kPad);
  if (p.large)
    run_logits_in<Large, GRAD>(p, a, rows, st);
  else if (rows <= Narrow::BN)
    run_logits_in<Narrow, GRAD>(p, a, rows, st);
  else
    run_logits_in<Small, GRAD>(p, a, rows, st);
}

template <typename C, Mode M, typename TO>
void launch_back(const Plan &p, Back a, bool dhidden, bool dweight, hipStream_t st) {
  const int64_t nt = (a.width + C::BN - 1) / C::BN, tiles = (a.valid + C::BM - 1) / C::BM * nt;
  a.blocks = dhidden ? (int)up((p.tcap + C::BM - 1) / C::BM * nt * a.splits, 8) : 0;
  const int64_t most = std::max<int64_t>(1, (1 << 22) / tiles);  // examples of a launch: grids below 2^32 threads
  for (int64_t b = 0; b < p.batch; b += most) {
    a.b0 = (int)b;
    const unsigned blocks = (unsigned)(a.blocks + (dweight ? tiles * std::min(most, p.batch - b) : 0));
    hipLaunchKernelGGL((k_back<C, M, TO>), dim3(blocks), dim3(C::TH), 0, st, a);
    a.blocks = 0;  // dH came with the first
    if (!dweight) break;
  }
}
template <Mode M, typename TO>
void run_back(const Plan &p, const Back &a, bool dhidden, bool dweight, hipStream_t st) {
  if constexpr (M != kPair)  // few rows an example
    if (p.huge) return launch_back<Huge, M, TO>(p, a, dhidden, dweight, st);
  if constexpr (M != kPair || sizeof(TO) == 4)
    if (p.large) return launch_back<Large, M, TO>(p, a, dhidden, dweight, st);
  launch_back<Small, M, TO>(p, a, dhidden, dweight, st);
}

}  // namespace

extern "C" {

int64_t sketch_linear_logp_work_bytes(const sk_linear *x) {
  if (check_linear(x) != SK_OK) return 0;
  return plan_of(x, 1, false, false, false, false).bytes;
}

int sketch_linear_logp(const sk_linear *x, float *logp, float *stats, void *work, int64_t work_bytes, void *stream) {
  int rc = check_linear(x);
  if (rc != SK_OK || x->rows == 0) return rc;
  if (!logp || !work) return train_fail(SK_EINVAL, "NULL argument");
  const Plan p = plan_of(x, 1, false, false, false, false);
  if (work_bytes < p.bytes) return train_fail(SK_EINVAL, "work is smaller than sketch_linear_logp_work_bytes");
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  if (p.few) {
    const int units = (int)p.units;
    const Few a{x->hidden, x->weight, x->targets, x->ld_hidden, x->ld_weight, (int)x->rows, (int)x->vocab, (int)x->width,
                (int)x->index, x->scale, ptr<float2>(work, p.part), ptr<float>(work, p.xt), units, logp, (float2 *)stats, 0, 0, nullptr,
                nullptr, nullptr, nullptr, nullptr, 0, 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
    if (p.f16)
      hipLaunchKernelGGL((k_few<float, false>), dim3(units), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((k_few<bf16, false>), dim3(units), dim3(256), 0, st, a);
    hipLaunchKernelGGL(k_few_join, dim3((unsigned)x->rows), dim3(512), 0, st, a);
    return train_launched();
  }
  begin(x, p, nullptr, nullptr, logp, stats, work, st);
  for (int64_t v0 = 0; v0 < x->vocab; v0 += p.piece) {
    const int64_t valid = std::min(p.piece, x->vocab - v0);
    Logit a = logit_of(x, p, v0, valid, weights(x, p, v0, valid, work, st), work);
    a.part = ptr<float2>(work, p.part);
    a.xt = ptr<float>(work, p.xt);
    run_logits<false>(p, a, st);
    const Join j{a.meta, ptr<int>(work, p.list), a.part, a.xt, p.tcap, (int)up(valid, 128) / 64, x->scale, v0 == 0,
                 v0 + valid == x->vocab, ptr<float2>(work, p.run), logp, (float2 *)stats};
    hipLaunchKernelGGL(k_join, dim3((unsigned)(up(x->rows, kPad) / 16)), dim3(1024), 0, st, j);
  }
  return train_launched();
}

int64_t sketch_linear_logp_grad_work_bytes(const sk_linear *x, int64_t batch, int32_t dhidden, int32_t dweight) {
  if (check_linear(x) != SK_OK || check_batch(x, batch) != SK_OK) return 0;
  // either type of dW
  return std::max(plan_of(x, batch, true, dhidden, dweight, false).bytes, plan_of(x, batch, true, dhidden, dweight, true).bytes);
}

int sketch_linear_logp_grad(const sk_linear *x, int64_t batch, const float *stats, const float *dlogp, void *dhidden,
                            int64_t ld_dhidden, void *dweight, sk_dtype dweight_dtype, int32_t accumulate, void *work,
                            int64_t work_bytes, void *stream) {
  int rc = check_linear(x);
  if (rc != SK_OK || (rc = check_batch(x, batch)) != SK_OK) return rc;
  if (dweight_dtype != SK_F32 && dweight_dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (x->dtype == SK_F32 && dweight_dtype != SK_F32) return train_fail(SK_EDTYPE, "dweight of fp32 weights is fp32");
  if (!work || (x->rows && (!stats || !dlogp)) || (!dhidden && !dweight)) return train_fail(SK_EINVAL, "NULL argument");
  if (dhidden && ld_dhidden < x->width) return train_fail(SK_EINVAL, "need ld_dhidden >= width");
  if (work_bytes < sketch_linear_logp_grad_work_bytes(x, batch, dhidden != nullptr, dweight != nullptr))
    return train_fail(SK_EINVAL, "work is smaller than sketch_linear_logp_grad_work_bytes");
  const Plan p = plan_of(x, batch, true, dhidden != nullptr, dweight != nullptr, dweight && dweight_dtype == SK_F32);
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  // the list takes dlogp = NULL for the forward direction; without rows nothing is read from it
  begin(x, p, dlogp ? dlogp : (const float *)work, stats, nullptr, nullptr, work, st);
  Meta *meta = ptr<Meta>(work, p.meta);
  const int64_t width = x->width;
  uint16_t *g = dhidden || !p.f16 ? ptr<uint16_t>(work, p.g) : nullptr;
  uint16_t *gw = dweight && p.f16 ? ptr<uint16_t>(work, p.gw) : nullptr;
  for (int64_t v0 = 0; v0 < x->vocab; v0 += p.piece) {
    const int64_t valid = std::min(p.piece, x->vocab - v0);
    const Operand w = x->rows ? weights(x, p, v0, valid, work, st) : Operand{};
    if (x->rows) {
      Logit a = logit_of(x, p, v0, valid, w, work);
      a.prm = ptr<RowPrm>(work, p.prm);
      a.g = g;
      a.rest = ptr<float>(work, p.rest);
      a.marks = ptr<uint8_t>(work, p.marks);
      a.gplane = p.tcap * p.piece;
      a.piece = p.piece;
      a.gw = gw;
      a.ph = ptr<int>(work, p.ph);
      a.pw = ptr<int>(work, p.pw);
      a.cs = ptr<float>(work, p.cs);
      if (x->rows <= kFew) {
        const Few f{x->hidden, x->weight, x->targets, x->ld_hidden, x->ld_weight, (int)x->rows, (int)x->vocab, (int)width,
                    (int)x->index, x->scale, nullptr, nullptr, 0, nullptr, nullptr, (int)v0, (int)valid, meta,
                    ptr<int>(work, p.pos), ptr<int>(work, p.list), a.prm, a.g, a.gplane, a.piece, a.gw, a.ph, a.pw, a.eh, a.ev,
                    a.cs};
        const dim3 grid((unsigned)((valid + kFewUnit - 1) / kFewUnit));
        if (p.f16)
          hipLaunchKernelGGL((k_few<float, true>), grid, dim3(256), 0, st, f);
        else
          hipLaunchKernelGGL((k_few<bf16, true>), grid, dim3(256), 0, st, f);
      } else {
        run_logits<true>(p, a, st);
      }
    }
    Back a{};
    a.width = (int)width;
    a.meta = meta;
    a.seg = ptr<int>(work, p.seg);
    a.tcap = p.tcap;
    const uint16_t *hd = ptr<uint16_t>(work, p.hc);
    a.g = Operand{{g, g + (p.pair ? p.tcap * p.piece : 0)}, p.piece * p.planes};
    a.w = w;
    a.steps = (int)(up(valid, kStep) / kStep);
    a.splits = (int)p.splits;
    a.per = (int)((a.steps + p.splits - 1) / p.splits);
    a.first = v0 == 0;
    a.acc = ptr<float>(work, p.acc);
    a.kp = (int)p.kp;
    a.gw = gw ? Operand{{gw, gw}, p.piece * p.planes} : a.g;
    a.ph = ptr<int>(work, p.ph);
    a.pw = Powers{ptr<int>(work, p.pw), p.piece};
    a.h = Operand{{hd, hd}, p.kp * p.planes};
    a.tgt = ptr<int>(work, p.tgt);
    a.rest = ptr<float>(work, p.rest);
    a.marks = ptr<uint8_t>(work, p.marks);
    a.v0 = (int)v0;
    a.valid = (int)valid;
    a.out = (char *)dweight + v0 * width * (dweight_dtype == SK_F32 ? 4 : 2);
    a.vocab = x->vocab;
    a.accumulate = accumulate != 0;
    a.past = batch * x->vocab * width * (dweight_dtype == SK_F32 ? 4 : 2) > kPastBytes;
    const bool dh = dhidden && x->rows;
    if (!dh && !dweight) continue;
    const bool dw = dweight != nullptr, single = dweight_dtype == SK_F32;
    if (p.f16)
      run_back<kSplit, float>(p, a, dh, dw, st);
    else if (p.pair)
      single ? run_back<kPair, float>(p, a, dh, dw, st) : run_back<kPair, bf16>(p, a, dh, dw, st);
    else
      single ? run_back<kBf16, float>(p, a, dh, dw, st) : run_back<kBf16, bf16>(p, a, dh, dw, st);
  }
  if (dhidden && x->rows) {
    const dim3 grid((unsigned)((x->rows + 3) / 4));
    const DHidden a{ptr<int>(work, p.pos), ptr<int>(work, p.tgt), ptr<float>(work, p.cs), p.pair ? nullptr : ptr<float>(work, p.rest),
                    ptr<float>(work, p.acc), p.tcap, (int)p.kp, (int)p.splits, (int)x->rows, (int)width, x->weight, x->ld_weight,
                    dhidden, ld_dhidden};
    if (p.f16)
      hipLaunchKernelGGL(k_dhidden_out<float>, grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_dhidden_out<bf16>, grid, dim3(256), 0, st, a);
  }
  return train_launched();
}

}  // extern "C"
