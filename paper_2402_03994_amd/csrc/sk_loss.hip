// sk_loss.hip -- token log-probabilities, the clipped policy loss and the
// preference loss, with their gradients with respect to the logits (C ABI of
// include/sketch_train.h).
//
// A row x of logits enters through its largest entry m and z = sum_j
// exp(scale (x_j - m)): log p_t = scale (x_t - m) - log z, and every gradient is
// a number c of the row times scale (onehot - p).  The exponentials are at most
// 1, so a row whose entries are all the type's lowest value is the uniform
// distribution; a row of -inf alone has m taken as 0 and z = 0.  Sums, statistics
// and factors are fp32 (over positions and texts fp64); a gradient is rounded
// once, to the type of the logits.
//
// Every kernel is bound by memory (a large copy reaches 4.9 TB/s on the card, a
// fill 6.8, reading alone 6.3):
//   k_logp       one read of the unmasked rows, by the threads of one workgroup
//                (or one wave) that hold a row, or stream it, in registers.
//                Each thread sums under its own maximum, so that one barrier
//                joins both.  10682 x 50257 bf16: 175 to 183 us, 6 TB/s.
//   k_policy     the same, then the token's loss and the row's gradient from
//                the registers: one read, one write, no second launch over the
//                logits.  8192 x 128256 bf16, 40% masked: 603 us, 5.6 TB/s.
//   k_logp_grad  the gradient from known (m, z).  The preference loss needs it:
//                a row's factor is known when its pair's rows have all been
//                read.  16384 x 50257 bf16, 40% masked: 179 us of k_logp, 447
//                us (5.9 TB/s), of a floor of 540 us for one read and one write.
//   k_pair       a workgroup a pair, 4 to 7 us; k_policy_total one workgroup, 2
//                to 5 us.
#include <algorithm>
#include <type_traits>

#include "sk_train.h"

using namespace sk;

namespace {

struct Rows {
  const void *x;
  const void *targets;
  int64_t ld;
  int32_t vocab;
  int32_t index;
  float scale;
  bool past;  // the gradient is stored past the caches
};

// the target of row t, -1 where it is masked
__device__ __forceinline__ int target_at(const Rows &r, int64_t t) {
  const int64_t v = r.index == SK_I64 ? ((const int64_t *)r.targets)[t] : ((const int32_t *)r.targets)[t];
  return v >= 0 && v < r.vocab ? (int)v : -1;
}

// A row cut at 16-byte boundaries: `head` entries before the first one, nv vectors, `rem` entries after the last.
// Odd vocabularies put rows of bf16 at any even address, where 16-byte accesses across the boundaries cost a fifth of
// the bandwidth (50257 columns: 5.2 TB/s read as they lie, 6.3 TB/s cut).
struct Cut {
  int head, nv, rem;
};
template <typename T>
__device__ __forceinline__ Cut cut_of(const T *x, int vocab) {
  constexpr int N = Vec<T>::N;
  int head = (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T);
  head = head < vocab ? head : vocab;
  const int nv = (vocab - head) / N;
  return Cut{head, nv, vocab - head - nv * N};
}

// The part of a row that a thread of THREADS holds: up to NV vectors, THREADS vectors apart, from vector v0 on, and
// (with the first tile) one of the entries outside the vectors: thread i < 8 the head's, thread 8 + i the last ones.
// What is beyond the row is -inf.  The last NL of the NV vectors lie in LDS, each thread's own (no barrier).
template <typename T, int THREADS, int NV, int NL = 0>
struct Tile {
  static constexpr int N = Vec<T>::N;
  static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
  static constexpr int NR = NV - NL;  // vectors in registers
  u32x4 raw[NR];
  float rest;
  u32x4 *lds;  // [NL][THREADS]

  __device__ __forceinline__ u32x4 vec(int k, int tid) const { return k < NR ? raw[k] : lds[(k - NR) * THREADS + tid]; }

  // where the thread's single entry lies, -1 if it has none
  static __device__ __forceinline__ int single(Cut q, int v0, int tid) {
    if (v0 == 0 && tid < q.head) return tid;
    if (v0 == 0 && tid >= 8 && tid < 8 + q.rem) return q.head + q.nv * N + tid - 8;
    return -1;
  }
  // the thread that holds entry j, within the tiles of v0
  static __device__ __forceinline__ int owner(Cut q, int j) {
    if (j < q.head) return j;
    const int i = (j - q.head) / N;
    return i < q.nv ? i % THREADS : 8 + j - q.head - q.nv * N;
  }
  __device__ __forceinline__ void load(const T *x, Cut q, int v0, int tid) {
    const T *a = x + q.head;
    auto one = [&](int k) {
      const int i = v0 + k * THREADS + tid;
      u32x4 v = u32x4{kNone, kNone, kNone, kNone};
      if (i < q.nv) v = Vec<T>::load(a + (int64_t)i * N);
      return v;
    };
    if (NL) {  // LDS first, so that the registers they pass through are free again for the others
#pragma unroll
      for (int k = 0; k < NL; ++k) lds[k * THREADS + tid] = one(NR + k);
      asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int k = 0; k < NR; ++k) raw[k] = one(k);
    const int j = single(q, v0, tid);
    rest = j >= 0 ? to_f32(x[j]) : -INFINITY;
  }
  // The vectors stay packed, and in LDS, between two uses: without this the compiler carries the unpacked bf16 values
  // along, twice the registers, and those of LDS too.
  __device__ __forceinline__ void stay() {
    if (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < NR; ++k) asm volatile("" : "+v"(raw[k]));
    }
    if (NL) asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ float largest(int tid) const {
    float m = rest;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const u32x4 v = vec(k, tid);
#pragma unroll
      for (int i = 0; i < N; ++i) m = fmaxf(m, Vec<T>::get(v, i));
    }
    return m;
  }
  __device__ __forceinline__ float expsum(float m, float k2, int tid) const {
    float z = __builtin_amdgcn_exp2f((rest - m) * k2);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const u32x4 v = vec(k, tid);
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((Vec<T>::get(v, i) - m) * k2);
      z += s;
    }
    return z;
  }
  // w exp(scale (x - m)) to the row d, past the caches where that keeps the logits in them for the gradient pass (4096 x
  // 50257 bf16 read twice and written once: 169 us with ordinary stores, 153 us)
  __device__ __forceinline__ void store(T *d, Cut q, int v0, int tid, float m, Power p, float w, bool past) const {
    T *a = d + q.head;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = v0 + k * THREADS + tid;
      if (i < q.nv) {
        const u32x4 v = vec(k, tid);
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = w * entry_exp<T>(Vec<T>::get(v, e) - m, p);
        Vec<T>::store(a + (int64_t)i * N, Vec<T>::pack(f), past);
      }
    }
    const int j = single(q, v0, tid);
    if (j >= 0) d[j] = from_f32<T>(w * entry_exp<T>(rest - m, p));
  }
};

// zeros to vectors v0 + tid, v0 + tid + THREADS, .. below v1 of a row and (with its first ones) to what lies outside them
template <typename T, int THREADS>
__device__ __forceinline__ void row_zero(T *d, int vocab, int v0, int v1, int tid, bool past) {
  const Cut q = cut_of(d, vocab);
  v1 = v1 < q.nv ? v1 : q.nv;
  for (int i = v0 + tid; i < v1; i += THREADS) Vec<T>::store(d + q.head + (int64_t)i * Vec<T>::N, u32x4{0, 0, 0, 0}, past);
  const int j = Tile<T, THREADS, 1>::single(q, v0, tid);
  if (j >= 0) d[j] = from_f32<T>(0.0f);
}

// exp(scale (x - m)) of what a thread has summed under its own largest entry, moved to the common m
__device__ __forceinline__ float moved(Stats s, float m, float k2) {
  return s.z == 0.0f ? 0.0f : s.z * __builtin_amdgcn_exp2f((s.m - m) * k2);
}

// Joins the threads' (m, z): within the waves, then the waves' through LDS (two rows of THREADS / 64 entries).
template <int THREADS>
__device__ __forceinline__ Stats join(Stats s, float k2, float (*lds)[16]) {
  constexpr int W = THREADS / 64;
  const float mw = wave_all(s.m, OpMax());
  Stats r{mw, wave_all(moved(s, mw, k2), OpAdd())};
  if (W > 1) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 0) {
      lds[0][wave] = r.m;
      lds[1][wave] = r.z;
    }
    __syncthreads();
    Stats q{lane < W ? lds[0][lane] : -INFINITY, lane < W ? lds[1][lane] : 0.0f};
    r.m = wave_all(q.m, OpMax());
    r.z = wave_all(moved(q, r.m, k2), OpAdd());
  }
  if (r.m == -INFINITY) r.m = 0.0f;
  return r;
}

// (m, z) of a tile's entries by one thread; an exponent of no entry at all is left out
template <typename TileT>
__device__ __forceinline__ Stats thread_stats(TileT &t, float k2, int tid) {
  const float m = t.largest(tid);
  t.stay();
  return Stats{m, t.expsum(m == -INFINITY ? 0.0f : m, k2, tid)};
}

// Writes the row c scale (onehot - p) of a target; called with what the threads hold of the row, or (RESIDENT false)
// with nothing: the row is read again, tile by tile.
template <typename T, int THREADS, int NV, bool RESIDENT, typename TileT>
__device__ __forceinline__ void row_grad(const T *x, T *d, int vocab, float scale, Stats s, int target, float xt, float c,
                                         bool past, TileT &t, int tid) {
  if (c == 0.0f || s.z == 0.0f) {
    row_zero<T, THREADS>(d, vocab, 0, INT32_MAX, tid, past);
    return;
  }
  const Cut q = cut_of(x, vocab);
  const Power p = power_of(scale);
  const float cs = c * scale, w = -cs / s.z;
  if (RESIDENT) {
    t.stay();
    t.store(d, q, 0, tid, s.m, p, w, past);
  } else {
    for (int v0 = 0; v0 < q.nv || v0 == 0; v0 += THREADS * NV) {
      t.load(x, q, v0, tid);
      t.store(d, q, v0, tid, s.m, p, w, past);
    }
  }
  // the target's entry, again by the thread that has just stored it
  if (tid == TileT::owner(q, target))
    d[target] = from_f32<T>(cs * (1.0f - entry_exp<T>(xt - s.m, p) / s.z));
}

template <typename T, int THREADS, int NV, bool RESIDENT, typename TileT>
__device__ __forceinline__ Stats row_stats(const T *x, int vocab, float k2, TileT &t, int tid, float (*lds)[16]) {
  const Cut q = cut_of(x, vocab);
  t.load(x, q, 0, tid);
  Stats s = thread_stats(t, k2, tid);
  if (!RESIDENT) {
    for (int v0 = THREADS * NV; v0 < q.nv; v0 += THREADS * NV) {
      t.load(x, q, v0, tid);
      const Stats o = thread_stats(t, k2, tid);
      const float m = fmaxf(s.m, o.m);
      s = Stats{m, moved(s, m, k2) + moved(o, m, k2)};
    }
  }
  return join<THREADS>(s, k2, lds);
}

struct Policy {
  const float *old_logp, *adv, *weights, *ref;
  float lo, hi, kl;
};

// l_t and its derivative with respect to logp
__device__ __forceinline__ void policy_token(const Policy &p, int64_t t, float logp, float &l, float &d) {
  const float A = p.adv[t], r = expf(logp - p.old_logp[t]);
  const float free = A * r, held = A * fminf(fmaxf(r, p.lo), p.hi);
  // of the two the smaller counts; NaN is kept
  l = free <= held || free != free ? -free : -held;
  d = free <= held || free != free ? -free : 0.0f;
  if (p.kl != 0.0f) {
    const float u = p.ref[t] - logp, e = expm1f(u);  // near the reference e^u - 1 would have lost what u is
    l += p.kl * (e - u);
    d -= p.kl * e;
  }
}

// One row by THREADS threads, from row0 on; rows of one wave share a workgroup of four.
template <int THREADS>
__device__ __forceinline__ int64_t row_of_thread(int64_t row0, int &tid) {
  if (THREADS > 64) {
    tid = threadIdx.x;
    return row0 + blockIdx.x;
  }
  tid = threadIdx.x & 63;
  return row0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
}

template <typename T, int THREADS, int NV, bool RESIDENT>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_logp(Rows r, int64_t row0, int64_t rows,
                                                                       float *__restrict__ logp,
                                                                       float2 *__restrict__ stats,
                                                                       float *__restrict__ rowc) {
  __shared__ float lds[2][16];
  int tid;
  const int64_t t = row_of_thread<THREADS>(row0, tid);
  if (t >= rows) return;
  const int target = target_at(r, t);
  const T *x = (const T *)r.x + t * r.ld;
  Stats s{0.0f, 0.0f};
  float lp = 0.0f;
  if (target >= 0) {
    const float xt = to_f32(x[target]);
    Tile<T, THREADS, NV> tile;
    s = row_stats<T, THREADS, NV, RESIDENT>(x, r.vocab, r.scale * kLog2e, tile, tid, lds);
    lp = logp_of(xt, s, r.scale);
  }
  if (tid == 0) {
    logp[t] = lp;
    if (stats) stats[t] = make_float2(s.m, s.z);
    if (rowc) rowc[t] = 0.0f;  // until a pair has its factors: rows outside all texts keep it
  }
}

// d (NULL: the loss alone) may be the logits: a row's threads hold it, or have all read it, before any of them writes.
template <typename T, int THREADS, int NV, bool RESIDENT, int NL>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_policy(Rows r, int64_t row0, int64_t rows, Policy p,
                                                                         float *__restrict__ logp,
                                                                         float *__restrict__ loss_t, void *d,
                                                                         int64_t ldd) {
  __shared__ float lds[2][16];
  int tid;
  const int64_t t = row_of_thread<THREADS>(row0, tid);
  if (t >= rows) return;
  const int target = target_at(r, t);
  const float w = target >= 0 ? p.weights[t] : 0.0f;
  const T *x = (const T *)r.x + t * r.ld;
  __shared__ u32x4 more[NL ? NL * THREADS : 1];
  Tile<T, THREADS, NV, NL> tile;
  tile.lds = more;
  Stats s{0.0f, 0.0f};
  float lp = 0.0f, l = 0.0f, c = 0.0f, xt = 0.0f;
  if (w != 0.0f) {
    xt = to_f32(x[target]);
    s = row_stats<T, THREADS, NV, RESIDENT>(x, r.vocab, r.scale * kLog2e, tile, tid, lds);
    lp = logp_of(xt, s, r.scale);
    policy_token(p, t, lp, l, c);
    c *= w;
  }
  if (tid == 0) {
    logp[t] = lp;
    loss_t[t] = l;
  }
  if (d) row_grad<T, THREADS, NV, RESIDENT>(x, (T *)d + t * ldd, r.vocab, r.scale, s, target, xt, c, r.past, tile, tid);
}

// the mean of the pairs' losses, by 256 threads
__device__ __forceinline__ void pair_total(const float *pair_loss, int64_t pairs, float *loss, double *lds) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < pairs; i += 256) s += pair_loss[i];
  s = block_all<4>(s, OpAdd(), lds);
  if (threadIdx.x == 0) *loss = (float)(s / (double)pairs);
}

// The gradient from known (m, z): nothing of a row has to be held, so a row is cut into pieces of 256 x NV vectors, one
// workgroup each.  The last rows come first: they are what the kernel that found (m, z) has left in the cache.
// One workgroup more (the preference loss) adds up the pairs' losses meanwhile.
template <typename T, int NV>
__global__ __launch_bounds__(256) void k_logp_grad(Rows r, int64_t rows, int pieces, const float2 *__restrict__ stats,
                                                   const float *__restrict__ dlogp, void *dl, int64_t ldd,
                                                   const float *__restrict__ pair_loss, int64_t pairs,
                                                   float *__restrict__ loss) {
  typedef Tile<T, 256, NV> TileT;
  __shared__ double lds[4];
  if (blockIdx.x >= rows * pieces) {
    pair_total(pair_loss, pairs, loss, lds);
    return;
  }
  const int64_t t = rows - 1 - blockIdx.x / (unsigned)pieces;
  const int v0 = (int)(blockIdx.x % (unsigned)pieces) * 256 * NV, tid = threadIdx.x;
  const int target = target_at(r, t), vocab = r.vocab;
  const T *x = (const T *)r.x + t * r.ld;
  T *d = (T *)dl + t * ldd;
  const float c = target >= 0 ? dlogp[t] : 0.0f;
  const float2 s = stats[t];
  if (c == 0.0f || s.y == 0.0f) {
    row_zero<T, 256>(d, vocab, v0, v0 + 256 * NV, tid, r.past);
    return;
  }
  const Power p = power_of(r.scale);
  const float cs = c * r.scale;
  const Cut q = cut_of(x, vocab);
  const int i = (target - q.head) / TileT::N;  // the target's vector; outside them the first piece's
  const bool here = target >= q.head && i < q.nv ? i >= v0 && i < v0 + 256 * NV : v0 == 0;
  const bool mine = here && tid == TileT::owner(q, target);
  const float xt = mine ? to_f32(x[target]) : 0.0f;  // read before the thread's stores, for the gradient in place
  TileT tile;
  tile.load(x, q, v0, tid);
  tile.store(d, q, v0, tid, s.x, p, -cs / s.y, r.past);
  if (mine) d[target] = from_f32<T>(cs * (1.0f - entry_exp<T>(xt - s.x, p) / s.y));
}

// sum_t w_t l_t over the unmasked rows, in fp64 in a fixed order
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_policy_total(Rows r, int64_t rows, const float *__restrict__ w,
                                                          const float *__restrict__ l, float *__restrict__ loss) {
  __shared__ double lds[THREADS / 64];
  double s = 0.0;
#pragma unroll 4
  for (int64_t t = threadIdx.x; t < rows; t += THREADS) {
    const float wt = w[t], lt = l[t];
    s += target_at(r, t) >= 0 && wt != 0.0f ? (double)wt * lt : 0.0;
  }
  s = block_all<THREADS / 64>(s, OpAdd(), lds);
  if (threadIdx.x == 0) *loss = (float)s;
}

struct Pairs {
  const void *offsets;
  int32_t index, average;
  int64_t pairs, rows;
  const float *ref;
  float beta, smoothing;
};

__device__ __forceinline__ int64_t offset_at(const Pairs &p, int64_t i) {
  const int64_t v = p.index == SK_I64 ? ((const int64_t *)p.offsets)[i] : ((const int32_t *)p.offsets)[i];
  return v < 0 ? 0 : v > p.rows ? p.rows : v;
}

__device__ __forceinline__ double softplus(double u) { return fmax(u, 0.0) + log1p(exp(-fabs(u))); }

// One workgroup per pair, half of it per text: the texts' sums, the pair's loss, and each row's factor d loss / d logp.
__global__ __launch_bounds__(512) void k_pair(Rows r, Pairs p, const float *__restrict__ logp,
                                              float *__restrict__ rowc, float *__restrict__ seq,
                                              float *__restrict__ pair_loss) {
  __shared__ double sums[3][8];
  const int64_t pair = blockIdx.x;
  const int h = threadIdx.x >> 8, tid = threadIdx.x & 255;
  const int64_t a = offset_at(p, 2 * pair + h), b = offset_at(p, 2 * pair + h + 1);
  double s = 0.0, g = 0.0, n = 0.0;
#pragma unroll 4
  for (int64_t t = a + tid; t < b; t += 256) {
    const float lp = logp[t], ref = p.ref[t];
    const bool live = target_at(r, t) >= 0;
    s += live ? (double)lp : 0.0;
    g += live ? (double)lp - ref : 0.0;
    n += live ? 1.0 : 0.0;
  }
  s = wave_all(s, OpAdd());
  g = wave_all(g, OpAdd());
  n = wave_all(n, OpAdd());
  if ((threadIdx.x & 63) == 0) {
    sums[0][threadIdx.x >> 6] = s;
    sums[1][threadIdx.x >> 6] = g;
    sums[2][threadIdx.x >> 6] = n;
  }
  __syncthreads();
  double share[2], gap[2], total[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const double *q = &sums[0][4 * i];
    total[i] = (q[0] + q[1]) + (q[2] + q[3]);
    gap[i] = (q[8] + q[9]) + (q[10] + q[11]);
    share[i] = p.average ? 1.0 / fmax((q[16] + q[17]) + (q[18] + q[19]), 1.0) : 1.0;
  }
  const double d = (double)p.beta * (gap[0] * share[0] - gap[1] * share[1]), eps = p.smoothing;
  if (tid == 0) seq[2 * pair + h] = (float)(total[h] * share[h]);
  if (threadIdx.x == 0)
    pair_loss[pair] = (float)((eps < 1.0 ? (1.0 - eps) * softplus(-d) : 0.0) + (eps > 0.0 ? eps * softplus(d) : 0.0));
  const double c = -(double)p.beta / (double)p.pairs * ((1.0 - eps) / (1.0 + exp(d)) - eps / (1.0 + exp(-d)));
  const float ch = (float)((h ? -c : c) * share[h]);
  for (int64_t t = a + tid; t < b; t += 256) rowc[t] = ch;
}

__global__ __launch_bounds__(256) void k_pair_total(const float *__restrict__ pair_loss, int64_t pairs,
                                                    float *__restrict__ loss) {
  __shared__ double lds[4];
  pair_total(pair_loss, pairs, loss, lds);
}

int check_logits(const sk_logits *x) {
  if (!x) return train_fail(SK_EINVAL, "NULL argument");
  if (x->dtype != SK_F32 && x->dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (x->index != SK_I32 && x->index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (x->rows < 0 || x->vocab < 1 || x->ld < x->vocab)
    return train_fail(SK_EINVAL, "need rows >= 0, vocab >= 1 and ld >= vocab");
  // scale log2 e stays finite, and where x - m overflows, the exponent -2^128 scale of its exponential is one of 0
  if (!(x->scale >= 0x1p-120f && x->scale <= 0x1p127f))
    return train_fail(SK_EINVAL, "scale must be in [2^-120, 2^127]");
  if (x->rows > INT32_MAX || x->vocab > INT32_MAX)
    return train_fail(SK_EUNSUPPORTED, "more than 2^31 - 1 rows or columns");
  if (x->rows && (!x->data || !x->targets)) return train_fail(SK_EINVAL, "NULL argument");
  return SK_OK;
}

int check_out(const sk_logits *x, const void *dlogits, int64_t ld_out) {
  if (!dlogits) return SK_OK;
  if (ld_out < x->vocab) return train_fail(SK_EINVAL, "need ld_out >= vocab");
  if (dlogits == x->data && ld_out != x->ld) return train_fail(SK_EINVAL, "in place needs ld_out = ld");
  return SK_OK;
}

Rows rows_of(const sk_logits *x) {
  const int64_t bytes = x->rows * x->vocab * (x->dtype == SK_F32 ? 4 : 2);
  return Rows{x->data, x->targets, x->ld, (int32_t)x->vocab, (int32_t)x->index, x->scale, bytes > kPastBytes};
}

template <int V>
using Int = std::integral_constant<int, V>;

// f(threads, vectors of a thread, resident, vectors of them in LDS) for rows of up to nv vectors.  Where there are
// many rows, what counts is how much of them the chip holds at a time: four to eight vectors a thread, so that a CU has
// several rows (bf16 columns, log-probabilities and policy update: 4142 columns 4.2 and 5.3 TB/s with 256 threads, 5.2
// and 5.6 with one wave; 16924 columns 4.3 and 4.9 with 1024 threads, 5.2 and 5.7 with 512).  Up to 512 rows leave
// waves to spare, and a row is done sooner by four of them (4000 columns, 64 rows, policy: 3.8 us, 5.1 us by one; 1024
// rows: 6.7 us, 5.9 us).  Six of eight vectors a thread are the most that 512 threads take: 8192 rows, policy update with
// 512 threads of 8 and 1024 of 4, bf16 95 and 118 us (2100 vectors), 154 and 153 (3100), 172 and 167 (3584), 218 and 200
// (4090); fp32 91 and 102, 151 and 142, 168 and 157, 216 and 189.
template <typename F>
void with_row_shape(int64_t nv, int64_t rows, F f) {
  const bool few = rows <= 512;
  if (nv <= 64 * 4)
    f(Int<64>(), Int<4>(), std::true_type(), Int<0>());
  else if (!few && nv <= 64 * 8)
    f(Int<64>(), Int<8>(), std::true_type(), Int<0>());
  else if (!few && nv <= 64 * 12)
    f(Int<64>(), Int<12>(), std::true_type(), Int<0>());
  else if (nv <= 256 * 4)
    f(Int<256>(), Int<4>(), std::true_type(), Int<0>());
  else if (nv <= 256 * 8)
    f(Int<256>(), Int<8>(), std::true_type(), Int<0>());
  else if (nv <= 512 * 6)
    f(Int<512>(), Int<8>(), std::true_type(), Int<0>());
  else if (nv <= 1024 * 4)
    f(Int<1024>(), Int<4>(), std::true_type(), Int<0>());
  else if (nv <= 1024 * 8)
    f(Int<1024>(), Int<8>(), std::true_type(), Int<0>());
  else if (nv <= 1024 * 16)
    f(Int<1024>(), Int<16>(), std::true_type(), Int<0>());
  else if (nv <= 1024 * 32)  // 384 KB of registers and 128 KB of LDS (128256 fp32 columns: 5.5 TB/s, 3.7 read twice)
    f(Int<1024>(), Int<32>(), std::true_type(), Int<8>());
  else
    f(Int<1024>(), Int<8>(), std::false_type(), Int<0>());
}

// launch(first row, workgroups) for all rows of a kernel that takes `per` rows a workgroup of `threads`: HIP refuses
// grids of 2^32 threads.
template <typename F>
void row_parts(int64_t rows, int per, int threads, F launch) {
  const int64_t most = ((1ll << 31) / threads) * per;
  for (int64_t r0 = 0; r0 < rows; r0 += most)
    launch(r0, (unsigned)((std::min(most, rows - r0) + per - 1) / per));
}

template <typename T, int TH, int NV, bool RES>
void launch_logp(const sk_logits *x, float *logp, float *stats, float *rowc, hipStream_t st) {
  constexpr int kPer = TH == 64 ? 4 : 1, kThreads = TH * kPer;
  row_parts(x->rows, kPer, kThreads, [&](int64_t r0, unsigned blocks) {
    hipLaunchKernelGGL((k_logp<T, TH, NV, RES>), dim3(blocks), dim3(kThreads), 0, st, rows_of(x), r0, x->rows, logp,
                       (float2 *)stats, rowc);
  });
}

template <typename T>
void run_logp_t(const sk_logits *x, float *logp, float *stats, float *rowc, hipStream_t st) {
  with_row_shape(x->vocab / Vec<T>::N, x->rows, [&](auto th, auto nv, auto res, auto) {
    // a row that is read once need not be held: above 1024 x 8 vectors it is streamed
    constexpr int TH = decltype(th)::value, NV = decltype(nv)::value;
    if constexpr (TH == 1024 && NV > 8)
      launch_logp<T, 1024, 8, false>(x, logp, stats, rowc, st);
    else
      launch_logp<T, TH, NV, decltype(res)::value>(x, logp, stats, rowc, st);
  });
}

void run_logp(const sk_logits *x, float *logp, float *stats, float *rowc, hipStream_t st) {
  if (x->dtype == SK_F32)
    run_logp_t<float>(x, logp, stats, rowc, st);
  else
    run_logp_t<bf16>(x, logp, stats, rowc, st);
}

template <typename T>
void run_policy_t(const sk_logits *x, const Policy &p, float *logp, float *token_loss, void *d, int64_t ldd,
                  hipStream_t st) {
  with_row_shape(x->vocab / Vec<T>::N, x->rows, [&](auto th, auto nv, auto res, auto nl) {
    constexpr int TH = decltype(th)::value, kPer = TH == 64 ? 4 : 1, kThreads = TH * kPer;
    row_parts(x->rows, kPer, kThreads, [&](int64_t r0, unsigned blocks) {
      hipLaunchKernelGGL((k_policy<T, TH, decltype(nv)::value, decltype(res)::value, decltype(nl)::value>), dim3(blocks),
                         dim3(kThreads), 0, st, rows_of(x), r0, x->rows, p, logp, token_loss, d, ldd);
    });
  });
}

struct PairTotal {  // of the preference loss
  const float *pair_loss = nullptr;
  int64_t pairs = 0;
  float *loss = nullptr;
};

template <typename T>
void run_logp_grad_t(const sk_logits *x, const float *stats, const float *dlogp, void *d, int64_t ldd, PairTotal total,
                     hipStream_t st) {
  constexpr int NV = 2;  // 16384 x 50257 bf16 rows, 40% masked, both passes: 642 us with 2, 649 with 4, 692 with 8
  const int64_t pieces = std::max<int64_t>(1, (x->vocab / Vec<T>::N + 256 * NV - 1) / (256 * NV));
  const int64_t most = std::max<int64_t>(1, kGridBlocks / pieces);
  for (int64_t r0 = 0; r0 < x->rows; r0 += most) {
    Rows r = rows_of(x);
    r.x = (const T *)r.x + r0 * r.ld;
    r.targets = (const char *)r.targets + r0 * (x->index == SK_I64 ? 8 : 4);
    const int64_t n = std::min(most, x->rows - r0);
    const int64_t blocks = n * pieces + (r0 == 0 && total.loss ? 1 : 0);
    hipLaunchKernelGGL((k_logp_grad<T, NV>), dim3((unsigned)blocks), dim3(256), 0, st, r, n, (int)pieces,
                       (const float2 *)stats + r0, dlogp + r0, (T *)d + r0 * ldd, ldd, total.pair_loss, total.pairs,
                       total.loss);
  }
}

void run_logp_grad(const sk_logits *x, const float *stats, const float *dlogp, void *d, int64_t ldd, PairTotal total,
                   hipStream_t st) {
  if (x->dtype == SK_F32)
    run_logp_grad_t<float>(x, stats, dlogp, d, ldd, total, st);
  else
    run_logp_grad_t<bf16>(x, stats, dlogp, d, ldd, total, st);
}

}  // namespace

extern "C" {

int sketch_token_logp(const sk_logits *x, float *logp, float *stats, void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK || x->rows == 0) return rc;
  if (!logp) return train_fail(SK_EINVAL, "NULL argument");
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  run_logp(x, logp, stats, nullptr, (hipStream_t)stream);
  return train_launched();
}

int sketch_token_logp_grad(const sk_logits *x, const float *stats, const float *dlogp, void *dlogits, int64_t ld_out,
                           void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK || x->rows == 0) return rc;
  if (!stats || !dlogp || !dlogits) return train_fail(SK_EINVAL, "NULL argument");
  if ((rc = check_out(x, dlogits, ld_out)) != SK_OK) return rc;
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  run_logp_grad(x, stats, dlogp, dlogits, ld_out, PairTotal(), (hipStream_t)stream);
  return train_launched();
}

int sketch_policy_loss(const sk_logits *x, const float *old_logp, const float *advantages, const float *weights,
                       const float *ref_logp, float clip_low, float clip_high, float kl_coef, float *loss, float *logp,
                       float *token_loss, void *dlogits, int64_t ld_out, void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK) return rc;
  if (!(clip_low >= 0.0f) || !(clip_high >= 0.0f)) return train_fail(SK_EINVAL, "clip bounds must be >= 0");
  if (!std::isfinite(kl_coef)) return train_fail(SK_EINVAL, "kl_coef must be finite");
  if (!loss) return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && (!old_logp || !advantages || !weights || !logp || !token_loss))
    return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && kl_coef != 0.0f && !ref_logp) return train_fail(SK_EINVAL, "kl_coef needs ref_logp");
  if ((rc = check_out(x, dlogits, ld_out)) != SK_OK) return rc;
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  const Rows r = rows_of(x);
  const Policy p{old_logp, advantages, weights, ref_logp, 1.0f - clip_low, 1.0f + clip_high, kl_coef};
  if (x->rows) {
    if (x->dtype == SK_F32)
      run_policy_t<float>(x, p, logp, token_loss, dlogits, ld_out, st);
    else
      run_policy_t<bf16>(x, p, logp, token_loss, dlogits, ld_out, st);
  }
  // one workgroup: four waves are done sooner with few rows (61: 1.8 us), sixteen with many (8192: 4.8 us)
  if (x->rows <= 1024)
    hipLaunchKernelGGL(k_policy_total<256>, dim3(1), dim3(256), 0, st, r, x->rows, weights, token_loss, loss);
  else
    hipLaunchKernelGGL(k_policy_total<1024>, dim3(1), dim3(1024), 0, st, r, x->rows, weights, token_loss, loss);
  return train_launched();
}

int64_t sketch_preference_work_bytes(int64_t rows) { return rows < 1 ? 0 : 16 * rows; }

int sketch_preference_loss(const sk_logits *x, const void *offsets, sk_index offsets_index, int64_t pairs,
                           const float *ref_logp, float beta, float smoothing, int32_t average, float *loss,
                           float *seq_logp, float *pair_loss, void *dlogits, int64_t ld_out, void *work,
                           int64_t work_bytes, void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK) return rc;
  if (offsets_index != SK_I32 && offsets_index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (pairs < 1) return train_fail(SK_EINVAL, "need at least one pair");
  if (pairs > (1 << 22)) return train_fail(SK_EUNSUPPORTED, "more than 2^22 pairs");  // a grid below 2^32 threads
  if (!std::isfinite(beta)) return train_fail(SK_EINVAL, "beta must be finite");
  if (!(smoothing >= 0.0f && smoothing <= 1.0f)) return train_fail(SK_EINVAL, "smoothing must be in [0, 1]");
  if (!offsets || !loss || !seq_logp || !pair_loss) return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && (!ref_logp || !work)) return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && work_bytes < sketch_preference_work_bytes(x->rows))
    return train_fail(SK_EINVAL, "work is smaller than sketch_preference_work_bytes");
  if ((rc = check_out(x, dlogits, ld_out)) != SK_OK) return rc;
  TrainGuard guard(x->device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  float *stats = (float *)work, *logp = stats + 2 * x->rows, *rowc = logp + x->rows;
  const Pairs p{offsets, (int32_t)offsets_index, average, pairs, x->rows, ref_logp, beta, smoothing};
  if (x->rows) run_logp(x, logp, stats, rowc, st);
  hipLaunchKernelGGL(k_pair, dim3((unsigned)pairs), dim3(512), 0, st, rows_of(x), p, logp, rowc, seq_logp, pair_loss);
  if (x->rows && dlogits)
    run_logp_grad(x, stats, rowc, dlogits, ld_out, PairTotal{pair_loss, pairs, loss}, st);
  else
    hipLaunchKernelGGL(k_pair_total, dim3(1), dim3(256), 0, st, pair_loss, pairs, loss);
  return train_launched();
}

}  // extern "C"
