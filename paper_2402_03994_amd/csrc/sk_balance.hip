// sk_balance.hip -- the balance loss of a router with its per-expert counts and its
// gradient at the router's logits (C ABI of include/sketch_train.h).
//
// With c_e the ids equal to e, n the tokens that have one, P_e the mean of their
// softmax, f_e = c_e / (n k):
//   loss = coef E sum_e f_e P_e,  dlogits_te = coef E / n p_te (f_e - sum_e' f_e' p_te').
// The gradient of any token needs all counts, so the logits are read twice:
// k_count sums probabilities (fp32, each thread its own columns) and counts (whole
// numbers, in LDS) of a run of tokens a workgroup, k_total joins the workgroups in
// their order (fp64), k_grad forms the softmax again.  A row is held by L lanes
// of eight columns each, as many rows in a wave as fit.  Bound by latency up to some
// thousand tokens (one workgroup does all three then), by memory above: 65536 x 256
// bf16, 8 ids, 36 us (3.0 TB/s of logits twice, ids and gradient; three launches).
#include <algorithm>
#include <type_traits>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kThreads = 512;
constexpr int kMaxBlocks = 512;

struct Balance {
  const void *x;
  const void *ids;
  int64_t tokens, ld;
  int32_t experts, k, index;
  float coef;
  float *loss, *probs;
  int64_t *counts;
  void *d;
  int64_t ld_out;
  // workspace: each workgroup's sums of probabilities, counts and tokens; f
  float *part;
  int *count;
  int *tokens_of;
  float *f;
  float *rate;    // coef E / n
  double *share;  // of 64 experts in the loss
  int64_t per;  // tokens of a workgroup
};

// op over the L lanes of a row, in every one of them: exchanges within 16 lanes cost one operation (65536 x 256 bf16, the
// three kernels: 45 us with shuffles through LDS, 37 us so)
template <int L, typename T, typename Op>
__device__ __forceinline__ T group_all(T v, Op op) {
  auto other = [](T x, auto ctrl) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  if (L >= 2) v = op(v, other(v, std::integral_constant<int, 0xB1>()));    // lane ^ 1
  if (L >= 4) v = op(v, other(v, std::integral_constant<int, 0x4E>()));    // lane ^ 2
  if (L >= 8) v = op(v, other(v, std::integral_constant<int, 0x141>()));   // the other four of eight
  if (L >= 16) v = op(v, other(v, std::integral_constant<int, 0x140>()));  // the other eight of sixteen
  if (L >= 32) v = op(v, __shfl_xor(v, 16, 64));
  if (L >= 64) v = op(v, __shfl_xor(v, 32, 64));
  return v;
}
struct OpOr {
  __device__ int operator()(int a, int b) const { return a | b; }
};

// A row's probabilities by L lanes; lane `at` holds columns (c L + at) 8 + 0 .. 7.
template <typename T, int L, int C>
struct Row {
  static constexpr int NV = 8 / Vec<T>::N;
  u32x4 raw[C][NV];
  float p[C][8];
  __device__ __forceinline__ void load(const T *x, int experts, int at) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = (c * L + at) * 8;
      if (e + 8 <= experts) {
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[c][v] = Vec<T>::load(x + e + v * Vec<T>::N);
      } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = e + i < experts ? to_f32(x[e + i]) : -INFINITY;
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[c][v] = Vec<T>::pack(f + v * Vec<T>::N);
      }
    }
  }
  __device__ __forceinline__ void softmax() {
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[c][i] = Vec<T>::get(raw[c][i / Vec<T>::N], i % Vec<T>::N);
        m = fmaxf(m, p[c][i]);
      }
    m = group_all<L>(m, OpMax());
    if (m == -INFINITY) m = 0.0f;
    float z = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[c][i] = entry_exp<T>(p[c][i] - m, Power{kLog2e, kLog2eLow});
        z += p[c][i];
      }
    z = group_all<L>(z, OpAdd());
    const float r = z == 0.0f ? 0.0f : 1.0f / z;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) p[c][i] *= r;
  }
};

__device__ __forceinline__ int id_at(const Balance &a, int64_t i) {
  const int64_t id = a.index == SK_I64 ? ((const int64_t *)a.ids)[i] : ((const int32_t *)a.ids)[i];
  return id >= 0 && id < a.experts ? (int)id : -1;
}
// whether a token has an id, from the first id that this lane has loaded; COUNT: its ids are counted
template <int L, bool COUNT>
__device__ __forceinline__ bool token_live(const Balance &a, int64_t t, int at, int id, int *counts) {
  int any = id >= 0;
  if (COUNT && id >= 0) atomicAdd(counts + id, 1);
  for (int j = at + L; j < a.k; j += L) {
    const int o = id_at(a, t * a.k + j);
    if (o >= 0) {
      any = 1;
      if (COUNT) atomicAdd(counts + o, 1);
    }
  }
  return group_all<L>(any, OpOr()) != 0;
}

template <int L, int C>
struct Shape {
  static constexpr int W = L * C * 8;     // columns
  static constexpr int G = kThreads / L;  // rows at a time
  static constexpr int U = C > 1 ? 1 : 4;   // rows of a thread whose loads are under way together
  static constexpr int UG = C > 1 ? 1 : 2;  // in the gradient
};

// Sums of the tokens t0 .. t1 - 1: probabilities in sums[e], counts in counts[e], how many in *tokens.
template <typename T, int L, int C>
__device__ __forceinline__ void count_part(const Balance &a, int64_t t0, int64_t t1, float *sums, int *counts, int *tokens) {
  using S = Shape<L, C>;
  const int tid = threadIdx.x, at = tid & (L - 1), lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e < a.experts; e += kThreads) counts[e] = 0;
  if (tid == 0) *tokens = 0;
  __syncthreads();
  float sum[C][8] = {};
  int live = 0;
  for (int64_t b = t0 + tid / L; b < t1; b += S::G * S::U) {  // the lanes of a row go together
    Row<T, L, C> r[S::U];
    int id[S::U];
    // a masked row's logits come too, and are left: waiting for its ids first would cost another trip to memory
#pragma unroll
    for (int u = 0; u < S::U; ++u) {
      const int64_t t = b + u * S::G;
      if (t < t1) {
        id[u] = at < a.k ? id_at(a, t * a.k + at) : -1;
        r[u].load((const T *)a.x + t * a.ld, a.experts, at);
      }
    }
#pragma unroll
    for (int u = 0; u < S::U; ++u) {
      const int64_t t = b + u * S::G;
      if (t < t1 && token_live<L, true>(a, t, at, id[u], counts)) {
        r[u].softmax();
        ++live;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[c][i] += r[u].p[c][i];
      }
    }
  }
  if (at == 0 && live) atomicAdd(tokens, live);
  // the groups of a wave, then the waves
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int d = L; d < 64; d <<= 1) sum[c][i] += __shfl_xor(sum[c][i], d, 64);
      if (lane < L) sums[wave * S::W + (c * L + at) * 8 + i] = sum[c][i];
    }
  __syncthreads();
  for (int e = tid; e < a.experts; e += kThreads) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += sums[w * S::W + e];
    sums[e] = s;
  }
}

// An expert's share of the loss from its sums over n tokens; writes its outputs and f.
__device__ __forceinline__ double finish(const Balance &a, int e, double s, int64_t c, double n) {
  const double p = n > 0 ? s / n : 0.0, f = n > 0 ? (double)c / (n * a.k) : 0.0;
  a.counts[e] = c;
  a.probs[e] = (float)p;
  a.f[e] = (float)f;
  return f * p;
}
__device__ __forceinline__ void finish_loss(const Balance &a, double loss) {
  *a.loss = (float)((double)a.coef * a.experts * loss);
}
__device__ __forceinline__ float rate_of(const Balance &a, double n) {
  return n > 0 ? (float)((double)a.coef * a.experts / n) : 0.0f;
}

// gradient rows from t0 on, `step` apart
template <typename T, int L, int C>
__device__ __forceinline__ void grad_part(const Balance &a, int64_t t0, int64_t step, float rate) {
  using S = Shape<L, C>;
  const int at = threadIdx.x & (L - 1);
  float f[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = (c * L + at) * 8 + i;
      f[c][i] = e < a.experts ? a.f[e] : 0.0f;
    }
  for (int64_t b = t0; b < a.tokens; b += step * S::UG) {
    Row<T, L, C> r[S::UG];
    int id[S::UG];
#pragma unroll
    for (int u = 0; u < S::UG; ++u) {
      const int64_t t = b + u * step;
      if (t < a.tokens) {
        id[u] = at < a.k ? id_at(a, t * a.k + at) : -1;
        r[u].load((const T *)a.x + t * a.ld, a.experts, at);
      }
    }
#pragma unroll
    for (int u = 0; u < S::UG; ++u) {
      const int64_t t = b + u * step;
      if (t >= a.tokens) continue;
      T *d = (T *)a.d + t * a.ld_out;
      if (token_live<L, false>(a, t, at, id[u], nullptr)) {
        r[u].softmax();
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) s += r[u].p[c][i] * f[c][i];
        s = group_all<L>(s, OpAdd());
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) r[u].p[c][i] *= rate * (f[c][i] - s);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) r[u].p[c][i] = 0.0f;
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = (c * L + at) * 8;
        if (e + 8 <= a.experts) {
#pragma unroll
          for (int i = 0; i < 8; i += Vec<T>::N) Vec<T>::store(d + e + i, Vec<T>::pack(&r[u].p[c][i]));
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (e + i < a.experts) d[e + i] = from_f32<T>(r[u].p[c][i]);
        }
      }
    }
  }
}

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_count(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  const int64_t t0 = blockIdx.x * a.per;
  count_part<T, L, C>(a, t0, t0 + a.per < a.tokens ? t0 + a.per : a.tokens, sums, counts, &tokens);
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    a.part[(int64_t)blockIdx.x * a.experts + e] = sums[e];
    a.count[(int64_t)blockIdx.x * a.experts + e] = counts[e];
  }
  if (threadIdx.x == 0) a.tokens_of[blockIdx.x] = tokens;
}

// Counts, mean probabilities, f and the experts' shares of the loss; 64 experts a workgroup, whose waves share the
// `blocks` parts.
__global__ __launch_bounds__(1024) void k_total(Balance a, int blocks) {
  __shared__ double lds[16], sums[16][64];
  __shared__ int counts[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
  int mine = 0;
  for (int b = threadIdx.x; b < blocks; b += 1024) mine += a.tokens_of[b];
  double s = 0.0;
  int c = 0;
  if (e < a.experts) {
#pragma unroll 8
    for (int b = wave; b < blocks; b += 16) {
      s += (double)a.part[(int64_t)b * a.experts + e];
      c += a.count[(int64_t)b * a.experts + e];
    }
  }
  sums[wave][lane] = s;
  counts[wave][lane] = c;
  const double n = block_all<16>((double)mine, OpAdd(), lds);
  if (wave) return;
  for (int w = 1; w < 16; ++w) {
    s += sums[w][lane];
    c += counts[w][lane];
  }
  const double loss = wave_all(e < a.experts ? finish(a, e, s, c, n) : 0.0, OpAdd());
  if (lane == 0) {
    a.share[blockIdx.x] = loss;
    if (blockIdx.x == 0) *a.rate = rate_of(a, n);
    if (gridDim.x == 1) finish_loss(a, loss);
  }
}

__device__ __forceinline__ void sum_shares(const Balance &a, int shares) {
  double loss = 0.0;
  for (int i = 0; i < shares; ++i) loss += a.share[i];
  finish_loss(a, loss);
}
__global__ void k_shares(Balance a, int shares) { sum_shares(a, shares); }

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_grad(Balance a, int shares) {
  if (shares > 1 && blockIdx.x == 0 && threadIdx.x == 0) sum_shares(a, shares);
  grad_part<T, L, C>(a, (int64_t)blockIdx.x * Shape<L, C>::G + threadIdx.x / L, (int64_t)gridDim.x * Shape<L, C>::G, *a.rate);
}

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_all(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  __shared__ double lds[kThreads / 64];
  count_part<T, L, C>(a, 0, a.tokens, sums, counts, &tokens);
  // *tokens and counts are complete behind the barrier inside
  const double n = tokens;
  double loss = 0.0;
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    loss += finish(a, e, sums[e], counts[e], n);
    sums[e] = n > 0 ? (float)((double)counts[e] / (n * a.k)) : 0.0f;
  }
  loss = block_all<kThreads / 64>(loss, OpAdd(), lds);
  if (threadIdx.x == 0) finish_loss(a, loss);
  if (!a.d) return;
  __syncthreads();
  a.f = sums;
  grad_part<T, L, C>(a, threadIdx.x / L, Shape<L, C>::G, rate_of(a, n));
}

template <typename T, int L, int C>
void run(Balance a, hipStream_t st) {
  constexpr int G = Shape<L, C>::G;
  if (a.tokens <= G) {
    hipLaunchKernelGGL((k_all<T, L, C>), dim3(1), dim3(kThreads), 0, st, a);
    return;
  }
  const int64_t blocks = std::min<int64_t>(kMaxBlocks, (a.tokens + G - 1) / G);
  const int shares = (a.experts + 63) / 64;
  a.per = (a.tokens + blocks - 1) / blocks;
  hipLaunchKernelGGL((k_count<T, L, C>), dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(k_total, dim3(shares), dim3(1024), 0, st, a, (int)blocks);
  if (a.d)
    hipLaunchKernelGGL((k_grad<T, L, C>), dim3((unsigned)std::min<int64_t>(1024, (a.tokens + G - 1) / G)), dim3(kThreads), 0, st,
                       a, shares);
  else if (shares > 1)
    hipLaunchKernelGGL(k_shares, dim3(1), dim3(1), 0, st, a, shares);
}

template <typename T>
void run_t(const Balance &a, hipStream_t st) {
  if (a.experts <= 8)
    run<T, 1, 1>(a, st);
  else if (a.experts <= 32)
    run<T, 4, 1>(a, st);
  else if (a.experts <= 64)
    run<T, 8, 1>(a, st);
  else if (a.experts <= 128)
    run<T, 16, 1>(a, st);
  else if (a.experts <= 256)
    run<T, 32, 1>(a, st);
  else if (a.experts <= 512)
    run<T, 64, 1>(a, st);
  else if (a.experts <= 1024)
    run<T, 64, 2>(a, st);
  else
    run<T, 64, 4>(a, st);
}

}  // namespace

extern "C" {

int64_t sketch_balance_work_bytes(int64_t experts) {
  return experts < 1 ? 0 : 8 * 32 + 4 * ((2 * kMaxBlocks + 1) * experts + kMaxBlocks + 1);
}

int sketch_balance_loss(const void *logits, sk_dtype dtype, int64_t tokens, int64_t experts, int64_t ld, const void *ids,
                        sk_index index, int64_t k, float coef, float *loss, int64_t *counts, float *probs, void *dlogits,
                        int64_t ld_out, void *work, int64_t work_bytes, int32_t device, void *stream) {
  if (dtype != SK_F32 && dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (tokens < 0 || experts < 1 || k < 1 || ld < experts || (dlogits && ld_out < experts))
    return train_fail(SK_EINVAL, "need tokens >= 0, experts >= 1, k >= 1 and row strides >= experts");
  if (!std::isfinite(coef)) return train_fail(SK_EINVAL, "coef must be finite");
  if (experts > 2048 || tokens > INT32_MAX || k > 1024 || tokens * k > INT32_MAX)
    return train_fail(SK_EUNSUPPORTED, "more than 2048 experts, 1024 ids a token or 2^31 - 1 ids");
  if (!loss || !counts || !probs || !work || (tokens && (!logits || !ids))) return train_fail(SK_EINVAL, "NULL argument");
  if (work_bytes < sketch_balance_work_bytes(experts))
    return train_fail(SK_EINVAL, "work is smaller than sketch_balance_work_bytes");
  if (dlogits && dlogits == logits && ld_out != ld) return train_fail(SK_EINVAL, "in place needs ld_out = ld");
  TrainGuard guard(device);
  if (!guard.ok) return train_no_device();
  // 32 doubles, then floats and ints
  float *part = (float *)((double *)work + 32), *count = part + kMaxBlocks * experts, *tokens_of = count + kMaxBlocks * experts,
        *f = tokens_of + kMaxBlocks, *rate = f + experts;
  const Balance a{logits, ids, tokens, ld, (int32_t)experts, (int32_t)k, (int32_t)index, coef, loss, probs, counts, dlogits,
                  ld_out, part, (int *)count, (int *)tokens_of, f, rate, (double *)work, 0};
  if (dtype == SK_F32)
    run_t<float>(a, (hipStream_t)stream);
  else
    run_t<bf16>(a, (hipStream_t)stream);
  return train_launched();
}

}  // extern "C"
