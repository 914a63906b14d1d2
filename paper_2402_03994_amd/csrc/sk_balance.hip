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
// thousand tokens (one workgroup does all three then), by memory above.
#include <algorithm>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kThreads = 512;
constexpr int kMaxBlocks = 256;

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
  float *rate;  // coef E / n
  int64_t per;  // tokens of a workgroup
};

template <int L>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}
template <int L>
__device__ __forceinline__ float group_add(float v) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// A row's probabilities by L lanes; lane `at` holds columns (c L + at) 8 + 0 .. 7.
template <typename T, int L, int C>
struct Row {
  float p[C][8];
  __device__ __forceinline__ void softmax(const T *x, int experts, int at) {
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = (c * L + at) * 8;
      if (e + 8 <= experts) {
#pragma unroll
        for (int i = 0; i < 8; i += Vec<T>::N) {
          const u32x4 v = Vec<T>::load(x + e + i);
#pragma unroll
          for (int j = 0; j < Vec<T>::N; ++j) p[c][i + j] = Vec<T>::get(v, j);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[c][i] = e + i < experts ? to_f32(x[e + i]) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, p[c][i]);
    }
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.0f;
    float z = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[c][i] = entry_exp<float>(p[c][i] - m, Power{kLog2e, kLog2eLow});
        z += p[c][i];
      }
    z = group_add<L>(z);
    const float r = z == 0.0f ? 0.0f : 1.0f / z;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) p[c][i] *= r;
  }
};

__device__ __forceinline__ int64_t id_at(const Balance &a, int64_t i) {
  return a.index == SK_I64 ? ((const int64_t *)a.ids)[i] : ((const int32_t *)a.ids)[i];
}
// whether a token has an id; COUNT: its ids are counted
template <int L, bool COUNT>
__device__ __forceinline__ bool token_live(const Balance &a, int64_t t, int at, int *counts) {
  int any = 0;
  for (int j = at; j < a.k; j += L) {
    const int64_t id = id_at(a, t * a.k + j);
    if (id >= 0 && id < a.experts) {
      any = 1;
      if (COUNT) atomicAdd(counts + id, 1);
    }
  }
#pragma unroll
  for (int d = 1; d < L; d <<= 1) any |= __shfl_xor(any, d, 64);
  return any != 0;
}

template <int L, int C>
struct Shape {
  static constexpr int W = L * C * 8;           // columns
  static constexpr int G = kThreads / L;        // rows at a time
};

// Sums of workgroup b's tokens into its part of the workspace.
template <typename T, int L, int C>
__device__ __forceinline__ void count_part(const Balance &a, int b, float *sums, int *counts, int *tokens) {
  using S = Shape<L, C>;
  const int tid = threadIdx.x, at = tid & (L - 1), lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e < a.experts; e += kThreads) counts[e] = 0;
  if (tid == 0) *tokens = 0;
  __syncthreads();
  float sum[C][8] = {};
  int live = 0;
  const int64_t t0 = b * a.per, t1 = t0 + a.per < a.tokens ? t0 + a.per : a.tokens;
  for (int64_t t = t0 + tid / L; t - tid / L < t1; t += S::G) {
    Row<T, L, C> r;
    const bool in = t < t1 && token_live<L, true>(a, t < t1 ? t : t0, at, counts);
    if (in) {
      r.softmax((const T *)a.x + t * a.ld, a.experts, at);
      ++live;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[c][i] += r.p[c][i];
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
    a.part[(int64_t)b * a.experts + e] = s;
    a.count[(int64_t)b * a.experts + e] = counts[e];
  }
  if (tid == 0) a.tokens_of[b] = *tokens;
}

// counts, mean probabilities, loss, f and the gradient's factor from `blocks` parts; one workgroup
__device__ __forceinline__ void total(const Balance &a, int blocks, double *lds) {
  const int tid = threadIdx.x;
  int mine = 0;
  for (int b = tid; b < blocks; b += kThreads) mine += a.tokens_of[b];
  const double n = block_all<kThreads / 64>((double)mine, OpAdd(), lds);
  __syncthreads();
  double loss = 0.0;
  for (int e = tid; e < a.experts; e += kThreads) {
    double s = 0.0;
    int64_t c = 0;
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) {
      s += (double)a.part[(int64_t)b * a.experts + e];
      c += a.count[(int64_t)b * a.experts + e];
    }
    const double p = n > 0 ? s / n : 0.0, f = n > 0 ? (double)c / (n * a.k) : 0.0;
    a.counts[e] = c;
    a.probs[e] = (float)p;
    a.f[e] = (float)f;
    loss += f * p;
  }
  loss = block_all<kThreads / 64>(loss, OpAdd(), lds);
  if (tid == 0) {
    *a.loss = (float)((double)a.coef * a.experts * loss);
    *a.rate = n > 0 ? (float)((double)a.coef * a.experts / n) : 0.0f;
  }
}

// gradient rows from t0 on, `step` apart
template <typename T, int L, int C>
__device__ __forceinline__ void grad_part(const Balance &a, int64_t t0, int64_t step) {
  const int at = threadIdx.x & (L - 1);
  const float rate = *a.rate;
  float f[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = (c * L + at) * 8 + i;
      f[c][i] = e < a.experts ? a.f[e] : 0.0f;
    }
  for (int64_t t = t0; t < a.tokens; t += step) {
    T *d = (T *)a.d + t * a.ld_out;
    Row<T, L, C> r;
    if (token_live<L, false>(a, t, at, nullptr)) {
      r.softmax((const T *)a.x + t * a.ld, a.experts, at);
      float s = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s += r.p[c][i] * f[c][i];
      s = group_add<L>(s);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) r.p[c][i] *= rate * (f[c][i] - s);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) r.p[c][i] = 0.0f;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = (c * L + at) * 8;
      if (e + 8 <= a.experts) {
#pragma unroll
        for (int i = 0; i < 8; i += Vec<T>::N) Vec<T>::store(d + e + i, Vec<T>::pack(&r.p[c][i]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (e + i < a.experts) d[e + i] = from_f32<T>(r.p[c][i]);
      }
    }
  }
}

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_count(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  count_part<T, L, C>(a, blockIdx.x, sums, counts, &tokens);
}

__global__ __launch_bounds__(kThreads) void k_total(Balance a, int blocks) {
  __shared__ double lds[kThreads / 64];
  total(a, blocks, lds);
}

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_grad(Balance a) {
  grad_part<T, L, C>(a, (int64_t)blockIdx.x * Shape<L, C>::G + threadIdx.x / L, (int64_t)gridDim.x * Shape<L, C>::G);
}

template <typename T, int L, int C>
__global__ __launch_bounds__(kThreads) void k_all(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  __shared__ double lds[kThreads / 64];
  count_part<T, L, C>(a, 0, sums, counts, &tokens);
  __syncthreads();
  total(a, 1, lds);
  __syncthreads();
  if (a.d) grad_part<T, L, C>(a, threadIdx.x / L, Shape<L, C>::G);
}

template <typename T, int L, int C>
void run(Balance a, hipStream_t st) {
  constexpr int G = Shape<L, C>::G;
  if (a.tokens <= G) {
    a.per = a.tokens;
    hipLaunchKernelGGL((k_all<T, L, C>), dim3(1), dim3(kThreads), 0, st, a);
    return;
  }
  const int64_t blocks = std::min<int64_t>(kMaxBlocks, (a.tokens + G - 1) / G);
  a.per = (a.tokens + blocks - 1) / blocks;
  hipLaunchKernelGGL((k_count<T, L, C>), dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(k_total, dim3(1), dim3(kThreads), 0, st, a, (int)blocks);
  if (a.d)
    hipLaunchKernelGGL((k_grad<T, L, C>), dim3((unsigned)std::min<int64_t>(1024, (a.tokens + G - 1) / G)), dim3(kThreads), 0, st,
                       a);
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

int64_t sketch_balance_work_bytes(int64_t experts) { return experts < 1 ? 0 : 4 * (2 * kMaxBlocks + 1) * experts + 4 * kMaxBlocks + 256; }

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
  float *w = (float *)work;
  Balance a{logits, ids, tokens, ld, (int32_t)experts, (int32_t)k, (int32_t)index, coef, loss, probs, counts, dlogits, ld_out,
            w, (int *)(w + kMaxBlocks * experts), (int *)(w + 2 * kMaxBlocks * experts),
            w + 2 * kMaxBlocks * experts + kMaxBlocks, w + (2 * kMaxBlocks + 1) * experts + kMaxBlocks, 0};
  if (dtype == SK_F32)
    run_t<float>(a, (hipStream_t)stream);
  else
    run_t<bf16>(a, (hipStream_t)stream);
  return train_launched();
}

}  // extern "C"
