// sk_balance.hip -- the balance loss of a router with its per-expert counts and its
// gradient at the router's logits (C ABI of include/sketch_train.h).
//
// With c_e the ids equal to e, n the tokens that have one, P_e the mean of their
// softmax, f_e = c_e / (n k):
//   loss = coef E sum_e f_e P_e,  dlogits_te = coef E / n p_te (f_e - sum_e' f_e' p_te').
// The gradient of any token needs all counts, and these need the ids alone: k_ids
// counts them (whole numbers, in LDS; of few ids each workgroup of k_rows counts all
// by itself, and without gradient its own), k_rows forms each softmax once, for the
// sums of probabilities (fp32, each thread its own columns) and for the gradient, and
// k_total joins the workgroups' sums in their order (fp64).  A row is held by L lanes
// of eight columns C times, as many rows in a wave as fit; up to 512 / L tokens k_all
// does all three.  Bound by latency up to some thousand tokens, above by the vector
// operations beside memory: 65536 x 256 bf16, 8 ids, 29 us with the call (reading the
// logits once for the sums and once for the gradient: 37 us).
#include <algorithm>
#include <type_traits>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kThreads = 512;
constexpr int kMaxBlocks = 512;
constexpr int kMaxExperts = 2048;
// Workgroups of k_ids at most, whose counts each of k_rows adds up: half as many of long rows (20000 x 2048: 73 and 59 us;
// 65536 x 256: 31 and 33 us).
constexpr int kParts = 64, kLongRow = 512;
// Ids up to which each workgroup of k_rows counts them itself (60 experts, 4 ids: 5000 tokens 16.9 and 20.2 us, 8000 tokens
// 21.5 and 19.8 us).
constexpr int64_t kOwnIds = 24576;

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
  // workspace: sums of probabilities of k_rows' workgroups; counts and tokens of k_ids' (without gradient: of k_rows');
  // tokens
  float *part;
  int *count;
  int *tokens_of;
  int *n;
  double *share;  // of k_rows' workgroups in the loss (without gradient: of k_total's)
  int64_t per;    // tokens of a workgroup
  int parts;      // workgroups of k_ids, 0: there is none
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
struct OpCount {
  __device__ int operator()(int a, int b) const { return a + b; }
};

// A row's probabilities by L lanes; lane `at` holds columns (c L + at) 8 + 0 .. 7.
template <typename T, int L, int C>
struct Row {
  static constexpr int NV = 8 / Vec<T>::N;
  u32x4 raw[C][NV];
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
  __device__ __forceinline__ void softmax(float (&p)[C][8]) const {
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

__device__ __forceinline__ void no_counts(const Balance &a, int *counts, int *tokens) {
  for (int e = threadIdx.x; e < a.experts; e += kThreads) counts[e] = 0;
  if (threadIdx.x == 0) *tokens = 0;
  __syncthreads();
}

// Counts of the ids of tokens t0 .. t1 - 1 in counts[e], how many of these have one in *tokens; a thread a token.
__device__ __forceinline__ void count_ids(const Balance &a, int64_t t0, int64_t t1, int *counts, int *tokens) {
  no_counts(a, counts, tokens);
  int live = 0;
  for (int64_t t = t0 + threadIdx.x; t < t1; t += kThreads) {
    bool any = false;
#pragma unroll 8
    for (int j = 0; j < a.k; ++j) {
      const int id = id_at(a, t * a.k + j);
      if (id >= 0) {
        any = true;
        atomicAdd(counts + id, 1);
      }
    }
    live += any;
  }
  live = group_all<64>(live, OpCount());
  if ((threadIdx.x & 63) == 0 && live) atomicAdd(tokens, live);
  __syncthreads();
}

template <int L, int C>
struct Shape {
  static constexpr int W = L * C * 8;     // columns
  static constexpr int G = kThreads / L;  // rows at a time
  static constexpr int U = C > 2 ? 1 : C > 1 ? 2 : 4;  // rows of a thread whose loads are under way together
};

// f of an expert, and P
__device__ __forceinline__ double share_of(const Balance &a, int count, int n) {
  return n > 0 ? (double)count / ((double)n * a.k) : 0.0;
}
__device__ __forceinline__ double mean_of(double sum, int n) { return n > 0 ? sum / n : 0.0; }
__device__ __forceinline__ float rate_of(const Balance &a, int n) {
  return n > 0 ? (float)((double)a.coef * a.experts / n) : 0.0f;
}

// Sums of the probabilities of tokens t0 .. t1 - 1 in sums[e], and their gradients from the call's counts and tokens; without
// gradient those of these tokens are added to counts and tokens.
template <typename T, int L, int C, bool GRAD>
__device__ __forceinline__ void rows_part(const Balance &a, int64_t t0, int64_t t1, int *counts, int *tokens, float *sums) {
  using S = Shape<L, C>;
  const int tid = threadIdx.x, at = tid & (L - 1), lane = tid & 63, wave = tid >> 6;
  const int n = GRAD ? *tokens : 0;
  const float rate = rate_of(a, n);
  int found = 0;
  float f[C][8], sum[C][8] = {};
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = (c * L + at) * 8 + i;
      f[c][i] = GRAD && e < a.experts ? (float)share_of(a, counts[e], n) : 0.0f;
    }
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
      if (t >= t1) continue;
      const bool live = token_live<L, !GRAD>(a, t, at, id[u], counts);
      float p[C][8] = {};
      if (live) {
        ++found;
        r[u].softmax(p);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[c][i] += p[c][i];
      }
      if (!GRAD) continue;
      T *d = (T *)a.d + t * a.ld_out;
      float s = 0.0f;
      if (live) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) s += p[c][i] * f[c][i];
        s = group_all<L>(s, OpAdd());
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[c][i] = live ? p[c][i] * (rate * (f[c][i] - s)) : 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = (c * L + at) * 8;
        if (e + 8 <= a.experts) {
#pragma unroll
          for (int i = 0; i < 8; i += Vec<T>::N) Vec<T>::store(d + e + i, Vec<T>::pack(&p[c][i]));
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (e + i < a.experts) d[e + i] = from_f32<T>(p[c][i]);
        }
      }
    }
  }
  if (!GRAD && at == 0 && found) atomicAdd(tokens, found);
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

__device__ __forceinline__ void finish_loss(const Balance &a, double loss) {
  *a.loss = (float)((double)a.coef * a.experts * loss);
}

__global__ __launch_bounds__(kThreads) void k_ids(Balance a, int64_t per) {
  __shared__ int counts[kMaxExperts];
  __shared__ int tokens;
  const int64_t t0 = blockIdx.x * per;
  count_ids(a, t0, t0 + per < a.tokens ? t0 + per : a.tokens, counts, &tokens);
  for (int e = threadIdx.x; e < a.experts; e += kThreads) a.count[(int64_t)blockIdx.x * a.experts + e] = counts[e];
  if (threadIdx.x == 0) a.tokens_of[blockIdx.x] = tokens;
}

template <typename T, int L, int C, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_rows(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  __shared__ double lds[kThreads / 64];
  if (!GRAD) {
    no_counts(a, counts, &tokens);
  } else if (a.parts) {
    if (threadIdx.x < 64) {
      const int n = group_all<64>((int)threadIdx.x < a.parts ? a.tokens_of[threadIdx.x] : 0, OpCount());
      if (threadIdx.x == 0) tokens = n;
    }
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      int c = 0;
#pragma unroll 32
      for (int b = 0; b < a.parts; ++b) c += a.count[(int64_t)b * a.experts + e];
      counts[e] = c;
    }
    __syncthreads();
  } else {
    count_ids(a, 0, a.tokens, counts, &tokens);
  }
  const int64_t t0 = blockIdx.x * a.per;
  rows_part<T, L, C, GRAD>(a, t0, t0 + a.per < a.tokens ? t0 + a.per : a.tokens, counts, &tokens, sums);
  // counts and tokens are complete behind the barrier inside
  double loss = 0.0;
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    a.part[(int64_t)blockIdx.x * a.experts + e] = sums[e];
    if (!GRAD) a.count[(int64_t)blockIdx.x * a.experts + e] = counts[e];
    if (GRAD && blockIdx.x == 0) a.counts[e] = counts[e];
    if (GRAD) loss += share_of(a, counts[e], tokens) * mean_of(sums[e], tokens);
  }
  if (GRAD) loss = block_all<kThreads / 64>(loss, OpAdd(), lds);
  if (threadIdx.x == 0) {
    if (GRAD)
      a.share[blockIdx.x] = loss;
    else
      a.tokens_of[blockIdx.x] = tokens;
    if (GRAD && blockIdx.x == 0) *a.n = tokens;
  }
}

// Mean probabilities, and without gradient counts; 64 experts a workgroup, whose waves share the `blocks` parts.  The loss,
// unless k_shares adds up the workgroups' shares.
template <bool GRAD>
__global__ __launch_bounds__(1024) void k_total(Balance a, int blocks) {
  __shared__ double sums[16][64], lds[16];
  __shared__ int counts[16][64], tokens[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
  double s = 0.0;
  int c = 0, n = 0;
  if (e < a.experts) {
#pragma unroll 8
    for (int b = wave; b < blocks; b += 16) {
      s += (double)a.part[(int64_t)b * a.experts + e];
      if (!GRAD) c += a.count[(int64_t)b * a.experts + e];
    }
  }
  if (!GRAD) n = group_all<64>((int)threadIdx.x < blocks ? a.tokens_of[threadIdx.x] : 0, OpCount());
  sums[wave][lane] = s;
  counts[wave][lane] = c;
  if (lane == 0) tokens[wave] = n;
  double loss = 0.0;
  if (GRAD && blockIdx.x == 0)
    loss = block_all<16>((int)threadIdx.x < blocks ? a.share[threadIdx.x] : 0.0, OpAdd(), lds);
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < 16; ++w) {
    s += sums[w][lane];
    c += counts[w][lane];
    n += tokens[w];
  }
  if (GRAD) n = *a.n;
  if (e < a.experts) {
    a.probs[e] = (float)mean_of(s, n);
    if (!GRAD) a.counts[e] = c;
  }
  if (!GRAD) {
    loss = wave_all(e < a.experts ? share_of(a, c, n) * mean_of(s, n) : 0.0, OpAdd());
    if (lane == 0) a.share[blockIdx.x] = loss;
  }
  if (lane == 0 && (GRAD ? blockIdx.x == 0 : gridDim.x == 1)) finish_loss(a, loss);
}

__global__ void k_shares(Balance a, int shares) {
  double loss = 0.0;
  for (int i = 0; i < shares; ++i) loss += a.share[i];
  finish_loss(a, loss);
}

template <typename T, int L, int C, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_all(Balance a) {
  __shared__ float sums[kThreads / 64 * Shape<L, C>::W];
  __shared__ int counts[Shape<L, C>::W];
  __shared__ int tokens;
  __shared__ double lds[kThreads / 64];
  if (GRAD)
    count_ids(a, 0, a.tokens, counts, &tokens);
  else
    no_counts(a, counts, &tokens);
  rows_part<T, L, C, GRAD>(a, 0, a.tokens, counts, &tokens, sums);
  double loss = 0.0;
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    a.counts[e] = counts[e];
    a.probs[e] = (float)mean_of(sums[e], tokens);
    loss += share_of(a, counts[e], tokens) * mean_of(sums[e], tokens);
  }
  loss = block_all<kThreads / 64>(loss, OpAdd(), lds);
  if (threadIdx.x == 0) finish_loss(a, loss);
}

template <typename T, int L, int C, bool GRAD>
void run_rows(Balance a, hipStream_t st) {
  constexpr int G = Shape<L, C>::G;
  if (a.tokens <= G) {
    hipLaunchKernelGGL((k_all<T, L, C, GRAD>), dim3(1), dim3(kThreads), 0, st, a);
    return;
  }
  if (GRAD && a.tokens * a.k > kOwnIds) {
    const int64_t most = a.experts > kLongRow ? kParts / 2 : kParts;
    const int64_t per = std::max<int64_t>(kThreads, (a.tokens + most - 1) / most);
    a.parts = (int)((a.tokens + per - 1) / per);
    hipLaunchKernelGGL(k_ids, dim3((unsigned)a.parts), dim3(kThreads), 0, st, a, per);
  }
  const int64_t blocks = std::min<int64_t>(kMaxBlocks, (a.tokens + G - 1) / G);
  a.per = (a.tokens + blocks - 1) / blocks;
  hipLaunchKernelGGL((k_rows<T, L, C, GRAD>), dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
  const int shares = (a.experts + 63) / 64;
  hipLaunchKernelGGL(k_total<GRAD>, dim3(shares), dim3(1024), 0, st, a, (int)blocks);
  if (!GRAD && shares > 1) hipLaunchKernelGGL(k_shares, dim3(1), dim3(1), 0, st, a, shares);
}
template <typename T, int L, int C>
void run(const Balance &a, hipStream_t st) {
  a.d ? run_rows<T, L, C, true>(a, st) : run_rows<T, L, C, false>(a, st);
}

// Sixteen columns a lane where a row has many: half the exchanges (65536 x 256, 32 lanes of eight: 32.3 us, 31 us so).
template <typename T>
void run_t(const Balance &a, hipStream_t st) {
  if (a.experts <= 8)
    run<T, 1, 1>(a, st);
  else if (a.experts <= 32)
    run<T, 4, 1>(a, st);
  else if (a.experts <= 64)
    run<T, 8, 1>(a, st);
  else if (a.experts <= 128)
    run<T, 8, 2>(a, st);
  else if (a.experts <= 256)
    run<T, 16, 2>(a, st);
  else if (a.experts <= 512)
    run<T, 32, 2>(a, st);
  else if (a.experts <= 1024)
    run<T, 64, 2>(a, st);
  else
    run<T, 64, 4>(a, st);
}

}  // namespace

extern "C" {

int64_t sketch_balance_work_bytes(int64_t experts) {
  return experts < 1 ? 0 : 8 * kMaxBlocks + 4 * (2 * kMaxBlocks * experts + kMaxBlocks + 1);
}

int sketch_balance_loss(const void *logits, sk_dtype dtype, int64_t tokens, int64_t experts, int64_t ld, const void *ids,
                        sk_index index, int64_t k, float coef, float *loss, int64_t *counts, float *probs, void *dlogits,
                        int64_t ld_out, void *work, int64_t work_bytes, int32_t device, void *stream) {
  if (dtype != SK_F32 && dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (tokens < 0 || experts < 1 || k < 1 || ld < experts || (dlogits && ld_out < experts))
    return train_fail(SK_EINVAL, "need tokens >= 0, experts >= 1, k >= 1 and row strides >= experts");
  if (!std::isfinite(coef)) return train_fail(SK_EINVAL, "coef must be finite");
  if (experts > kMaxExperts || tokens > INT32_MAX || k > 1024 || tokens * k > INT32_MAX)
    return train_fail(SK_EUNSUPPORTED, "more than 2048 experts, 1024 ids a token or 2^31 - 1 ids");
  if (!loss || !counts || !probs || !work || (tokens && (!logits || !ids))) return train_fail(SK_EINVAL, "NULL argument");
  if (work_bytes < sketch_balance_work_bytes(experts))
    return train_fail(SK_EINVAL, "work is smaller than sketch_balance_work_bytes");
  if (dlogits && dlogits == logits && ld_out != ld) return train_fail(SK_EINVAL, "in place needs ld_out = ld");
  TrainGuard guard(device);
  if (!guard.ok) return train_no_device();
  float *part = (float *)((double *)work + kMaxBlocks);
  int *count = (int *)(part + kMaxBlocks * experts), *tokens_of = count + kMaxBlocks * experts, *n = tokens_of + kMaxBlocks;
  const Balance a{logits, ids, tokens, ld, (int32_t)experts, (int32_t)k, (int32_t)index, coef, loss, probs, counts, dlogits,
                  ld_out, part, count, tokens_of, n, (double *)work, 0, 0};
  if (dtype == SK_F32)
    run_t<float>(a, (hipStream_t)stream);
  else
    run_t<bf16>(a, (hipStream_t)stream);
  return train_launched();
}

}  // extern "C"
