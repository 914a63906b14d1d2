// sk_loss.hip -- token log-probabilities, the clipped policy loss and the
// preference loss, with their gradients with respect to the logits (C ABI of
// include/sketch_train.h).
//
// A row x of logits enters through its largest entry m and z = sum_j
// exp(scale (x_j - m)): log p_t = scale (x_t - m) - log z, and every gradient is
// a number c of the row times scale (onehot - p).  The exponentials are at most
// 1, so a row whose entries are all the type's lowest value is the uniform
// distribution; a row of -inf alone has m taken as 0 and z = 0.
#include "sk_train.h"

using namespace sk;

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

struct Rows {
  const void *x;
  const void *targets;
  int64_t ld;
  int32_t vocab;
  int32_t index;
  float scale;
};

// the target of row t, -1 where it is masked
__device__ __forceinline__ int target_at(const Rows &r, int64_t t) {
  const int64_t v = r.index == SK_I64 ? ((const int64_t *)r.targets)[t] : ((const int32_t *)r.targets)[t];
  return v >= 0 && v < r.vocab ? (int)v : -1;
}

// (m, log z) of one row by a workgroup of 256
template <typename T>
__device__ __forceinline__ float2 row_stats(const T *x, int vocab, float scale, float *lds) {
  float m = -INFINITY;
  for (int j = threadIdx.x; j < vocab; j += 256) m = fmaxf(m, to_f32(x[j]));
  m = block_all<4>(m, OpMax(), lds);
  if (m == -INFINITY) m = 0.0f;
  float z = 0.0f;
  for (int j = threadIdx.x; j < vocab; j += 256) z += __builtin_amdgcn_exp2f((to_f32(x[j]) - m) * (scale * kLog2e));
  z = block_all<4>(z, OpAdd(), lds + 4);
  return make_float2(m, logf(z));
}

__device__ __forceinline__ float logp_of(float xt, float2 s, float scale) {
  return s.y == -INFINITY ? -INFINITY : (xt - s.x) * scale - s.y;
}

// row of c scale (onehot - p); zeros where c = 0 or the row is empty
template <typename T>
__device__ __forceinline__ void row_grad(const T *x, T *d, int vocab, float scale, float2 s, int target, float c) {
  const bool none = c == 0.0f || s.y == -INFINITY;
  for (int j = threadIdx.x; j < vocab; j += 256) {
    float g = 0.0f;
    if (!none) {
      const float p = __builtin_amdgcn_exp2f(((to_f32(x[j]) - s.x) * scale - s.y) * kLog2e);
      g = c * scale * ((j == target ? 1.0f : 0.0f) - p);
    }
    d[j] = from_f32<T>(g);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_logp(Rows r, float *__restrict__ logp, float2 *__restrict__ stats) {
  __shared__ float lds[8];
  const int64_t t = blockIdx.x;
  const int target = target_at(r, t);
  const T *x = (const T *)r.x + t * r.ld;
  float2 s = make_float2(0.0f, 0.0f);
  float lp = 0.0f;
  if (target >= 0) {
    s = row_stats(x, r.vocab, r.scale, lds);
    lp = logp_of(to_f32(x[target]), s, r.scale);
  }
  if (threadIdx.x == 0) {
    logp[t] = lp;
    if (stats) stats[t] = s;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_logp_grad(Rows r, const float2 *__restrict__ stats,
                                                   const float *__restrict__ dlogp, void *d, int64_t ldd) {
  const int64_t t = blockIdx.x;
  const int target = target_at(r, t);
  const float c = target >= 0 ? dlogp[t] : 0.0f;
  row_grad((const T *)r.x + t * r.ld, (T *)d + t * ldd, r.vocab, r.scale, stats[t], target, c);
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
    const float u = p.ref[t] - logp, e = expf(u);
    l += p.kl * (e - u - 1.0f);
    d += p.kl * (1.0f - e);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_policy(Rows r, Policy p, float *__restrict__ logp, float *__restrict__ loss_t,
                                                void *d, int64_t ldd) {
  __shared__ float lds[8];
  const int64_t t = blockIdx.x;
  const int target = target_at(r, t);
  const float w = target >= 0 ? p.weights[t] : 0.0f;
  const T *x = (const T *)r.x + t * r.ld;
  float2 s = make_float2(0.0f, 0.0f);
  float lp = 0.0f, l = 0.0f, c = 0.0f;
  if (w != 0.0f) {
    s = row_stats(x, r.vocab, r.scale, lds);
    lp = logp_of(to_f32(x[target]), s, r.scale);
    policy_token(p, t, lp, l, c);
    c *= w;
  }
  __syncthreads();  // x[target] is read before the row may be overwritten
  if (threadIdx.x == 0) {
    logp[t] = lp;
    loss_t[t] = l;
  }
  if (d) row_grad(x, (T *)d + t * ldd, r.vocab, r.scale, s, target, c);
}

// sum_t w_t l_t over the unmasked rows, in fp64 in a fixed order
__global__ __launch_bounds__(1024) void k_policy_total(Rows r, int64_t rows, const float *__restrict__ w,
                                                       const float *__restrict__ l, float *__restrict__ loss) {
  __shared__ double lds[16];
  double s = 0.0;
  for (int64_t t = threadIdx.x; t < rows; t += 1024)
    if (target_at(r, t) >= 0 && w[t] != 0.0f) s += (double)w[t] * l[t];
  s = block_all<16>(s, OpAdd(), lds);
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

// One workgroup per pair: both texts' sums, the pair's loss, and each row's factor d loss / d logp.
__global__ __launch_bounds__(256) void k_pair(Rows r, Pairs p, const float *__restrict__ logp,
                                              float *__restrict__ rowc, float *__restrict__ seq,
                                              float *__restrict__ pair_loss) {
  __shared__ double lds[2][12];
  const int64_t pair = blockIdx.x;
  double gap[2];
  float share[2];
  for (int h = 0; h < 2; ++h) {
    const int64_t a = offset_at(p, 2 * pair + h), b = offset_at(p, 2 * pair + h + 1);
    double s = 0.0, g = 0.0, n = 0.0;
    for (int64_t t = a + threadIdx.x; t < b; t += 256)
      if (target_at(r, t) >= 0) {
        s += logp[t];
        g += (double)logp[t] - p.ref[t];
        n += 1.0;
      }
    s = block_all<4>(s, OpAdd(), lds[h]);
    g = block_all<4>(g, OpAdd(), lds[h] + 4);
    n = block_all<4>(n, OpAdd(), lds[h] + 8);
    share[h] = p.average ? (float)(1.0 / fmax(n, 1.0)) : 1.0f;
    gap[h] = p.average ? g / fmax(n, 1.0) : g;
    if (threadIdx.x == 0) seq[2 * pair + h] = (float)(p.average ? s / fmax(n, 1.0) : s);
  }
  const double d = (double)p.beta * (gap[0] - gap[1]), eps = p.smoothing;
  const double loss = (eps < 1.0 ? (1.0 - eps) * softplus(-d) : 0.0) + (eps > 0.0 ? eps * softplus(d) : 0.0);
  const double c = -(double)p.beta / (double)p.pairs * ((1.0 - eps) / (1.0 + exp(d)) - eps / (1.0 + exp(-d)));
  if (threadIdx.x == 0) pair_loss[pair] = (float)loss;
  for (int h = 0; h < 2; ++h) {
    const int64_t a = offset_at(p, 2 * pair + h), b = offset_at(p, 2 * pair + h + 1);
    const float ch = (float)(h ? -c : c) * share[h];
    for (int64_t t = a + threadIdx.x; t < b; t += 256) rowc[t] = ch;
  }
}

// Rows outside all texts: before the first offset and from the last one on.
__global__ __launch_bounds__(256) void k_pair_rest(Pairs p, float *__restrict__ rowc) {
  const int64_t a = offset_at(p, 0), b = offset_at(p, 2 * p.pairs);
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t < p.rows && (t < a || t >= b)) rowc[t] = 0.0f;
}

__global__ __launch_bounds__(256) void k_pair_total(const float *__restrict__ pair_loss, int64_t pairs,
                                                    float *__restrict__ loss) {
  __shared__ double lds[4];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < pairs; i += 256) s += pair_loss[i];
  s = block_all<4>(s, OpAdd(), lds);
  if (threadIdx.x == 0) *loss = (float)(s / (double)pairs);
}

int check_logits(const sk_logits *x) {
  if (!x) return train_fail(SK_EINVAL, "NULL argument");
  if (x->dtype != SK_F32 && x->dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (x->index != SK_I32 && x->index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (x->rows < 0 || x->vocab < 1 || x->ld < x->vocab)
    return train_fail(SK_EINVAL, "need rows >= 0, vocab >= 1 and ld >= vocab");
  if (!(x->scale > 0.0f) || !std::isfinite(x->scale)) return train_fail(SK_EINVAL, "scale must be positive and finite");
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
  return Rows{x->data, x->targets, x->ld, (int32_t)x->vocab, (int32_t)x->index, x->scale};
}

void run_logp(const sk_logits *x, float *logp, float *stats, hipStream_t st) {
  const dim3 g((unsigned)x->rows), b(256);
  if (x->dtype == SK_F32)
    hipLaunchKernelGGL((k_logp<float>), g, b, 0, st, rows_of(x), logp, (float2 *)stats);
  else
    hipLaunchKernelGGL((k_logp<bf16>), g, b, 0, st, rows_of(x), logp, (float2 *)stats);
}

void run_logp_grad(const sk_logits *x, const float *stats, const float *dlogp, void *d, int64_t ldd, hipStream_t st) {
  const dim3 g((unsigned)x->rows), b(256);
  if (x->dtype == SK_F32)
    hipLaunchKernelGGL((k_logp_grad<float>), g, b, 0, st, rows_of(x), (const float2 *)stats, dlogp, d, ldd);
  else
    hipLaunchKernelGGL((k_logp_grad<bf16>), g, b, 0, st, rows_of(x), (const float2 *)stats, dlogp, d, ldd);
}

}  // namespace

extern "C" {

int sketch_token_logp(const sk_logits *x, float *logp, float *stats, void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK || x->rows == 0) return rc;
  if (!logp) return train_fail(SK_EINVAL, "NULL argument");
  TrainGuard guard(x->device);
  run_logp(x, logp, stats, (hipStream_t)stream);
  return train_launched();
}

int sketch_token_logp_grad(const sk_logits *x, const float *stats, const float *dlogp, void *dlogits, int64_t ld_out,
                           void *stream) {
  int rc = check_logits(x);
  if (rc != SK_OK || x->rows == 0) return rc;
  if (!stats || !dlogp || !dlogits) return train_fail(SK_EINVAL, "NULL argument");
  if ((rc = check_out(x, dlogits, ld_out)) != SK_OK) return rc;
  TrainGuard guard(x->device);
  run_logp_grad(x, stats, dlogp, dlogits, ld_out, (hipStream_t)stream);
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
  hipStream_t st = (hipStream_t)stream;
  const Rows r = rows_of(x);
  const Policy p{old_logp, advantages, weights, ref_logp, 1.0f - clip_low, 1.0f + clip_high, kl_coef};
  if (x->rows) {
    const dim3 g((unsigned)x->rows), b(256);
    if (x->dtype == SK_F32)
      hipLaunchKernelGGL((k_policy<float>), g, b, 0, st, r, p, logp, token_loss, dlogits, ld_out);
    else
      hipLaunchKernelGGL((k_policy<bf16>), g, b, 0, st, r, p, logp, token_loss, dlogits, ld_out);
  }
  hipLaunchKernelGGL(k_policy_total, dim3(1), dim3(1024), 0, st, r, x->rows, weights, token_loss, loss);
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
  if (pairs > INT32_MAX) return train_fail(SK_EUNSUPPORTED, "more than 2^31 - 1 pairs");
  if (!std::isfinite(beta)) return train_fail(SK_EINVAL, "beta must be finite");
  if (!(smoothing >= 0.0f && smoothing <= 1.0f)) return train_fail(SK_EINVAL, "smoothing must be in [0, 1]");
  if (!offsets || !loss || !seq_logp || !pair_loss) return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && (!ref_logp || !work)) return train_fail(SK_EINVAL, "NULL argument");
  if (x->rows && work_bytes < sketch_preference_work_bytes(x->rows))
    return train_fail(SK_EINVAL, "work is smaller than sketch_preference_work_bytes");
  if ((rc = check_out(x, dlogits, ld_out)) != SK_OK) return rc;
  TrainGuard guard(x->device);
  hipStream_t st = (hipStream_t)stream;
  float *stats = (float *)work, *logp = stats + 2 * x->rows, *rowc = logp + x->rows;
  const Pairs p{offsets, (int32_t)offsets_index, average, pairs, x->rows, ref_logp, beta, smoothing};
  if (x->rows) run_logp(x, logp, stats, st);
  hipLaunchKernelGGL(k_pair, dim3((unsigned)pairs), dim3(256), 0, st, rows_of(x), p, logp, rowc, seq_logp, pair_loss);
  hipLaunchKernelGGL(k_pair_total, dim3(1), dim3(256), 0, st, pair_loss, pairs, loss);
  if (x->rows && dlogits) {
    hipLaunchKernelGGL(k_pair_rest, dim3((unsigned)((x->rows + 255) / 256)), dim3(256), 0, st, p, rowc);
    run_logp_grad(x, stats, rowc, dlogits, ld_out, st);
  }
  return train_launched();
}

}  // extern "C"
