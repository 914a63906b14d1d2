// sk_embed.hip -- embedding lookup and its gradient (C ABI of
// include/sketch_train.h).
#include "sk_train.h"

using namespace sk;

namespace {

__device__ __forceinline__ int64_t id_at(const void *ids, int index, int64_t t) {
  return index == SK_I64 ? ((const int64_t *)ids)[t] : ((const int32_t *)ids)[t];
}

template <typename W, typename O>
__global__ __launch_bounds__(256) void k_embed(const W *__restrict__ w, int64_t vocab, int64_t width, int64_t ld,
                                               const void *__restrict__ ids, int index, float scale,
                                               O *__restrict__ out) {
  const int64_t t = blockIdx.x, v = id_at(ids, index, t);
  const bool live = v >= 0 && v < vocab;
  for (int64_t c = threadIdx.x; c < width; c += 256)
    out[t * width + c] = from_f32<O>(live ? scale * to_f32(w[v * ld + c]) : 0.0f);
}

template <typename O>
__global__ __launch_bounds__(256) void k_eg_zero(O *__restrict__ out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    out[i] = from_f32<O>(0.0f);
}

// One workgroup per token: the first one of its id in the group adds up all of them in order.
template <typename G, typename O>
__global__ __launch_bounds__(256) void k_eg_sum(const G *__restrict__ dy, int64_t ld, const void *__restrict__ ids,
                                                int index, int64_t n, int64_t vocab, int64_t width, float scale,
                                                O *__restrict__ out, int accumulate) {
  __shared__ int found;
  __shared__ int match[256];
  const int64_t b = blockIdx.y, t = blockIdx.x, base = b * n, v = id_at(ids, index, base + t);
  if (v < 0 || v >= vocab) return;
  if (threadIdx.x == 0) found = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < t; i += 256)
    if (id_at(ids, index, base + i) == v) found = 1;
  __syncthreads();
  if (found) return;
  O *o = out + (b * vocab + v) * width;
  for (int64_t c0 = 0; c0 < width; c0 += 256) {
    const int64_t c = c0 + threadIdx.x;
    float sum = 0.0f;
    for (int64_t i0 = t; i0 < n; i0 += 256) {
      const int64_t i = i0 + threadIdx.x;
      __syncthreads();
      match[threadIdx.x] = i < n && id_at(ids, index, base + i) == v;
      __syncthreads();
      for (int k = 0; k < 256; ++k)
        if (match[k] && c < width) sum += to_f32(dy[(base + i0 + k) * ld + c]);
    }
    if (c < width) o[c] = from_f32<O>(scale * sum + (accumulate ? to_f32(o[c]) : 0.0f));
  }
}

template <typename W>
void run_embed(const void *w, int64_t vocab, int64_t width, int64_t ld, const void *ids, int index, int64_t n,
               float scale, void *out, sk_dtype od, hipStream_t st) {
  const dim3 g((unsigned)n), b(256);
  if (od == SK_F32)
    hipLaunchKernelGGL((k_embed<W, float>), g, b, 0, st, (const W *)w, vocab, width, ld, ids, index, scale,
                       (float *)out);
  else
    hipLaunchKernelGGL((k_embed<W, bf16>), g, b, 0, st, (const W *)w, vocab, width, ld, ids, index, scale,
                       (bf16 *)out);
}

template <typename G, typename O>
void run_eg(const void *dy, int64_t ld, const void *ids, int index, int64_t batch, int64_t n, int64_t vocab,
            int64_t width, float scale, O *out, int accumulate, hipStream_t st) {
  if (!accumulate)
    hipLaunchKernelGGL((k_eg_zero<O>), dim3(4096), dim3(256), 0, st, out, batch * vocab * width);
  if (n)
    hipLaunchKernelGGL((k_eg_sum<G, O>), dim3((unsigned)n, (unsigned)batch), dim3(256), 0, st, (const G *)dy, ld, ids,
                       index, n, vocab, width, scale, out, accumulate);
}

bool dtype_ok(int d) { return d == SK_F32 || d == SK_BF16; }

}  // namespace

extern "C" {

int sketch_embed(const void *weight, sk_dtype dtype, int64_t vocab, int64_t width, int64_t ld, const void *ids,
                 sk_index index, int64_t n, float scale, void *out, sk_dtype out_dtype, int32_t device, void *stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (vocab < 1 || width < 1 || n < 0 || ld < width)
    return train_fail(SK_EINVAL, "need vocab, width >= 1, n >= 0 and ld >= width");
  if (n > INT32_MAX) return train_fail(SK_EUNSUPPORTED, "more than 2^31 - 1 ids");
  if (n == 0) return SK_OK;
  if (!weight || !ids || !out) return train_fail(SK_EINVAL, "NULL argument");
  TrainGuard guard(device);
  if (dtype == SK_F32)
    run_embed<float>(weight, vocab, width, ld, ids, index, n, scale, out, out_dtype, (hipStream_t)stream);
  else
    run_embed<bf16>(weight, vocab, width, ld, ids, index, n, scale, out, out_dtype, (hipStream_t)stream);
  return train_launched();
}

int64_t sketch_embed_grad_work_bytes(int64_t batch, int64_t n, int64_t width) {
  if (batch < 1 || n < 0 || width < 1) return 0;
  return 256;
}

int sketch_embed_grad(const void *dy, sk_dtype dtype, int64_t ld, const void *ids, sk_index index, int64_t batch,
                      int64_t n, int64_t vocab, int64_t width, float scale, void *out, sk_dtype out_dtype,
                      int32_t accumulate, void *work, int64_t work_bytes, int32_t device, void *stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (batch < 1 || vocab < 1 || width < 1 || n < 0 || ld < width)
    return train_fail(SK_EINVAL, "need batch, vocab, width >= 1, n >= 0 and ld >= width");
  if (vocab > (1 << 20) || batch > (1 << 30) || n > (1 << 30) || batch * n > (1 << 30))
    return train_fail(SK_EUNSUPPORTED, "vocab above 2^20 or batch * n above 2^30");
  if (!out || (n && (!dy || !ids || !work))) return train_fail(SK_EINVAL, "NULL argument");
  if (n && work_bytes < sketch_embed_grad_work_bytes(batch, n, width))
    return train_fail(SK_EINVAL, "work is smaller than sketch_embed_grad_work_bytes");
  TrainGuard guard(device);
  hipStream_t st = (hipStream_t)stream;
  if (dtype == SK_F32 && out_dtype == SK_F32)
    run_eg<float>(dy, ld, ids, index, batch, n, vocab, width, scale, (float *)out, accumulate, st);
  else if (dtype == SK_F32)
    run_eg<float>(dy, ld, ids, index, batch, n, vocab, width, scale, (bf16 *)out, accumulate, st);
  else if (out_dtype == SK_F32)
    run_eg<bf16>(dy, ld, ids, index, batch, n, vocab, width, scale, (float *)out, accumulate, st);
  else
    run_eg<bf16>(dy, ld, ids, index, batch, n, vocab, width, scale, (bf16 *)out, accumulate, st);
  return train_launched();
}

}  // extern "C"
