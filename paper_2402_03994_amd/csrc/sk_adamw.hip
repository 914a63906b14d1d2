// sk_adamw.hip -- AdamW over a list of parameter tensors, with moments in 32
// or in 8 bits (C ABI of include/sketch_train.h).
//
// The tensors are cut into chunks of 4096 elements, one workgroup each, by a
// table made at creation, so that one launch covers up to 128 tensors (their
// addresses travel in the kernel's arguments).  A thread owns four consecutive
// elements at a time and 16 lanes a 64-element block, whose largest moment is
// found within the lanes' row.
#include <cmath>
#include <vector>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kAdamChunk = 4096;
constexpr int kAdamPtrs = 128;  // tensors per launch
constexpr uint32_t ST_ADAMW = SK_STREAM_ADAMW, ST_ADAMW_P = SK_STREAM_ADAMW_P;

struct AdamTensor {
  int64_t n, at;  // elements, first element of its moments
  float decay;
};
struct AdamChunk {
  int32_t tensor, pad;
  int64_t e0;
};
struct AdamPtrs {
  void *p[kAdamPtrs];
  const void *g[kAdamPtrs];
  float *master[kAdamPtrs];
};
struct AdamStep {
  float b1, c1, b2, c2;  // c = 1 - b
  float lr_wd, rate, root, eps;  // lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t step;
  Key key;
  const float *scale;
};

// four consecutive elements from e on, `live` of them valid
template <typename T>
__device__ __forceinline__ void load4(const T *p, int64_t e, int live, float v[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < live ? to_f32(p[e + i]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store4(T *p, int64_t e, int live, const float v[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < live) p[e + i] = from_f32<T>(v[i]);
}

// the largest of the 16 lanes of a row
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, d, 16);
    v = v > o ? v : o;
  }
  return v;
}

// Codes of four values (of a 64-element block spread over 16 lanes) and the block's exponent byte.  TOP: the largest
// exponent field, 15 with a sign bit (m), 31 without (v).
template <int TOP>
__device__ __forceinline__ uint32_t encode4(const float x[4], const uint32_t dither[4], uint32_t &eb) {
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    big = big > a ? big : a;
  }
  big = row_max(big);
  if (big >= 0x7F800000u) {  // an infinity or NaN: the block stands for NaNs
    eb = 255;
    return 0;
  }
  eb = (big + 0x0FFFFFu) >> 23;
  // a carry to the infinities' exponent (values above 1.875 * 2^127) is left to 255 as well
  if (eb == 255) return 0;
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t y = __float_as_uint(ldexpf(fabsf(x[i]), TOP - (int)eb));
    uint32_t c = (y + ((dither[i] << 4) | 8u)) >> 20;
    if (TOP == 15) c |= (__float_as_uint(x[i]) >> 24) & 0x80u;
    out |= c << (8 * i);
  }
  return out;
}

template <int TOP>
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t eb, float x[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = (codes >> (8 * i)) & 0xFFu;
    float y = ldexpf(__uint_as_float((TOP == 15 ? c & 0x7Fu : c) << 20), (int)eb - TOP);
    if (TOP == 15) y = __uint_as_float(__float_as_uint(y) | ((c & 0x80u) << 24));
    x[i] = eb == 255 ? NAN : y;
  }
}

template <typename P, typename G, int STATE, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(const AdamTensor *__restrict__ tensors,
                                               const AdamChunk *__restrict__ chunks, int first, AdamPtrs ptrs,
                                               AdamStep s, void *__restrict__ mp, void *__restrict__ vp,
                                               uint8_t *__restrict__ mexp, uint8_t *__restrict__ vexp) {
#pragma clang fp contract(off)
  const float scale = s.scale ? *s.scale : 1.0f;
  if (!(fabsf(scale) < INFINITY)) return;
  const AdamChunk ck = chunks[blockIdx.x];
  const AdamTensor t = tensors[ck.tensor];
  const int slot = ck.tensor - first;
  P *p = (P *)ptrs.p[slot];
  const G *g = (const G *)ptrs.g[slot];
  float *master = MASTER ? ptrs.master[slot] : nullptr;
  const float shrink = s.lr_wd * t.decay;
  for (int it = 0; it < kAdamChunk / 1024; ++it) {
    const int64_t e = ck.e0 + it * 1024 + 4 * threadIdx.x;
    if (e >= ((t.n + 63) & ~63ll)) break;  // whole blocks, so whole rows of lanes
    const int live = t.n - e < 4 ? (t.n - e > 0 ? (int)(t.n - e) : 0) : 4;
    float gv[4], pv[4], m[4], v[4];
    load4(g, e, live, gv);
    if (MASTER)
      load4(master, e, live, pv);
    else
      load4((const P *)p, e, live, pv);
    const int64_t at = t.at + e;
    if (STATE == SK_ADAMW_F32) {
      *(float4 *)m = *(const float4 *)((const float *)mp + at);
      *(float4 *)v = *(const float4 *)((const float *)vp + at);
    } else {
      decode4<15>(*(const uint32_t *)((const uint8_t *)mp + at), mexp[at >> 6], m);
      decode4<31>(*(const uint32_t *)((const uint8_t *)vp + at), vexp[at >> 6], v);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float gi = gv[i] * scale;
      const float ma = m[i] * s.b1, mb = gi * s.c1;
      m[i] = ma + mb;
      const float gg = gi * gi;
      const float va = v[i] * s.b2, vb = gg * s.c2;
      v[i] = va + vb;
      // the change is formed first, so that the parameter is rounded once
      const float change = s.rate * (m[i] / (sqrtf(v[i]) * s.root + s.eps));
      pv[i] -= shrink * pv[i] + change;
    }
    if (STATE == SK_ADAMW_F32) {
      *(float4 *)((float *)mp + at) = *(const float4 *)m;
      *(float4 *)((float *)vp + at) = *(const float4 *)v;
    } else {
      const W4 w = philox((uint64_t)(uint32_t)(e >> 2) | ((uint64_t)s.step << 32), (uint32_t)ck.tensor, ST_ADAMW,
                          s.key);
      uint32_t dm[4], dv[4], eb;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dm[i] = w.w[i] >> 16;
        dv[i] = w.w[i] & 0xFFFFu;
      }
      const uint32_t cm = encode4<15>(m, dm, eb);
      *(uint32_t *)((uint8_t *)mp + at) = cm;
      if ((threadIdx.x & 15) == 0) mexp[at >> 6] = (uint8_t)eb;
      const uint32_t cv = encode4<31>(v, dv, eb);
      *(uint32_t *)((uint8_t *)vp + at) = cv;
      if ((threadIdx.x & 15) == 0) vexp[at >> 6] = (uint8_t)eb;
    }
    if (MASTER) store4(master, e, live, pv);
    if (sizeof(P) == 2 && !MASTER) {
      const W4 w = philox((uint64_t)(uint32_t)(e >> 3) | ((uint64_t)s.step << 32), (uint32_t)ck.tensor, ST_ADAMW_P,
                          s.key);
      const bool hi = (e >> 2) & 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t word = i < 2 ? (hi ? w.w[2] : w.w[0]) : (hi ? w.w[3] : w.w[1]);
        const uint32_t u = (i & 1) ? word >> 16 : word & 0xFFFFu;
        const uint32_t b = __float_as_uint(pv[i]);
        if ((b & 0x7FFFFFFFu) < 0x7F800000u) pv[i] = __uint_as_float((b + u) & 0xFFFF0000u);
      }
    }
    store4(p, e, live, pv);
  }
}

template <typename G>
__global__ __launch_bounds__(256) void k_adamw_norm(const AdamTensor *__restrict__ tensors,
                                                    const AdamChunk *__restrict__ chunks, int first, AdamPtrs ptrs,
                                                    double *__restrict__ part) {
  __shared__ double lds[4];
  const AdamChunk ck = chunks[blockIdx.x];
  const AdamTensor t = tensors[ck.tensor];
  const G *g = (const G *)ptrs.g[ck.tensor - first];
  double s = 0.0;
  for (int it = 0; it < kAdamChunk / 1024; ++it) {
    const int64_t e = ck.e0 + it * 1024 + 4 * threadIdx.x;
    const int live = t.n - e < 4 ? (t.n - e > 0 ? (int)(t.n - e) : 0) : 4;
    float gv[4];
    load4(g, e, live, gv);
#pragma unroll
    for (int i = 0; i < 4; ++i) s += (double)gv[i] * gv[i];
  }
  s = block_all<4>(s, OpAdd(), lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm and the scale of the gradients: NaN where the norm is not finite, so that the step changes nothing.
__global__ __launch_bounds__(1024) void k_adamw_scale(const double *__restrict__ part, int64_t n,
                                                      const float *__restrict__ grad_scale, float max_norm,
                                                      float *__restrict__ norm, float *__restrict__ scale) {
  __shared__ double lds[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_all<16>(s, OpAdd(), lds);
  if (threadIdx.x == 0) {
    const float gs = grad_scale ? *grad_scale : 1.0f;
    const float nm = (float)(fabs((double)gs) * sqrt(s));
    if (norm) *norm = nm;
    *scale = nm < INFINITY ? gs * fminf(1.0f, max_norm / (nm + 1e-6f)) : NAN;
  }
}

__global__ __launch_bounds__(256) void k_adamw_moments(int64_t groups, const uint32_t *__restrict__ m,
                                                       const uint8_t *__restrict__ mexp,
                                                       const uint32_t *__restrict__ v,
                                                       const uint8_t *__restrict__ vexp, float4 *__restrict__ mo,
                                                       float4 *__restrict__ vo) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= groups) return;
  float x[4];
  decode4<15>(m[i], mexp[i >> 4], x);
  mo[i] = make_float4(x[0], x[1], x[2], x[3]);
  decode4<31>(v[i], vexp[i >> 4], x);
  vo[i] = make_float4(x[0], x[1], x[2], x[3]);
}

}  // namespace

struct sk_adamw {
  int device = 0;
  sk_adamw_state state = SK_ADAMW_F32;
  Key key{};
  int n_tensors = 0;
  int64_t elems = 0, n_chunks = 0;
  std::vector<int64_t> numel, first_chunk;  // first chunk of each tensor, and the end
  AdamTensor *d_tensors = nullptr;
  AdamChunk *d_chunks = nullptr;
  double *d_part = nullptr;
  float *d_scale = nullptr;
};

namespace {

void free_adamw(sk_adamw *h) {
  for (void *p : {(void *)h->d_tensors, (void *)h->d_chunks, (void *)h->d_part, (void *)h->d_scale})
    if (p) (void)hipFree(p);
  delete h;
}

template <typename P, typename G>
void launch_adamw(int state, bool master, dim3 grid, hipStream_t st, const AdamTensor *t, const AdamChunk *c, int first,
                  const AdamPtrs &ptrs, const AdamStep &s, const sk_adamw_step *a) {
#define SK_ADAMW(STATE, MASTER)                                                                                 \
  hipLaunchKernelGGL((k_adamw<P, G, STATE, MASTER>), grid, dim3(256), 0, st, t, c, first, ptrs, s, a->m, a->v, \
                     a->m_exp, a->v_exp)
  if (state == SK_ADAMW_F32) {
    if (master)
      SK_ADAMW(SK_ADAMW_F32, true);
    else
      SK_ADAMW(SK_ADAMW_F32, false);
  } else {
    if (master)
      SK_ADAMW(SK_ADAMW_8BIT, true);
    else
      SK_ADAMW(SK_ADAMW_8BIT, false);
  }
#undef SK_ADAMW
}

}  // namespace

extern "C" {

int sketch_adamw_create(const int64_t *numel, const float *decay, int32_t n_tensors, sk_adamw_state state,
                        uint64_t seed, int32_t device, sk_adamw **out) try {
  if (!out) return train_fail(SK_EINVAL, "out is NULL");
  *out = nullptr;
  if (!numel || n_tensors < 1) return train_fail(SK_EINVAL, "need at least one tensor");
  if (state != SK_ADAMW_F32 && state != SK_ADAMW_8BIT) return train_fail(SK_EINVAL, "unknown state type");
  for (int l = 0; l < n_tensors; ++l) {
    if (numel[l] < 1 || numel[l] >= (1ll << 34))
      return train_fail(SK_EINVAL, "a tensor must have 1 to 2^34 - 1 elements");
    if (decay && !std::isfinite(decay[l])) return train_fail(SK_EINVAL, "decay must be finite");
  }
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || device < 0 || device >= ndev)
    return train_fail(SK_EINVAL, "device out of range");
  std::vector<AdamTensor> tensors;
  std::vector<AdamChunk> chunks;
  sk_adamw *h = new sk_adamw();
  try {
    h->device = device;
    h->state = state;
    h->key = make_key(seed);
    h->n_tensors = n_tensors;
    for (int l = 0; l < n_tensors; ++l) {
      h->numel.push_back(numel[l]);
      h->first_chunk.push_back((int64_t)chunks.size());
      tensors.push_back(AdamTensor{numel[l], h->elems, decay ? decay[l] : 1.0f});
      h->elems += (numel[l] + 63) / 64 * 64;
      for (int64_t e = 0; e < numel[l]; e += kAdamChunk) chunks.push_back(AdamChunk{l, 0, e});
    }
    h->n_chunks = (int64_t)chunks.size();
    h->first_chunk.push_back(h->n_chunks);
  } catch (...) {
    delete h;
    throw;
  }
  TrainGuard guard(device);
  if (hipMalloc((void **)&h->d_tensors, sizeof(AdamTensor) * tensors.size()) != hipSuccess ||
      hipMalloc((void **)&h->d_chunks, sizeof(AdamChunk) * chunks.size()) != hipSuccess ||
      hipMalloc((void **)&h->d_part, sizeof(double) * chunks.size()) != hipSuccess ||
      hipMalloc((void **)&h->d_scale, sizeof(float)) != hipSuccess) {
    (void)hipGetLastError();
    free_adamw(h);
    return train_fail(SK_ENOMEM, "hipMalloc failed");
  }
  if (hipMemcpy(h->d_tensors, tensors.data(), sizeof(AdamTensor) * tensors.size(), hipMemcpyHostToDevice) !=
          hipSuccess ||
      hipMemcpy(h->d_chunks, chunks.data(), sizeof(AdamChunk) * chunks.size(), hipMemcpyHostToDevice) != hipSuccess) {
    free_adamw(h);
    return train_fail(SK_EHIP, "hipMemcpy of the tables failed");
  }
  *out = h;
  return SK_OK;
} catch (const std::bad_alloc &) {
  return train_fail(SK_ENOMEM, "out of memory");
}

int64_t sketch_adamw_state_elems(const sk_adamw *h) { return h ? h->elems : 0; }

int sketch_adamw_apply(sk_adamw *h, const sk_adamw_step *a, void *const *params, sk_dtype pdtype,
                       const void *const *grads, sk_dtype gdtype, float *const *masters, void *stream) {
  if (!h || !a || !params || !grads || !a->m || !a->v) return train_fail(SK_EINVAL, "NULL argument");
  if (pdtype != SK_F32 && pdtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown parameter dtype");
  if (gdtype != SK_F32 && gdtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown gradient dtype");
  if (h->state == SK_ADAMW_8BIT && (!a->m_exp || !a->v_exp))
    return train_fail(SK_EINVAL, "moments in 8 bits need their exponents");
  if (masters && pdtype == SK_F32) return train_fail(SK_EINVAL, "fp32 parameters take no masters");
  if (a->step < 1 || a->step > (int64_t)UINT32_MAX) return train_fail(SK_EINVAL, "step must be in [1, 2^32)");
  if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0))
    return train_fail(SK_EINVAL, "betas must be in [0, 1)");
  if (!std::isfinite(a->lr) || !std::isfinite(a->weight_decay) || !(a->eps >= 0.0) || !std::isfinite(a->eps))
    return train_fail(SK_EINVAL, "lr and weight_decay must be finite, eps finite and >= 0");
  if (!(a->max_norm >= 0.0)) return train_fail(SK_EINVAL, "max_norm must be >= 0");
  for (int l = 0; l < h->n_tensors; ++l)
    if (!params[l] || !grads[l] || (masters && !masters[l])) return train_fail(SK_EINVAL, "NULL tensor pointer");
  TrainGuard guard(h->device);
  hipStream_t st = (hipStream_t)stream;
  AdamStep s;
  s.b1 = (float)a->beta1;
  s.c1 = (float)(1.0 - a->beta1);
  s.b2 = (float)a->beta2;
  s.c2 = (float)(1.0 - a->beta2);
  s.lr_wd = (float)(a->lr * a->weight_decay);
  s.rate = (float)(a->lr / (1.0 - std::pow(a->beta1, (double)a->step)));
  s.root = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, (double)a->step)));
  s.eps = (float)a->eps;
  s.step = (uint32_t)a->step;
  s.key = h->key;
  s.scale = a->max_norm > 0.0 ? h->d_scale : a->grad_scale;
  for (int pass = a->max_norm > 0.0 ? 0 : 1; pass < 2; ++pass) {
    for (int l0 = 0; l0 < h->n_tensors; l0 += kAdamPtrs) {
      const int l1 = std::min(l0 + kAdamPtrs, h->n_tensors);
      AdamPtrs ptrs;
      for (int l = l0; l < l1; ++l) {
        ptrs.p[l - l0] = params[l];
        ptrs.g[l - l0] = grads[l];
        ptrs.master[l - l0] = masters ? masters[l] : nullptr;
      }
      const int64_t c0 = h->first_chunk[l0];
      const dim3 grid((unsigned)(h->first_chunk[l1] - c0));
      const AdamChunk *ck = h->d_chunks + c0;
      if (pass == 0) {
        if (gdtype == SK_F32)
          hipLaunchKernelGGL((k_adamw_norm<float>), grid, dim3(256), 0, st, h->d_tensors, ck, l0, ptrs, h->d_part + c0);
        else
          hipLaunchKernelGGL((k_adamw_norm<bf16>), grid, dim3(256), 0, st, h->d_tensors, ck, l0, ptrs, h->d_part + c0);
      } else if (pdtype == SK_F32 && gdtype == SK_F32) {
        launch_adamw<float, float>(h->state, false, grid, st, h->d_tensors, ck, l0, ptrs, s, a);
      } else if (pdtype == SK_F32) {
        launch_adamw<float, bf16>(h->state, false, grid, st, h->d_tensors, ck, l0, ptrs, s, a);
      } else if (gdtype == SK_F32) {
        launch_adamw<bf16, float>(h->state, masters != nullptr, grid, st, h->d_tensors, ck, l0, ptrs, s, a);
      } else {
        launch_adamw<bf16, bf16>(h->state, masters != nullptr, grid, st, h->d_tensors, ck, l0, ptrs, s, a);
      }
    }
    if (pass == 0)
      hipLaunchKernelGGL(k_adamw_scale, dim3(1), dim3(1024), 0, st, h->d_part, h->n_chunks, a->grad_scale,
                         (float)a->max_norm, a->norm, h->d_scale);
  }
  return train_launched();
}

int sketch_adamw_moments(sk_adamw *h, const uint8_t *m, const uint8_t *m_exp, const uint8_t *v, const uint8_t *v_exp,
                         float *m_out, float *v_out, void *stream) {
  if (!h || !m || !m_exp || !v || !v_exp || !m_out || !v_out) return train_fail(SK_EINVAL, "NULL argument");
  if (h->state != SK_ADAMW_8BIT) return train_fail(SK_EINVAL, "the moments of this handle are fp32");
  TrainGuard guard(h->device);
  const int64_t groups = h->elems / 4;
  hipLaunchKernelGGL(k_adamw_moments, dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, (hipStream_t)stream, groups,
                     (const uint32_t *)m, m_exp, (const uint32_t *)v, v_exp, (float4 *)m_out, (float4 *)v_out);
  return train_launched();
}

void sketch_adamw_destroy(sk_adamw *h) {
  if (!h) return;
  TrainGuard guard(h->device);
  (void)hipDeviceSynchronize();
  free_adamw(h);
}

}  // extern "C"
