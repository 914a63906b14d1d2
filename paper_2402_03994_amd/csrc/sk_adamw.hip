// sk_adamw.hip -- AdamW over a list of parameter tensors, with moments in 32
// or in 8 bits (C ABI of include/sketch_train.h).
//
// The tensors are cut into chunks of 4096 elements, one workgroup each, by a
// table made at creation, so that one launch covers up to 160 tensors (their
// addresses travel in the kernel's arguments).  A thread owns eight consecutive
// elements at a time (16-byte loads of bf16, one Philox block for its
// parameters and two for its moments) and eight lanes a 64-element block, whose
// largest moment they find among themselves.
//
// GPT-2 small, 124 million elements (medians of traced calls; calls in a row
// take 583 and 246 us):
//   fp32 moments, parameters and gradients: 629 us, bound by memory (28 bytes an
//   element, 5.5 TB/s; the vector units are busy for 22% of it).
//   8-bit moments, bf16 parameters and gradients: 271 us, bound by the vector
//   units, busy all the time with 68 instructions an element (random words,
//   square root, codes) beside 10 bytes (4.6 TB/s).
//   k_adamw_moments writes 8 bytes an element: 239 us, 5.2 TB/s.
//   k_adamw_norm reads the gradients once more: 127 us, 3.9 TB/s.
#include <cmath>
#include <vector>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kAdamChunk = 4096;
constexpr int kAdamPtrs = 160;  // tensors per launch: 3840 bytes of the 4 KB that arguments may take
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
  // a list of up to kFewChunks chunks: its norm's partial sums are added up here
  const double *part;
  int64_t n_part;
  float max_norm;
  float *norm;
};

constexpr int64_t kFewChunks = 256;

// The scale of the gradients from the sum of their squares: NaN where the norm is not finite, so that the step changes
// nothing.
__device__ __forceinline__ float clip_scale(double sum, float gs, float max_norm, float *norm) {
  const float nm = (float)(fabs((double)gs) * sqrt(sum));
  if (norm) *norm = nm;
  return nm < INFINITY ? gs * fminf(1.0f, max_norm / (nm + 1e-6f)) : NAN;
}

constexpr int kPer = 8;  // consecutive elements of a thread: a 64-element block is 8 lanes

// the kPer elements from e on, `live` of them valid (the others 0)
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t e, int live, float v[kPer]) {
  if (live == kPer) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int k = 0; k < kPer; k += N) {
      const u32x4 r = Vec<T>::load(p + e + k);
#pragma unroll
      for (int i = 0; i < N; ++i) v[k + i] = Vec<T>::get(r, i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = i < live ? to_f32(p[e + i]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t e, int live, const float v[kPer]) {
  if (live == kPer) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int k = 0; k < kPer; k += N) Vec<T>::store(p + e + k, Vec<T>::pack(v + k));
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i < live) p[e + i] = from_f32<T>(v[i]);
  }
}

// the largest among 8 neighbouring lanes: neighbours, pairs of a quad, the two quads
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  v = max_dpp<0xB1>(v);   // quad_perm [1, 0, 3, 2]
  v = max_dpp<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  return max_dpp<0x141>(v);  // row_half_mirror
}

// Codes of eight values (of a 64-element block spread over 8 lanes) and the block's exponent byte.  TOP: the largest
// exponent field, 15 with a sign bit (m), 31 without (v); dither: what is added below the codes.
template <int TOP>
__device__ __forceinline__ uint2 encode8(const float x[kPer], const uint32_t dither[kPer], uint32_t &eb) {
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    big = big > a ? big : a;
  }
  big = block_max(big);
  // an infinity or NaN: the block stands for NaNs; so it does where 2^E with E = 128 would be needed
  eb = (big + 0x0FFFFFu) >> 23;
  if (eb >= 255) {
    eb = 255;
    return make_uint2(0, 0);
  }
  uint32_t top[kPer];  // the codes in the highest byte
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t y = __float_as_uint(ldexpf(fabsf(x[i]), TOP - (int)eb));
    top[i] = (y + dither[i]) << 4;
    if (TOP == 15) top[i] = (top[i] & 0x7FFFFFFFu) | (__float_as_uint(x[i]) & 0x80000000u);
  }
  uint32_t out[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // v_perm_b32: bytes 0 .. 3 of the second operand, 4 .. 7 of the first
    const uint32_t lo = __builtin_amdgcn_perm(top[4 * i + 1], top[4 * i], 0x0C0C0703u);
    const uint32_t hi = __builtin_amdgcn_perm(top[4 * i + 3], top[4 * i + 2], 0x07030C0Cu);
    out[i] = lo | hi;
  }
  return make_uint2(out[0], out[1]);
}

// What eight codes stand for.  The block's 2^E comes in two factors (2^(127 - TOP) times a code is exact, and E may
// reach beyond either side of what one factor holds); the second is NaN for exponent byte 255.
template <int TOP>
__device__ __forceinline__ void decode8(uint2 codes, uint32_t eb, float x[kPer]) {
  const float unit = __uint_as_float((254u - TOP) << 23);
  const float block = __uint_as_float(eb == 255 ? 0x7FC00000u : eb == 0 ? 0x00400000u : eb << 23);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t w = i < 4 ? codes.x : codes.y;
    const int at = 8 * (i & 3);
    uint32_t y;
    if (TOP == 15)  // sign, then seven bits from bit 20
      y = (uint32_t)((int32_t)(w << (24 - at)) >> 4) & 0x87F00000u;
    else
      y = (at <= 20 ? w << (20 - at) : w >> (at - 20)) & 0x0FF00000u;
    x[i] = __uint_as_float(y) * unit * block;
  }
}

// m / (sqrt(v) root + eps), square root and quotient rounded correctly where the parameter is held in 32 bits (EXACT).
// Where it is about to be rounded at random to 8 bits, the hardware's square root and reciprocal serve (one unit in the
// last of 24 each, nothing for inputs below 2^-126), with an eps beside which root 2^-63 is nothing.  124 million
// elements, moments in 32 bits: 583 us exact and 588 us by the hardware's; in 8 bits, fp32 parameters and bf16
// gradients: 314 us, 299 us.
template <bool EXACT>
__device__ __forceinline__ float ratio(float m, float v, float root, float eps, bool tiny_eps) {
  if (EXACT || tiny_eps) return m / __builtin_fmaf(sqrtf(v), root, eps);
  return m * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_sqrtf(v), root, eps));
}

template <typename P, typename G, int STATE, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(const AdamTensor *__restrict__ tensors,
                                               const AdamChunk *__restrict__ chunks, int first, AdamPtrs ptrs,
                                               AdamStep s, void *__restrict__ mp, void *__restrict__ vp,
                                               uint8_t *__restrict__ mexp, uint8_t *__restrict__ vexp) {
#pragma clang fp contract(off)
  float scale = s.scale ? *s.scale : 1.0f;
  if (s.part) {  // in the order of the chunks, by every workgroup: one launch and one wait less than k_adamw_scale
    __shared__ double lds[4];
    const double sum = block_all<4>(threadIdx.x < s.n_part ? s.part[threadIdx.x] : 0.0, OpAdd(), lds);
    scale = clip_scale(sum, scale, s.max_norm, blockIdx.x == 0 && first == 0 && threadIdx.x == 0 ? s.norm : nullptr);
  }
  if (!(fabsf(scale) < INFINITY)) return;
  const AdamChunk ck = chunks[blockIdx.x];
  const AdamTensor t = tensors[ck.tensor];
  const int slot = ck.tensor - first;
  P *p = (P *)ptrs.p[slot];
  const G *g = (const G *)ptrs.g[slot];
  float *master = MASTER ? ptrs.master[slot] : nullptr;
  const float shrink = s.lr_wd * t.decay;
#pragma unroll
  for (int it = 0; it < kAdamChunk / (256 * kPer); ++it) {
    const int64_t e = ck.e0 + it * 256 * kPer + kPer * threadIdx.x;
    if (e >= ((t.n + 63) & ~63ll)) break;  // whole blocks, so whole groups of 8 lanes
    const int live = t.n - e < kPer ? (t.n - e > 0 ? (int)(t.n - e) : 0) : kPer;
    float gv[kPer], pv[kPer], m[kPer], v[kPer];
    load8(g, e, live, gv);
    if (MASTER)
      load8((const float *)master, e, live, pv);
    else
      load8((const P *)p, e, live, pv);
    const int64_t at = t.at + e;
    if (STATE == SK_ADAMW_F32) {
      load8((const float *)mp, at, kPer, m);
      load8((const float *)vp, at, kPer, v);
    } else {
      decode8<15>(*(const uint2 *)((const uint8_t *)mp + at), mexp[at >> 6], m);
      decode8<31>(*(const uint2 *)((const uint8_t *)vp + at), vexp[at >> 6], v);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float gi = gv[i] * scale;
      const float ma = m[i] * s.b1, mb = gi * s.c1;
      m[i] = ma + mb;
      const float gg = gi * gi;
      const float va = v[i] * s.b2, vb = gg * s.c2;
      v[i] = va + vb;
    }
    // the change is formed first, so that the parameter is rounded once
    const bool tiny_eps = s.eps < s.root * 0x1p-39f;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      pv[i] -= __builtin_fmaf(s.rate, ratio<sizeof(P) == 4 || MASTER>(m[i], v[i], s.root, s.eps, tiny_eps), shrink * pv[i]);
    if (STATE == SK_ADAMW_F32) {
      store8((float *)mp, at, kPer, m);
      store8((float *)vp, at, kPer, v);
    } else {
      uint32_t dm[kPer], dv[kPer], eb;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const W4 w = philox_at<true>((uint32_t)(e >> 2) + q, s.step, (uint32_t)ck.tensor, ST_ADAMW, s.key);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 16 u + 8
          dm[4 * q + i] = ((w.w[i] >> 12) & 0xFFFF0u) | 8u;
          dv[4 * q + i] = ((w.w[i] << 4) & 0xFFFF0u) | 8u;
        }
      }
      *(uint2 *)((uint8_t *)mp + at) = encode8<15>(m, dm, eb);
      if ((threadIdx.x & 7) == 0) mexp[at >> 6] = (uint8_t)eb;
      *(uint2 *)((uint8_t *)vp + at) = encode8<31>(v, dv, eb);
      if ((threadIdx.x & 7) == 0) vexp[at >> 6] = (uint8_t)eb;
    }
    if (MASTER) store8(master, e, live, pv);
    if (sizeof(P) == 2 && !MASTER) {
      // An infinity has nothing below its 16 bits and stays one.  A NaN may have all of its bits set, where u would carry
      // into the sign and beyond: eight values that hold one (four comparisons of two) are rounded apart.
      const W4 w = philox_at<true>((uint32_t)(e >> 3), s.step, (uint32_t)ck.tensor, ST_ADAMW_P, s.key);
      const bool nan = __builtin_isunordered(pv[0], pv[1]) || __builtin_isunordered(pv[2], pv[3]) ||
                       __builtin_isunordered(pv[4], pv[5]) || __builtin_isunordered(pv[6], pv[7]);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        uint32_t u = (i & 1) ? w.w[i >> 1] >> 16 : w.w[i >> 1] & 0xFFFFu;
        if (__builtin_expect(nan, 0)) u = pv[i] != pv[i] ? 0 : u;
        pv[i] = __uint_as_float((__float_as_uint(pv[i]) + u) & 0xFFFF0000u);
      }
    }
    store8(p, e, live, pv);
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
#pragma unroll
  for (int it = 0; it < kAdamChunk / (256 * kPer); ++it) {
    const int64_t e = ck.e0 + it * 256 * kPer + kPer * threadIdx.x;
    const int live = t.n - e < kPer ? (t.n - e > 0 ? (int)(t.n - e) : 0) : kPer;
    float gv[kPer];
    load8(g, e, live, gv);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s += (double)gv[i] * gv[i];
  }
  s = block_all<4>(s, OpAdd(), lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void k_adamw_scale(const double *__restrict__ part, int64_t n,
                                                      const float *__restrict__ grad_scale, float max_norm,
                                                      float *__restrict__ norm, float *__restrict__ scale) {
  __shared__ double lds[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_all<16>(s, OpAdd(), lds);
  if (threadIdx.x == 0) *scale = clip_scale(s, grad_scale ? *grad_scale : 1.0f, max_norm, norm);
}

__global__ __launch_bounds__(256) void k_adamw_moments(int64_t groups, const uint2 *__restrict__ m,
                                                       const uint8_t *__restrict__ mexp, const uint2 *__restrict__ v,
                                                       const uint8_t *__restrict__ vexp, float *__restrict__ mo,
                                                       float *__restrict__ vo) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= groups) return;
  float x[kPer], y[kPer];
  decode8<15>(m[i], mexp[i >> 3], x);
  decode8<31>(v[i], vexp[i >> 3], y);
  store8(mo, i * kPer, kPer, x);
  store8(vo, i * kPer, kPer, y);
}

}  // namespace

struct sk_adamw {
  int device = 0;
  sk_adamw_state state = SK_ADAMW_F32;
  Key key{};
  int n_tensors = 0;
  int64_t elems = 0, n_chunks = 0;
  std::vector<int64_t> numel, first_chunk;  // first chunk of each tensor, and the end
  // one allocation: scale, partial sums of the norm, tensors, chunks
  void *d_block = nullptr;
  AdamTensor *d_tensors = nullptr;
  AdamChunk *d_chunks = nullptr;
  double *d_part = nullptr;
  float *d_scale = nullptr;
};

namespace {

void free_adamw(sk_adamw *h) {
  if (h->d_block) (void)hipFree(h->d_block);
  delete h;
}

// MASTER goes with bf16 parameters alone
template <typename P, typename G>
void launch_adamw(int state, bool master, dim3 grid, hipStream_t st, const AdamTensor *t, const AdamChunk *c, int first,
                  const AdamPtrs &ptrs, const AdamStep &s, const sk_adamw_step *a) {
#define SK_ADAMW(STATE, MASTER)                                                                                 \
  hipLaunchKernelGGL((k_adamw<P, G, STATE, MASTER>), grid, dim3(256), 0, st, t, c, first, ptrs, s, a->m, a->v, \
                     a->m_exp, a->v_exp)
  if constexpr (sizeof(P) == 2) {
    if (master && state == SK_ADAMW_F32) SK_ADAMW(SK_ADAMW_F32, true);
    if (master && state != SK_ADAMW_F32) SK_ADAMW(SK_ADAMW_8BIT, true);
    if (master) return;
  }
  if (state == SK_ADAMW_F32)
    SK_ADAMW(SK_ADAMW_F32, false);
  else
    SK_ADAMW(SK_ADAMW_8BIT, false);
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
  std::vector<char> tables;  // tensors, then chunks
  sk_adamw *h = new sk_adamw();
  try {
    h->device = device;
    h->state = state;
    h->key = make_key(seed);
    h->n_tensors = n_tensors;
    for (int l = 0; l < n_tensors; ++l) {
      h->numel.push_back(numel[l]);
      h->first_chunk.push_back(h->n_chunks);
      h->n_chunks += (numel[l] + kAdamChunk - 1) / kAdamChunk;
    }
    h->first_chunk.push_back(h->n_chunks);
    if (h->n_chunks >= (1 << 24)) {  // a grid of 2^32 threads
      delete h;
      return train_fail(SK_EUNSUPPORTED, "more than 2^36 elements");
    }
    tables.resize(sizeof(AdamTensor) * n_tensors + sizeof(AdamChunk) * h->n_chunks);
  } catch (...) {
    delete h;
    throw;
  }
  AdamTensor *tensors = (AdamTensor *)tables.data();
  AdamChunk *chunks = (AdamChunk *)(tensors + n_tensors);
  for (int l = 0; l < n_tensors; ++l) {
    tensors[l] = AdamTensor{numel[l], h->elems, decay ? decay[l] : 1.0f};
    h->elems += (numel[l] + 63) / 64 * 64;
    for (int64_t e = 0; e < numel[l]; e += kAdamChunk) *chunks++ = AdamChunk{l, 0, e};
  }
  TrainGuard guard(device);
  const size_t at_tensors = 16 + sizeof(double) * h->n_chunks;
  if (hipMalloc(&h->d_block, at_tensors + tables.size()) != hipSuccess) {
    (void)hipGetLastError();
    h->d_block = nullptr;
    free_adamw(h);
    return train_fail(SK_ENOMEM, "hipMalloc failed");
  }
  h->d_scale = (float *)h->d_block;
  h->d_part = (double *)((char *)h->d_block + 16);
  h->d_tensors = (AdamTensor *)((char *)h->d_block + at_tensors);
  h->d_chunks = (AdamChunk *)(h->d_tensors + n_tensors);
  if (hipMemcpy(h->d_tensors, tables.data(), tables.size(), hipMemcpyHostToDevice) != hipSuccess) {
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
  if (!std::isfinite(s.lr_wd) || !std::isfinite(s.rate) || !std::isfinite(s.eps) || (a->eps > 0.0 && s.eps == 0.0f))
    return train_fail(SK_EINVAL, "lr, lr weight_decay, lr / (1 - beta1^step) or eps is outside fp32");
  for (int l = 0; l < h->n_tensors; ++l)
    if (!params[l] || !grads[l] || (masters && !masters[l])) return train_fail(SK_EINVAL, "NULL tensor pointer");
  TrainGuard guard(h->device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  const bool clip = a->max_norm > 0.0, few = h->n_chunks <= kFewChunks;
  s.scale = clip && !few ? h->d_scale : a->grad_scale;
  s.part = clip && few ? h->d_part : nullptr;
  s.n_part = h->n_chunks;
  s.max_norm = (float)a->max_norm;
  s.norm = a->norm;
  for (int pass = clip ? 0 : 1; pass < 2; ++pass) {
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
    if (pass == 0 && !few)
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
  if (!guard.ok) return train_no_device();
  const int64_t groups = h->elems / kPer;
  hipLaunchKernelGGL(k_adamw_moments, dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, (hipStream_t)stream, groups,
                     (const uint2 *)m, m_exp, (const uint2 *)v, v_exp, m_out, v_out);
  return train_launched();
}

void sketch_adamw_destroy(sk_adamw *h) {
  if (!h) return;
  TrainGuard guard(h->device);
  (void)hipDeviceSynchronize();
  free_adamw(h);
}

}  // extern "C"
