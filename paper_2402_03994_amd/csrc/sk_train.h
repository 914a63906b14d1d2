// sk_train.h -- what the training-step operators (sk_embed.hip, sk_loss.hip,
// sk_adamw.hip) share: argument failures, the device guard, element access and
// ordered workgroup reductions.
#pragma once

#include <cmath>
#include <new>
#include <string>

#include "../../include/sketch_train.h"
#include "sk_launch.h"

namespace sk {

inline int train_fail(int code, const char *msg) noexcept {
  try {
    set_error(code, msg);
  } catch (...) {  // no memory for the message: the code alone
  }
  return code;
}

inline int train_launched() noexcept {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SK_OK : train_fail(SK_EHIP, hipGetErrorString(e));
}

// The call's device, and the caller's current one again on scope exit.  An error that an earlier call to the runtime has
// left is dropped: train_launched() would report it as this call's.
struct TrainGuard {
  int prev = -1, dev;
  bool ok;  // false: there is no device `dev`
  explicit TrainGuard(int d) : dev(d) {
    (void)hipGetLastError();
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    ok = dev >= 0 && (prev == dev || hipSetDevice(dev) == hipSuccess);
    if (!ok) (void)hipGetLastError();
  }
  ~TrainGuard() {
    if (prev >= 0 && prev != dev) (void)hipSetDevice(prev);
  }
};
inline int train_no_device() noexcept { return train_fail(SK_EINVAL, "device out of range"); }

// Elements: float or bf16 (held as its 16 bits).
struct bf16 {
  uint16_t u;
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
// to nearest even, NaN kept
__device__ __forceinline__ uint32_t bf16_bits(float f) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f);
}
template <typename T>
__device__ __forceinline__ T from_f32(float f);
template <>
__device__ __forceinline__ float from_f32<float>(float f) {
  return f;
}
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float f) {
  return bf16{(uint16_t)bf16_bits(f)};
}

struct OpMax {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct OpAdd {
  template <typename T>
  __device__ T operator()(T a, T b) const {
    return a + b;
  }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
// Reduction over a wave (all 64 lanes active): rotations within the rows of 16 lanes, then the four rows' results.
template <typename Op>
__device__ __forceinline__ float wave_all(float v, Op op) {
  v = op(v, dpp<0x128>(v));
  v = op(v, dpp<0x124>(v));
  v = op(v, dpp<0x122>(v));
  v = op(v, dpp<0x121>(v));
  return op(op(lane_of(v, 0), lane_of(v, 16)), op(lane_of(v, 32), lane_of(v, 48)));
}
template <typename Op>
__device__ __forceinline__ double wave_all(double v, Op op) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = op(v, __shfl_xor(v, d, 64));
  return v;
}

// Reduction over a workgroup of W waves, in a fixed order; every thread gets the result.  `lds` holds W entries and
// is free again after the next barrier.
template <int W, typename Op, typename T>
__device__ __forceinline__ T block_all(T v, Op op, T *lds) {
  v = wave_all(v, op);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = lds[0];
#pragma unroll
  for (int i = 1; i < W; ++i) r = op(r, lds[i]);
  return r;
}

// Outputs above this size are stored past the caches (32 MB of L2, 256 MB in front of the memory), so that the inputs stay
// there; what is smaller is left there for the next kernel to read.  By the call alone, past the caches and through them:
// preference loss of 411 x 50257 fp32 (82 MB) 36 and 41 us, policy update in bf16 of 120 MB 42 and 45, of 160 MB 55 and
// 64, of 240 MB 79 and 97; lookup of 98 MB 29 and 31, of 246 MB 73 and 90.  What follows reads from memory instead: with
// the products before and after it (width 256) a preference loss in bf16 takes 386 and 377 us at 100 MB, 468 and 477 at
// 160 MB; at width 2048 971 and 979, 1222 and 1209; with one plain pass over the gradient alone, 80 MB, 83 and 74.
constexpr int64_t kPastBytes = 64 << 20;

// 16 bytes of elements, aligned to one element only: the loads and stores of gfx950 take any alignment.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Any {
    u32x4 v;
  };
  static __device__ __forceinline__ u32x4 load(const T *p) { return ((const Any *)p)->v; }
  static __device__ __forceinline__ void store(T *p, u32x4 v) { ((Any *)p)->v = v; }
  // past the caches: for more than they hold, so that something else stays there
  static __device__ __forceinline__ void store(T *p, u32x4 v, bool past) {
    if (past) {
      asm volatile("");  // or the compiler makes one ordinary store of the two
      stream(p, v);
      asm volatile("");
    } else {
      store(p, v);
    }
  }
  static __device__ __forceinline__ void stream(T *p, u32x4 v) {
    if (sizeof(T) == 4)
      __builtin_nontemporal_store(v, (u32x4_at4 *)p);
    else
      __builtin_nontemporal_store(v, (u32x4_at2 *)p);
  }
  static __device__ __forceinline__ float get(u32x4 v, int i) {
    if (sizeof(T) == 4) return __uint_as_float(v[i]);
    return __uint_as_float((i & 1) ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4 pack(const float *f) {
    u32x4 v;
    if (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
    } else {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2));
    }
    return v;
  }
};

// Softmax of rows: what the losses on given logits and those on hidden states share.
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.92596299113e-8f;  // log2 e - kLog2e

// scale log2 e as a sum, for exp(scale d) = 2^(d (k + low))
struct Power {
  float k, low;
};
__device__ __forceinline__ Power power_of(float scale) {
  const float k = scale * kLog2e;
  return Power{k, __builtin_fmaf(scale, kLog2eLow, __builtin_fmaf(scale, kLog2e, -k))};
}

// exp(scale d) for an entry of a gradient of type T.  The hardware's exponential of the rounded product d k is off by
// 5e-7 of its value at an exponent of -20 and 9e-7 at -40.  Beside bf16's 2^-8 that is nothing; fp32 entries get what the
// product has lost as a factor 1 + r ln 2 (policy update of 4096 x 50257 fp32: 323 us, 317 us without).  The sums z need no
// such care: exponentials count there by their size.
template <typename T>
__device__ __forceinline__ float entry_exp(float d, Power p) {
  const float t = d * p.k, e = __builtin_amdgcn_exp2f(t);
  if (sizeof(T) == 2) return e;
  const float r = __builtin_fmaf(d, p.low, __builtin_fmaf(d, p.k, -t));
  // d = -inf leaves a NaN in r, and a NaN in d one in e
  return __builtin_fmaf(e, 0.69314718055994530942f * __builtin_amdgcn_fmed3f(r, -1.0f, 1.0f), e);
}

// A row's numbers: the largest entry m and z = sum_j exp(scale (x_j - m)).
struct Stats {
  float m, z;
};

__device__ __forceinline__ float logp_of(float xt, Stats s, float scale) {
  if (s.z == 0.0f) return -INFINITY;
  float a = (xt - s.m) * scale;
  if (a == -INFINITY) a = (0.5f * xt - 0.5f * s.m) * scale * 2.0f;  // the difference alone may have overflowed
  return a - logf(s.z);
}

}  // namespace sk
