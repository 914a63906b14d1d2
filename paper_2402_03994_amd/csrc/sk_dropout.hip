// sk_dropout.hip -- dropout whose mask is drawn again wherever it is needed, with
// the residual sum (C ABI of include/sketch_train.h).
//
// Element i is kept where 16 bits of the Philox block at counter
// (i / 8, step, site, SK_STREAM_DROPOUT) are at least t = round(65536 p), and
// scaled by 65536 / (65536 - t); the gradient is the same call on dy.  A thread
// takes the eight elements of one block, which it evaluates in registers, so that
// the mask costs no memory; 16 bits an element keep the ten rounds (30 vector
// operations an element with 32 bits, more than memory allows) beside the reads.
// Bound by memory: 32768 x 4096 bf16 with the residual 134 us, 6.0 TB/s.
#include <algorithm>

#include "sk_train.h"

using namespace sk;

namespace {

struct Drop {
  const void *x, *res;
  void *out;
  int64_t n, width, ld, ld_res, ld_out;  // elements; of a row; row strides
  int64_t first, groups;  // of the launch; of the call
  uint32_t drop, step, site;
  const int64_t *step_at;
  float scale;
  Key key;
  bool past;
};

// the block's 16 bits for element e of eight
__device__ __forceinline__ uint32_t bits_of(const W4 &w, int e) { return (e & 1) ? w.w[e >> 1] >> 16 : w.w[e >> 1] & 0xFFFFu; }

// FLAT: rows follow each other without gaps in all three, so that groups of eight are eight elements in a row.
template <typename T, bool RES, bool FLAT>
__global__ __launch_bounds__(256) void k_dropout(Drop a) {
  constexpr int N = Vec<T>::N, NV = 8 / N;
  const int64_t q = a.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= a.groups) return;
  const uint32_t step = a.step_at ? (uint32_t)*a.step_at : a.step;
  const int64_t i = q * 8;
  const int count = (int)(a.n - i < 8 ? a.n - i : 8);
  int64_t xi = i, ri = i, oi = i;
  bool vec = count == 8;
  int64_t row = 0, col = i;
  if (!FLAT) {
    row = i / a.width;
    col = i - row * a.width;
    vec = vec && col + 8 <= a.width;
    xi = row * a.ld + col;
    ri = row * a.ld_res + col;
    oi = row * a.ld_out + col;
  }
  u32x4 x[NV], r[NV];
  if (vec) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      x[k] = Vec<T>::load((const T *)a.x + xi + k * N);
      if (RES) r[k] = Vec<T>::load((const T *)a.res + ri + k * N);
    }
  }
  const W4 w = philox_at<true>((uint32_t)q, step, a.site, SK_STREAM_DROPOUT, a.key);
  if (vec) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = Vec<T>::get(x[e / N], e % N), s = RES ? Vec<T>::get(r[e / N], e % N) : 0.0f;
      // a choice, not a product: what is dropped may be an infinity or a NaN
      f[e] = bits_of(w, e) >= a.drop ? (RES ? __builtin_fmaf(v, a.scale, s) : v * a.scale) : s;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) Vec<T>::store((T *)a.out + oi + k * N, Vec<T>::pack(f + k * N), a.past);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e < count) {
        const float v = to_f32(((const T *)a.x)[row * a.ld + col]), s = RES ? to_f32(((const T *)a.res)[row * a.ld_res + col]) : 0.0f;
        ((T *)a.out)[row * a.ld_out + col] =
            from_f32<T>(bits_of(w, e) >= a.drop ? (RES ? __builtin_fmaf(v, a.scale, s) : v * a.scale) : s);
        if (++col == a.width) {
          col = 0;
          ++row;
        }
      }
    }
  }
}

template <typename T>
void run(Drop a, bool flat, hipStream_t st) {
  constexpr int64_t kMost = (int64_t)1 << 31;  // groups of a launch: grids below 2^32 threads
  for (; a.first < a.groups; a.first += kMost) {
    const dim3 grid((unsigned)((std::min(kMost, a.groups - a.first) + 255) / 256)), block(256);
    if (a.res) {
      if (flat)
        hipLaunchKernelGGL((k_dropout<T, true, true>), grid, block, 0, st, a);
      else
        hipLaunchKernelGGL((k_dropout<T, true, false>), grid, block, 0, st, a);
    } else {
      if (flat)
        hipLaunchKernelGGL((k_dropout<T, false, true>), grid, block, 0, st, a);
      else
        hipLaunchKernelGGL((k_dropout<T, false, false>), grid, block, 0, st, a);
    }
  }
}

}  // namespace

extern "C" int sketch_dropout(const void *x, sk_dtype dtype, int64_t rows, int64_t width, int64_t ld, const void *residual,
                              int64_t ld_residual, void *out, int64_t ld_out, double p, uint64_t seed, int64_t step,
                              const int64_t *step_at, int64_t site, int32_t device, void *stream) {
  if (dtype != SK_F32 && dtype != SK_BF16) return train_fail(SK_EDTYPE, "unknown dtype");
  if (rows < 0 || width < 1 || ld < width || ld_out < width || (residual && ld_residual < width))
    return train_fail(SK_EINVAL, "need rows >= 0, width >= 1 and row strides >= width");
  if (!(p >= 0.0 && p <= 1.0)) return train_fail(SK_EINVAL, "p must be in [0, 1]");
  if (step < 0 || step >> 32 || site < 0 || site >> 32) return train_fail(SK_EINVAL, "step and site must be in [0, 2^32)");
  if (rows && width > ((int64_t)1 << 35) / rows) return train_fail(SK_EUNSUPPORTED, "more than 2^35 elements");
  if (rows && (!x || !out)) return train_fail(SK_EINVAL, "NULL argument");
  if ((out == x && ld_out != ld) || (residual && out == residual && ld_out != ld_residual))
    return train_fail(SK_EINVAL, "in place needs the same row stride");
  if (rows == 0) return SK_OK;
  TrainGuard guard(device);
  if (!guard.ok) return train_no_device();
  const uint32_t drop = (uint32_t)(p * 65536.0 + 0.5);
  Drop a{x, residual, out, rows * width, width, ld, ld_residual, ld_out, 0, 0, drop, (uint32_t)step, (uint32_t)site, step_at,
         drop < 65536 ? 65536.0f / (float)(65536 - drop) : 0.0f, make_key(seed), false};
  a.groups = (a.n + 7) / 8;
  // fp32 leaves in two stores of 16 bytes of every 32, which the caches put together (32768 x 4096 with residual past them 538
  // us, 304 us so; bf16 136 us either way)
  a.past = dtype == SK_BF16 && a.n * 2 > kPastBytes;
  const bool flat = rows == 1 || (ld == width && ld_out == width && (!residual || ld_residual == width));
  if (dtype == SK_F32)
    run<float>(a, flat, (hipStream_t)stream);
  else
    run<bf16>(a, flat, (hipStream_t)stream);
  return train_launched();
}
