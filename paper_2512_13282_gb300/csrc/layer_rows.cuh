// layer_rows.cuh -- element access and row sums shared by the layer
// operators' kernels (layer_rows.cu).
#pragma once
#include <cuda_bf16.h>

#include "layer_internal.h"

namespace gb300 {

using bf16 = __nv_bfloat16;
struct Q8 {};  // element type tag: a value held in a checkpoint

// 2^(e - 127) of a block exponent: e = 255 stands for NaN.
__device__ __forceinline__ float q8_scale(uint32_t e) {
  return __uint_as_float(e == 255u ? 0x7FC00000u : e << 23);
}

// The block exponent of a block whose largest magnitude has the float bits
// `top` (sign bit clear): the least E >= -126 with top <= 127 * 2^E, plus
// 127.  With top = 1.f * 2^k that is E = k - 6 while 1.f <= 127/64 =
// 1.984375, else k - 5; 0.984375 * 2^23 = 0x7E0000 is the last mantissa of
// the first kind, and adding 0x1FFFF carries into the exponent exactly for
// the mantissas past it.  A NaN or an infinity (bits >= 0x7F800000) gives
// 255.  A subnormal top (exponent field 0) falls under the lower limit.
__device__ __forceinline__ uint32_t q8_exponent(uint32_t top) {
  const int e = static_cast<int>((top + 0x1FFFFu) >> 23) - 6;
  return top >= 0x7F800000u ? 255u : static_cast<uint32_t>(max(e, 1));
}
// 2^-E for that exponent, by which a block is multiplied (exactly) before
// rounding; 0 for a block of NaN, whose bytes are 0.  E lies in -126 .. 122.
__device__ __forceinline__ float q8_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// round_half_even(x * inverse) of a finite block; 0 where the block holds a
// NaN or an infinity; limited to 63 at the largest exponent (E = 122), where
// 64 * 2^122 would be past float32.
__device__ __forceinline__ int q8_quantise(float x, float inverse, uint32_t e) {
  int v = __float2int_rn(x * inverse);
  if (e >= 249u) v = e == 255u ? 0 : min(max(v, -63), 63);
  return v;
}

template <typename T>
__device__ __forceinline__ float load_value(const void *p, int64_t i) {
  if constexpr (sizeof(T) == 4)
    return static_cast<const float *>(p)[i];
  else
    return __bfloat162float(static_cast<const bf16 *>(p)[i]);
}
template <typename T>
__device__ __forceinline__ void store_value(void *p, int64_t i, float v) {
  if constexpr (sizeof(T) == 4)
    static_cast<float *>(p)[i] = v;
  else
    static_cast<bf16 *>(p)[i] = __float2bfloat16_rn(v);
}
// v as its stored type holds it.
template <typename T>
__device__ __forceinline__ float as_stored(float v) {
  if constexpr (sizeof(T) == 4)
    return v;
  else
    return __bfloat162float(__float2bfloat16_rn(v));
}

// A parameter vector of either type, or absent.
__device__ __forceinline__ float load_param(const void *p, int type, int c, float absent) {
  if (!p) return absent;
  return type == GEMM_TYPE_F32 ? static_cast<const float *>(p)[c] : __bfloat162float(static_cast<const bf16 *>(p)[c]);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum of a pair over the block (a whole number of warps, at most 32); every
// thread receives it.  `buf` alternates between calls, so that one barrier a
// call suffices: what a call writes is last read before the next call's
// barrier.  The order of the additions is fixed by the block's shape.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 (*sm)[32], int buf) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  a = warp_sum(a);
  b = warp_sum(b);
  if (lane == 0) sm[buf][warp] = make_float2(a, b);
  __syncthreads();
  const float2 v = lane < warps ? sm[buf][lane] : make_float2(0.f, 0.f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}

}  // namespace gb300
