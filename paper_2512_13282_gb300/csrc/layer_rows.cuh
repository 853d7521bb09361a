// layer_rows.cuh -- element access and row sums shared by the layer
// operators' kernels (layer_ln_fwd.cu, layer_ln_bwd.cu,
// layer_q8.cu, layer_gate.cu, layer_dropout.cu).
#pragma once
#include <cuda_bf16.h>

#include "layer_internal.h"

namespace gb300 {

using bf16 = __nv_bfloat16;
struct Q8 {     // element type: a value held in a checkpoint, as its byte
  int8_t byte;
};

// Pairs of float32 operations in one instruction each; both halves round as
// the scalar ones do.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(d)
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)),
        "l"(*reinterpret_cast<unsigned long long *>(&c)));
  return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
  return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
  return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

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
// rounding.  E lies in -126 .. 122; what it gives for a block of NaN (e = 255,
// minus infinity) stands for nothing: the callers make that block's bytes 0.
__device__ __forceinline__ float q8_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// Float bits of the largest magnitude among 2 * N bf16 values, two to a word;
// a NaN if there is one.
template <int N>
__device__ __forceinline__ uint32_t max_magnitude_bf16(const uint32_t (&w)[N]) {
  __nv_bfloat162 m[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t a = w[i] & 0x7FFF7FFFu;
    m[i] = *reinterpret_cast<const __nv_bfloat162 *>(&a);
  }
#pragma unroll
  for (int n = N; n > 1; n /= 2)
#pragma unroll
    for (int i = 0; i < n / 2; ++i) m[i] = __hmax2_nan(m[i], m[i + n / 2]);
  const uint32_t t = *reinterpret_cast<const uint32_t *>(m);
  return max(t << 16, t & 0xFFFF0000u);
}

// The byte of a value of a block with exponent e: round_half_even(x * inverse),
// 0 where the block holds a NaN or an infinity, limited to 63 at the largest
// exponent (E = 122), where 64 * 2^122 would be past float32.  Rounded by
// adding 1.5 * 2^23, where a float's unit in the last place is 1; what is left
// in the sum's low byte is the result.  (min and max drop a NaN.)
__device__ __forceinline__ uint32_t q8_byte(float x, float inverse, uint32_t e) {
  constexpr float kMagic = 12582912.0f;
  const float limit = e == 255u ? 0.f : e == 249u ? 63.f : 127.f;
  const float v = fminf(fmaxf(fmaf(x, inverse, kMagic) - kMagic, -limit), limit);
  return __float_as_uint(v + kMagic) & 0xFFu;
}

// The same for eight values of a block below the largest exponent, packed
// (v[0].x in the low byte of x); rounded as in q8_byte.
__device__ __forceinline__ uint2 q8_pack8(const float2 (&v)[4], float inverse) {
  const float2 scale = both(inverse), magic = both(12582912.0f);
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = fma2(v[2 * i], scale, magic), b = fma2(v[2 * i + 1], scale, magic);
    const uint32_t lo = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040);
    w[i] = __byte_perm(lo, hi, 0x5410);
  }
  return make_uint2(w[0], w[1]);
}
// ... and of any block: zeros where e = 255; at e = 249, where no value is past
// 64, bytes of 64 (0x40) become 63 and bytes of -64 (0xC0) -63, four at a time.
__device__ __forceinline__ uint2 q8_pack8(const float2 (&v)[4], uint32_t e) {
  uint2 w = q8_pack8(v, q8_inverse(e));
  if (e >= 249u) {
    if (e == 249u) {
      w.x += (__vcmpeq4(w.x, 0xC0C0C0C0u) & 0x01010101u) - (__vcmpeq4(w.x, 0x40404040u) & 0x01010101u);
      w.y += (__vcmpeq4(w.y, 0xC0C0C0C0u) & 0x01010101u) - (__vcmpeq4(w.y, 0x40404040u) & 0x01010101u);
    } else {
      w = make_uint2(0, 0);
    }
  }
  return w;
}

// Byte i of w as a float (see s8x4_to_bf16x4 for the arithmetic).
__device__ __forceinline__ float s8_to_float(uint32_t w, int i) {
  const uint32_t u = w ^ 0x80808080u;
  return __fsub_rn(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7650 + i)), 8388736.0f);
}

// Scaling by 2^E in bf16 arithmetic is exact: a byte has at most 8
// significant bits, and no product with E >= -126 is subnormal.
__device__ __forceinline__ uint32_t scale_bf16x2(uint32_t v, __nv_bfloat162 s) {
  const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&v), s);
  return *reinterpret_cast<const uint32_t *>(&p);
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

// V consecutive elements of a row as they are in memory, loaded with the
// widest loads V allows (the address is a multiple of V elements), so that a
// row can be fetched ahead of its use in half the registers.
template <typename T, int V>
struct Chunk {
  static constexpr int kBytes = V * (int)sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void *row, int64_t c) {
    const char *p = static_cast<const char *>(row) + c * (int64_t)sizeof(T);
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 v = *reinterpret_cast<const uint2 *>(p);
      w[0] = v.x, w[1] = v.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t *>(p);
    } else if constexpr (kBytes == 2) {
      w[0] = *reinterpret_cast<const uint16_t *>(p);
    } else {
      w[0] = *reinterpret_cast<const uint8_t *>(p);
    }
  }
  // The first n of the chunk's elements, one by one.
  __device__ __forceinline__ void load_part(const void *row, int64_t c, int n) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4)
          w[i] = static_cast<const uint32_t *>(row)[c + i];
        else if constexpr (sizeof(T) == 2)
          w[i / 2] |= (uint32_t) static_cast<const uint16_t *>(row)[c + i] << (16 * (i & 1));
        else
          w[i / 4] |= (uint32_t) static_cast<const uint8_t *>(row)[c + i] << (8 * (i & 3));
      }
  }
  // Element i (of a checkpoint: its byte, unscaled).
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[i]);
    else if constexpr (sizeof(T) == 2)
      return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else
      return s8_to_float(w[i / 4], i & 3);
  }
  __device__ __forceinline__ float2 get2(int i) const { return make_float2(get(2 * i), get(2 * i + 1)); }
};

// 32 bytes as eight words (any address that is a multiple of 16; one access
// where it is one of 32).
__device__ __forceinline__ void store_32_bytes(void *p, const uint32_t (&w)[8]) {
  if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(__cvta_generic_to_global(p)),
                 "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    uint4 *d = static_cast<uint4 *>(p);
    d[0] = make_uint4(w[0], w[1], w[2], w[3]);
    d[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// V consecutive results rounded to T and stored (address a multiple of V
// elements); the first n of them, one by one, where n < V.
template <typename T, int V>
__device__ __forceinline__ void store_chunk(void *row, int64_t c, const float *v, int n) {
  if (n < V) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) store_value<T>(row, c + i, v[i]);
    return;
  }
  if constexpr (sizeof(T) == 4) {
    float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(row) + c);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) d[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  } else {
    uint4 *d = reinterpret_cast<uint4 *>(static_cast<char *>(row) + c * 2);
#pragma unroll
    for (int i = 0; i < V / 8; ++i)
      d[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                        pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
  }
}

// Rows at any alignment.  A lane's values fill pieces of 16 bytes (P = 4 words;
// 8 bytes, P = 2, where they are no more), but lie in one piece more where the
// row does not start on a piece: what is loaded from whole pieces is shifted
// down, what is stored is shifted up.

// W words from byte `by` (below a piece's size) of w on.
template <int W, int P>
__device__ __forceinline__ void shift_words(uint32_t (&w)[W + P], uint32_t by) {
  if constexpr (P == 4) {
#pragma unroll
    for (int i = 0; i < W + 2; ++i) w[i] = by & 8u ? w[i + 2] : w[i];
  }
#pragma unroll
  for (int i = 0; i < W + 1; ++i) w[i] = by & 4u ? w[i + 1] : w[i];
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (by & 3u) * 8);
}

// Bytes [b, SIZE) and [0, b) of a piece as naturally aligned runs of a power of
// two: f(first byte, bytes).
template <uint32_t SIZE, typename F>
__device__ __forceinline__ void upper_runs(uint32_t b, F f) {
#pragma unroll
  for (uint32_t n = 1; n < SIZE; n *= 2)
    if (b & n) {
      f(b, n);
      b += n;
    }
}
template <uint32_t SIZE, typename F>
__device__ __forceinline__ void lower_runs(uint32_t b, F f) {
  uint32_t at = 0;
#pragma unroll
  for (uint32_t n = SIZE / 2; n >= 1; n /= 2)
    if (b & n) {
      f(at, n);
      at += n;
    }
}
// A run of the piece w[0 .. P - 1] to its place in the piece at p.
template <int P, int N>
__device__ __forceinline__ void store_run(char *p, uint32_t at, uint32_t n, const uint32_t (&w)[N]) {
  const uint32_t i = at >> 2;
  uint32_t v = i & 1u ? w[1] : w[0];
  if constexpr (P == 4) v = i & 2u ? (i & 1u ? w[3] : w[2]) : v;
  v >>= 8 * (at & 3u);
  if (P == 4 && n == 8)
    *reinterpret_cast<uint2 *>(p + at) = at ? make_uint2(w[P - 2], w[P - 1]) : make_uint2(w[0], w[1]);
  else if (n == 4)
    *reinterpret_cast<uint32_t *>(p + at) = v;
  else if (n == 2)
    *reinterpret_cast<uint16_t *>(p + at) = (uint16_t)v;
  else
    *reinterpret_cast<uint8_t *>(p + at) = (uint8_t)v;
}

// A lane's W words to dst, any address that its type allows.  All lanes of the
// warp call it, what neighbouring ones hold being neighbours in memory.  whole:
// the lane has words to store; joined: the lane before it has the words before
// them; taken: the lane after it has the words after them.  The later lane
// writes a piece shared by two; where there is none, each writes its part.
template <int P, int W>
__device__ __forceinline__ void store_shifted(void *dst, bool whole, bool joined, bool taken, const uint32_t (&in)[W]) {
  constexpr uint32_t kSize = 4 * P;
  const auto store_piece = [](char *p, const uint32_t *w) {
    if constexpr (P == 4)
      *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else
      *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
  };
  const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(dst) & (kSize - 1);
  char *p = static_cast<char *>(dst) - off;
  uint32_t w[W + P];
#pragma unroll
  for (int i = 0; i < P; ++i) w[i] = __shfl_up_sync(0xffffffffu, in[W - P + i], 1);
  if (!whole) return;
  if (off == 0) {
#pragma unroll
    for (int i = 0; i < W / P; ++i) store_piece(p + i * kSize, in + i * P);
    return;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) w[P + i] = in[i];
  if (!taken) {  // bytes [0, off) of the last piece
    uint32_t t[2 * P] = {};
#pragma unroll
    for (int i = 0; i < P; ++i) t[i] = in[W - P + i];
    shift_words<P, P>(t, kSize - off);
    lower_runs<kSize>(off, [&](uint32_t at, uint32_t n) { store_run<P>(p + 4 * W, at, n, t); });
  }
  shift_words<W, P>(w, kSize - off);
#pragma unroll
  for (int i = 0; i < W / P; ++i) {
    if (i == 0 && !joined)
      upper_runs<kSize>(off, [&](uint32_t at, uint32_t n) { store_run<P>(p, at, n, w); });
    else
      store_piece(p + i * kSize, w + i * P);
  }
}

// A run of the piece at p into its words w[AT ..] (zero before).
template <int AT, int N>
__device__ __forceinline__ void load_run(const char *p, uint32_t at, uint32_t n, uint32_t (&w)[N]) {
  uint2 v = make_uint2(0, 0);
  if (n == 8)
    v = *reinterpret_cast<const uint2 *>(p + at);
  else
    v.x = (n == 4   ? *reinterpret_cast<const uint32_t *>(p + at)
           : n == 2 ? *reinterpret_cast<const uint16_t *>(p + at)
                    : *reinterpret_cast<const uint8_t *>(p + at))
          << (8 * (at & 3u));
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) w[AT + k] |= at >> 2 == k ? v.x : n == 8 && (at >> 2) + 1 == k ? v.y : 0u;
}

// A lane's W words at src, any address.  Pieces that reach past the row (first: it
// starts with these words; after: its bytes that follow) are read in runs.
template <int W>
__device__ __forceinline__ void load_half(const void *src, bool first, int64_t after, uint32_t (&out)[W]) {
  const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(src) & 15u;
  const char *p = static_cast<const char *>(src) - off;
  uint32_t w[W + 4] = {};
#pragma unroll
  for (int i = 0; i <= W / 4; ++i) {
    if (i == 0 && first && off) {
      upper_runs<16>(off, [&](uint32_t at, uint32_t n) { load_run<0>(p, at, n, w); });
    } else if (i == W / 4 && after < 16 - (int)off) {
      lower_runs<16>(off, [&](uint32_t at, uint32_t n) { load_run<W>(p + 4 * W, at, n, w); });
    } else if (i < W / 4 || off) {
      const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  }
  shift_words<W, 4>(w, off);
#pragma unroll
  for (int i = 0; i < W; ++i) out[i] = w[i];
}

// Piece h of the matrix, V columns, -> its row and first column, `pieces` of them
// a row.  With rows laid end to end a launcher may make the matrix one row, and
// 32-bit arithmetic serves any matrix below 2^32 pieces.
template <int V>
__device__ __forceinline__ void row_piece(int64_t h, int64_t pieces, int64_t *r, int64_t *c) {
  int64_t row;
  if ((uint64_t)h <= 0xFFFFFFFFull && pieces <= 0xFFFFFFFFll)
    row = (uint32_t)h / (uint32_t)pieces;
  else
    row = h / pieces;
  *r = row;
  *c = (h - row * pieces) * V;
}
// Half block h of a checkpoint (`halves` is even).
__device__ __forceinline__ void half_block(int64_t h, int64_t halves, int64_t *r, int64_t *c) {
  row_piece<16>(h, halves, r, c);
}

// The first n of a half block's bytes.
__device__ __forceinline__ void store_bytes(int8_t *q, const uint32_t (&w)[4], int n) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < n) q[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
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

// The second half of a block-wide sum, after the barrier: the sum of the
// values of up to WARPS warps (a multiple of four; absent ones zero), read by
// broadcast (cheaper, and sooner done, than another tree of shuffles).
template <int WARPS>
__device__ __forceinline__ float2 sum_over_warps(const float2 *sm) {
  float2 s = both(0.f), t = s;
#pragma unroll
  for (int w = 0; w < WARPS; w += 4) {
    const float4 a = *reinterpret_cast<const float4 *>(sm + w), b = *reinterpret_cast<const float4 *>(sm + w + 2);
    s = add2(s, add2(make_float2(a.x, a.y), make_float2(a.z, a.w)));
    t = add2(t, add2(make_float2(b.x, b.y), make_float2(b.z, b.w)));
  }
  return add2(s, t);
}
template <int WARPS>
__device__ __forceinline__ float sum_over_warps(const float *sm) {
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < WARPS; w += 4) {
    const float4 a = *reinterpret_cast<const float4 *>(sm + w);
    s += (a.x + a.y) + (a.z + a.w);
  }
  return s;
}

// A place in a ring of row slots in shared memory that bulk copies fill ahead
// of their use: counted, not computed from the row's number (a division per
// row and thread is a tenth of a row's instructions).
struct RingPlace {
  int slot = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void advance(int stages) {
    if (++slot == stages) {
      slot = 0;
      parity ^= 1u;
    }
  }
};
// After giving up (thread 0): the fills issued and not waited for -- `use` is
// the first of them, `pending` their number -- have landed before the block's
// memory is given up.
__device__ __forceinline__ void ring_drain(uint32_t bars, int stages, RingPlace use, int64_t pending) {
  for (; pending > 0; --pending, use.advance(stages))
    mbar_wait_drain(bars + 8u * use.slot, use.parity, 200ull * 1000 * 1000);
}

// Elements n .. 7 of a group to zero.
__device__ __forceinline__ void zero_from(float2 (&x)[4], int n) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = make_float2(2 * j < n ? x[j].x : 0.f, 2 * j + 1 < n ? x[j].y : 0.f);
}
// A group's words, as stored in a row of T at column c of `cols`: in one piece
// where the row is aligned, else shifted; a row's last few values one by one.
// All lanes of the warp call it.
template <typename T, bool SHIFT>
__device__ __forceinline__ void store_group(T *row, int c, int cols, const uint32_t (&w)[2 * sizeof(T)]) {
  constexpr int W = 2 * (int)sizeof(T), P = W < 4 ? 2 : 4;
  if constexpr (!SHIFT) {
    if (c >= cols) return;
    if constexpr (P == 2)
      *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
    else
#pragma unroll
      for (int i = 0; i < W / 4; ++i)
        reinterpret_cast<uint4 *>(row + c)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
    const int lane = threadIdx.x & 31;
    store_shifted<P>(row + c, c + 8 <= cols, lane > 0, lane < 31 && c + 16 <= cols, w);
    if (c < cols && c + 8 > cols) {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (c + i < cols) {
          if constexpr (sizeof(T) == 4)
            reinterpret_cast<uint32_t *>(row)[c + i] = w[i];
          else if constexpr (sizeof(T) == 2)
            reinterpret_cast<uint16_t *>(row)[c + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
          else
            reinterpret_cast<uint8_t *>(row)[c + i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
        }
    }
  }
}

// A row of T values on its way through a ring slot, its elements taken in
// groups of eight a thread.
//
// V = 8: rows start on 16 bytes and are whole 16-byte pieces.  The slot is the
// row, group v of thread t the eight values from column (v * threads + t) * 8.
//
// V = 1: any alignment.  The slot keeps the row's place within 16 bytes, so
// that a bulk copy brings the aligned pieces that lie wholly inside the row;
// the ends, up to kEdge values on each side, are read by the threads that own
// them, a row ahead, and put into the slot by them: a thread reads only its
// own columns from a slot, so that takes no barrier.  Value i of group v is
// column (v * 8 + i) * threads + t, neighbouring lanes being neighbours in
// memory.  Rows have at least 2 * kEdge values.  Its blocks have exactly THREADS
// threads, which makes every address of a thread's values a constant distance
// from its first (the many small accesses of V = 1 cost instructions, not
// bytes); with V = 8 THREADS is only the most.
template <typename T, int V, int THREADS>
struct SlotRow {
  static constexpr int kSize = (int)sizeof(T), kEdge = 16 / kSize;
  uint32_t head, tail;  // the ends' bits, fetched ahead
  int tail_col;         // column of the tail value that this thread owns, or -1
  __device__ __forceinline__ void init(int cols) {
    const int c0 = cols - kEdge, d = ((int)threadIdx.x - c0 % THREADS + THREADS) % THREADS;
    tail_col = d < kEdge ? c0 + d : -1;
  }
  __device__ __forceinline__ static uint32_t offset(const void *row) {
    return V == 1 ? (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u : 0u;
  }
  // Thread 0: the copy into the slot at `dst`; bytes to expect.
  __device__ __forceinline__ static uint32_t copy_bytes(const void *row, int cols) {
    if constexpr (V != 1) return (uint32_t)cols * kSize;
    const uintptr_t a = reinterpret_cast<uintptr_t>(row), lo = (a + 15) & ~(uintptr_t)15;
    return (uint32_t)(((a + (uintptr_t)cols * kSize) & ~(uintptr_t)15) - lo);
  }
  __device__ __forceinline__ static void copy(uint32_t dst, const void *row, uint32_t bytes, uint32_t bar) {
    const uint32_t skip = (16u - offset(row)) & 15u;
    bulk_load(dst + (skip ? 16u : 0u), static_cast<const char *>(row) + skip, bytes, bar);
  }
  __device__ __forceinline__ static uint32_t bits(const void *row, int c) {
    if constexpr (kSize == 4) return static_cast<const uint32_t *>(row)[c];
    if constexpr (kSize == 2) return static_cast<const uint16_t *>(row)[c];
    return static_cast<const uint8_t *>(row)[c];
  }
  __device__ __forceinline__ static void put(uint8_t *at, uint32_t b) {
    if constexpr (kSize == 4)
      *reinterpret_cast<uint32_t *>(at) = b;
    else if constexpr (kSize == 2)
      *reinterpret_cast<uint16_t *>(at) = (uint16_t)b;
    else
      *at = (uint8_t)b;
  }
  __device__ __forceinline__ void fetch_ends(const void *row) {
    if constexpr (V == 1) {
      head = threadIdx.x < kEdge ? bits(row, threadIdx.x) : 0;
      tail = tail_col >= 0 ? bits(row, tail_col) : 0;
    }
  }
  // After the copy into the slot has been waited for.  The fence orders these
  // writes before the copy that will refill the slot.
  __device__ __forceinline__ void put_ends(uint8_t *slot, uint32_t off) const {
    if constexpr (V == 1) {
      if (threadIdx.x < kEdge) put(slot + off + threadIdx.x * kSize, head);
      if (tail_col >= 0) put(slot + off + tail_col * kSize, tail);
      if (threadIdx.x < kEdge || tail_col >= 0) fence_proxy_async_smem();
    }
  }
  // Group v of the row; zero past the row's end (V = 8: the group at column 0
  // instead, for the caller to leave out).
  __device__ __forceinline__ static void load(const uint8_t *slot, uint32_t off, int v, int cols, float2 (&x)[4]) {
    const int t = (int)threadIdx.x;
    if constexpr (V == 8) {
      const int c = (v * (int)blockDim.x + t) * 8;
      Chunk<T, 8> raw;
      raw.load(slot, c < cols ? c : 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = raw.get2(j);
    } else {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = (v * 8 + i) * THREADS + t;
        Chunk<T, 1> raw;
        raw.w[0] = 0;
        if (c < cols) raw.load(slot + off, c);
        e[i] = c < cols ? raw.get(0) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = make_float2(e[2 * j], e[2 * j + 1]);
    }
  }
};
// Column of value i of group v (see SlotRow).
template <int V, int THREADS>
__device__ __forceinline__ int group_col(int v, int i) {
  return V != 1 ? (v * (int)blockDim.x + (int)threadIdx.x) * 8 + i : (v * 8 + i) * THREADS + (int)threadIdx.x;
}

// The same for groups of eight consecutive values at any alignment (V = kShifted;
// columns as with V = 8), rows of at least 2 * kEdge values.  The ends are put
// into the slot by the block's first threads, a barrier before it is read; a
// group is read in whole 16-byte pieces and shifted into place.
constexpr int kShifted = 0;
template <typename T>
struct ShiftedRow {
  static constexpr int kSize = (int)sizeof(T), kEdge = 16 / kSize;
  static_assert(kSize > 1, "a group fills pieces of 16 bytes");
  using Any = SlotRow<T, 1, 32>;
  uint32_t end;  // bits of the end value fetched ahead
  __device__ __forceinline__ static uint32_t offset(const void *row) { return Any::offset(row); }
  __device__ __forceinline__ static uint32_t copy_bytes(const void *row, int cols) { return Any::copy_bytes(row, cols); }
  __device__ __forceinline__ static void copy(uint32_t dst, const void *row, uint32_t bytes, uint32_t bar) {
    Any::copy(dst, row, bytes, bar);
  }
  // The end value of this thread: threads 0 .. kEdge - 1 have the row's first
  // values, the next kEdge its last.
  __device__ __forceinline__ static int end_col(int cols) {
    const int t = (int)threadIdx.x;
    return t < kEdge ? t : cols - 2 * kEdge + t;
  }
  __device__ __forceinline__ void fetch_ends(const void *row, int cols) {
    if (threadIdx.x < 2 * kEdge) end = Any::bits(row, end_col(cols));
  }
  // Into the slot of that row, where the copy does not bring the value; no
  // thread reads the slot's former row any more.  The fence orders the write
  // before the copy that will refill the slot.
  __device__ __forceinline__ void put_ends(uint8_t *slot, uint32_t off, int cols) const {
    if (threadIdx.x >= 2 * kEdge) return;
    const uint32_t at = off + (uint32_t)end_col(cols) * kSize, last = (off + (uint32_t)cols * kSize) & ~15u;
    if ((off == 0 || at >= 16) && at < last) return;
    Any::put(slot + at, end);
    fence_proxy_async_smem();
  }
  // Group v of the row, zero past its end (the group at column 0 for a thread
  // whose group starts past it, for the caller to leave out).
  __device__ __forceinline__ static void load(const uint8_t *slot, uint32_t off, int v, int cols, float2 (&x)[4]) {
    constexpr int W = 2 * kSize;
    const int c = (v * (int)blockDim.x + (int)threadIdx.x) * 8, at = c < cols ? c : 0;
    const uint4 *p = reinterpret_cast<const uint4 *>(slot + (uint32_t)at * kSize);
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i <= W / 4; ++i) {
      const uint4 u = p[i];
      w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
    }
    shift_words<W, 4>(w, off);
    Chunk<T, 8> raw;
#pragma unroll
    for (int i = 0; i < W; ++i) raw.w[i] = w[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = raw.get2(j);
    if (at + 8 > cols) zero_from(x, cols - at);
  }
};

// Bytes of a slot for a row of cols values of `size` bytes.
inline uint32_t slot_bytes(int64_t cols, int size, bool aligned) {
  return (uint32_t)(aligned ? cols * size : (cols * size + 30) / 16 * 16);
}
// The same for ShiftedRow: whole groups, and the piece more that they reach into.
inline uint32_t shifted_slot_bytes(int64_t cols, int size) {
  return (uint32_t)(((cols + 7) / 8 * 8 * size + 31) / 16 * 16);
}

constexpr int kMaxStages = 8;
constexpr int64_t kRingBytes = 200 * 1024;  // shared memory of an SM's rings together

// Whether rows of elements of `size` bytes at p, pitch ld, all start on a
// multiple of `align` bytes.
inline bool rows_on(const void *p, int64_t ld, int size, int align) {
  return (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0 && ld * size % align == 0;
}

}  // namespace gb300
