// layer_dropout.cu -- dropout with a residual, and its gradient.
//
// Whether the value at (row, column) is kept is a function of the key, the
// step and its place: one Philox4x32-10 block (ten rounds of two 32 x 32 -> 64
// bit products) gives eight 16-bit numbers, those of eight neighbouring
// columns.  Sixteen bits a value and not 32, which halves the generator's
// instructions, most of the kernel's; P is exact to 2^-17.  So it runs at the
// rate of its bytes: 8192 x 12288 bf16 into a float32 residual 142 us (7.1 TB/s),
// its schedulers 60 % busy.
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kThreads = 256;

// The 128 bits of counter (c0, c1, c2, c3) under the key.
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ (k0 + r * 0x9E3779B9u);
    c2 = (uint32_t)(a >> 32) ^ c3 ^ (k1 + r * 0xBB67AE85u);
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
  }
  return make_uint4(c0, c1, c2, c3);
}

// A thread takes the eight values of a row that share a counter.  VEC: all rows
// start on 16 bytes; else values are shifted between registers and the 16-byte
// pieces of memory that they lie in.
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const Dropout p, float scale) {
  griddep_launch_dependents();
  griddep_wait();
  const uint64_t draw = p.step + (p.step_device ? *p.step_device : 0);
  const int64_t groups = (p.cols + 7) / 8, items = p.rows * groups, step = (int64_t)gridDim.x * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t h0 = (int64_t)blockIdx.x * kThreads; h0 < items; h0 += step) {
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    const int64_t at = live ? h : items - 1;
    const int64_t r = at <= 0xFFFFFFFFll ? (int64_t)((uint32_t)at / (uint32_t)groups) : at / groups;
    const int64_t c = (at - r * groups) * 8;
    const int n = live ? (int)min((int64_t)8, p.cols - c) : 0;
    const auto load = [&](auto tag, const void *m, int64_t ld) {
      using T = decltype(tag);
      const T *row = static_cast<const T *>(m) + r * ld;
      Chunk<T, 8> v;
      if (n < 8)
        v.load_part(row, c, n);
      else if constexpr (VEC)
        v.load(row, c);
      else
        load_half(row + c, c == 0, (p.cols - c - 8) * (int64_t)sizeof(T), v.w);
      return v;
    };
    const Chunk<TX, 8> x = load(TX{}, p.x, p.ldx);
    Chunk<TY, 8> b;
    if (p.residual)
      b = load(TY{}, p.residual, p.ldr);
    else
      b.load_part(nullptr, 0, 0);
    const uint4 w = philox((uint32_t)(c >> 3), (uint32_t)r, (uint32_t)draw, (uint32_t)(draw >> 32), (uint32_t)p.seed,
                           (uint32_t)(p.seed >> 32));
    const uint32_t bits[4] = {w.x, w.y, w.z, w.w};
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t number = i & 1 ? bits[i / 2] >> 16 : bits[i / 2] & 0xFFFFu;
      v[i] = number >= p.threshold ? fmaf(x.get(i), scale, b.get(i)) : b.get(i);
    }
    TY *row = static_cast<TY *>(p.y) + r * p.ldy;
    if constexpr (VEC) {
      store_chunk<TY, 8>(row, c, v, n);
    } else {
      uint32_t o[2 * sizeof(TY)];
#pragma unroll
      for (int i = 0; i < 2 * (int)sizeof(TY); ++i)
        o[i] = sizeof(TY) == 4 ? __float_as_uint(v[i & 7]) : pack_bf16x2(v[(2 * i) & 7], v[(2 * i + 1) & 7]);
      store_shifted<4>(row + c, n == 8, lane > 0 && c > 0, lane < 31 && c + 16 <= p.cols, o);
      if (n < 8) store_chunk<TY, 8>(row, c, v, n);
    }
  }
}

template <bool VEC>
auto dropout_kernel_of(int x_type, int y_type) {
  const bool xb = x_type == GEMM_TYPE_BF16, yb = y_type == GEMM_TYPE_BF16;
  return xb ? yb ? dropout_kernel<bf16, bf16, VEC> : dropout_kernel<bf16, float, VEC>
            : yb ? dropout_kernel<float, bf16, VEC> : dropout_kernel<float, float, VEC>;
}

}  // namespace

cudaError_t launch_dropout(const Dropout &p, cudaStream_t st) {
  const int64_t blocks = (p.rows * ((p.cols + 7) / 8) + kThreads - 1) / kThreads;
  const float scale = p.threshold < 65536 ? (float)(65536.0 / (65536 - p.threshold)) : 0.f;
  const auto on16 = [](const void *m, int64_t ld, int type) {
    return rows_on(m, ld, type == GEMM_TYPE_BF16 ? 2 : 4, 16);
  };
  const bool vec = on16(p.x, p.ldx, p.x_type) && on16(p.y, p.ldy, p.y_type) &&
                   (!p.residual || on16(p.residual, p.ldr, p.y_type));
  return launch_ex(vec ? dropout_kernel_of<true>(p.x_type, p.y_type) : dropout_kernel_of<false>(p.x_type, p.y_type),
                   dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(kThreads), 0, st, 1, p, scale);
}

}  // namespace gb300
