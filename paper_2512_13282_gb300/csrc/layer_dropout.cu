// layer_dropout.cu -- dropout with a residual, and its gradient.
//
// Whether the value at (row, column) is kept is a function of the key, the
// step and its place: one Philox4x32-10 block (ten rounds of two 32 x 32 -> 64
// bit products) gives eight 16-bit numbers, those of eight neighbouring
// columns.  Sixteen bits a value and not 32: the generator's instructions are
// the kernel's, half as many, and P is exact to 2^-17.
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

// A thread takes eight values of a row, element by element.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const Dropout p, float scale) {
  griddep_launch_dependents();
  griddep_wait();
  const uint64_t step = p.step + (p.step_device ? *p.step_device : 0);
  const int64_t groups = (p.cols + 7) / 8, items = p.rows * groups;
  for (int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x; t < items; t += (int64_t)gridDim.x * kThreads) {
    const int64_t r = t / groups, c = (t - r * groups) * 8;
    const uint4 w = philox((uint32_t)(c >> 3), (uint32_t)r, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)p.seed,
                           (uint32_t)(p.seed >> 32));
    const uint32_t n[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c + i >= p.cols) break;
      const bool keep = ((n[i / 2] >> (16 * (i & 1))) & 0xFFFFu) >= p.threshold;
      const float v = keep ? load_value<TX>(p.x, r * p.ldx + c + i) * scale : 0.f;
      const float b = p.residual ? load_value<TY>(p.residual, r * p.ldr + c + i) : 0.f;
      store_value<TY>(p.y, r * p.ldy + c + i, b + v);
    }
  }
}

}  // namespace

cudaError_t launch_dropout(const Dropout &p, cudaStream_t st) {
  const int64_t blocks = (p.rows * ((p.cols + 7) / 8) + kThreads - 1) / kThreads;
  const float scale = p.threshold < 65536 ? (float)(65536.0 / (65536 - p.threshold)) : 0.f;
  const bool xb = p.x_type == GEMM_TYPE_BF16, yb = p.y_type == GEMM_TYPE_BF16;
  const auto kern = xb ? yb ? dropout_kernel<bf16, bf16> : dropout_kernel<bf16, float>
                       : yb ? dropout_kernel<float, bf16> : dropout_kernel<float, float>;
  return launch_ex(kern, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(kThreads), 0, st, 1, p, scale);
}

}  // namespace gb300
