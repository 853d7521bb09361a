// layer_gate.cu -- the gated feed-forward block's gate: both projections with
// it, and its gradient with and without the down projection's product.
#include "gate_math.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kTile = 32;

// A 32 x 32 tile of A . B^T (A rows x K, K contiguous; B(k, c) at b[k * sk +
// c * sc]) a block of 16 x 16 threads, 2 x 2 sums a thread (rows ty + 16 i,
// columns tx + 16 j).
__device__ __forceinline__ void tile_product(const uint16_t *a, int64_t lda, int64_t rows, const uint16_t *b, int64_t sk,
                                             int64_t sc, int cols, int K, int64_t r0, int c0, float (&acc)[2][2],
                                             float (*as)[kTile + 1], float (*bs)[kTile + 1]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int k0 = 0; k0 < K; k0 += kTile) {
    for (int i = threadIdx.x; i < kTile * kTile; i += 256) {
      const int y = i / kTile, x = i % kTile;
      as[y][x] = r0 + y < rows && k0 + x < K ? load_value<bf16>(a, (r0 + y) * lda + k0 + x) : 0.f;
      const int k = sc == 1 ? y : x, c = sc == 1 ? x : y;  // along the contiguous index
      bs[k][c] = k0 + k < K && c0 + c < cols ? load_value<bf16>(b, (k0 + k) * sk + (c0 + c) * sc) : 0.f;
    }
    __syncthreads();
#pragma unroll 8
    for (int k = 0; k < kTile; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = fmaf(as[ty + 16 * i][k], bs[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
}

template <int ACT>
__global__ void __launch_bounds__(256) gated_forward_kernel(const GatedForward p) {
  griddep_launch_dependents();
  griddep_wait();
  __shared__ float as[kTile][kTile + 1], bs[kTile][kTile + 1];
  const int64_t r0 = (int64_t)blockIdx.x * kTile;
  const int c0 = blockIdx.y * kTile, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float g[2][2] = {}, u[2][2] = {};
  const auto sk = [&](int64_t ld) { return p.w_kmajor ? (int64_t)1 : ld; };
  const auto sc = [&](int64_t ld) { return p.w_kmajor ? ld : (int64_t)1; };
  tile_product(p.x, p.ldx, p.T, p.wg, sk(p.ldwg), sc(p.ldwg), p.F, p.K, r0, c0, g, as, bs);
  tile_product(p.x, p.ldx, p.T, p.wu, sk(p.ldwu), sc(p.ldwu), p.F, p.K, r0, c0, u, as, bs);
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) {
      const int64_t r = r0 + ty + 16 * i;
      const int c = c0 + tx + 16 * j;
      if (r >= p.T || c >= p.F) continue;
      store_value<bf16>(p.h, r * p.ldh + c, gate<ACT, false>(g[i][j]).a * u[i][j]);
      if (!p.g) continue;
      store_value<bf16>(p.g, r * p.ldg + c, g[i][j]);
      store_value<bf16>(p.u, r * p.ldu + c, u[i][j]);
    }
}

// Gradient of one element; returns act(g) * u.
template <int ACT>
__device__ __forceinline__ float gate_backward(const GatedBackward &p, int64_t r, int c, float dh) {
  const float g = load_value<bf16>(p.g, r * p.ldg + c), u = load_value<bf16>(p.u, r * p.ldu + c);
  const GateValue v = gate<ACT, true>(g);
  store_value<bf16>(p.dg, r * p.lddg + c, dh * u * v.slope);
  store_value<bf16>(p.du, r * p.lddu + c, dh * v.a);
  return v.a * u;
}

// The checkpoint of 32 values, one a lane (0 past the row's end).
__device__ __forceinline__ void q8_by_warp(const Q8Ref &ck, int64_t r, int c, int cols, float h) {
  uint32_t top = c < cols ? __float_as_uint(h) & 0x7FFFFFFFu : 0u;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (c >= cols) return;
  const uint32_t e = q8_exponent(top);
  ck.q[r * ck.ldq + c] = (int8_t)q8_byte(h, q8_inverse(e), e);
  if ((c & 31) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)e;
}

// A warp per 32 values of a row.
template <int ACT>
__global__ void __launch_bounds__(256) gated_backward_kernel(const GatedBackward p) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31, groups = (p.F + 31) / 32;
  const int64_t items = p.T * groups;
  for (int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); t < items; t += (int64_t)gridDim.x * 8) {
    const int64_t r = t / groups;
    const int c = (int)(t - r * groups) * 32 + lane;
    float h = 0.f;
    if (c < p.F) h = gate_backward<ACT>(p, r, c, p.dh ? load_value<bf16>(p.dh, r * p.lddh + c) : 0.f);
    if (p.ck.q) q8_by_warp(p.ck, r, c, p.F, h);
  }
}

template <int ACT>
__global__ void __launch_bounds__(256) gated_down_backward_kernel(const GatedDownBackward p) {
  griddep_launch_dependents();
  griddep_wait();
  __shared__ float as[kTile][kTile + 1], bs[kTile][kTile + 1];
  const int64_t r0 = (int64_t)blockIdx.x * kTile;
  const int c0 = blockIdx.y * kTile, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float dh[2][2] = {};
  tile_product(p.d, p.ldd, p.b.T, p.w, p.w_kmajor ? 1 : p.ldw, p.w_kmajor ? p.ldw : 1, p.b.F, p.N, r0, c0, dh, as, bs);
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) as[ty + 16 * i][tx + 16 * j] = dh[i][j];
  __syncthreads();
  const int c = c0 + (threadIdx.x & 31);
  for (int y = threadIdx.x >> 5; y < kTile; y += 8) {
    const int64_t r = r0 + y;
    if (r >= p.b.T) break;
    float h = 0.f;
    if (c < p.b.F) h = gate_backward<ACT>(p.b, r, c, as[y][threadIdx.x & 31]);
    if (p.b.ck.q) q8_by_warp(p.b.ck, r, c, p.b.F, h);
  }
}

}  // namespace

cudaError_t launch_gated_forward(const GatedForward &p, const OpContext &c) {
  const dim3 grid((unsigned)((p.T + kTile - 1) / kTile), (unsigned)((p.F + kTile - 1) / kTile));
  cudaError_t e = cudaSuccess;
  with_activation(p.act, [&](auto act) {
    e = launch_ex(gated_forward_kernel<decltype(act)::value>, grid, dim3(256), 0, c.st, 1, p);
  });
  return e;
}

cudaError_t launch_gated_backward(const GatedBackward &p, cudaStream_t st) {
  const int64_t blocks = (p.T * ((p.F + 31) / 32) + 7) / 8;
  cudaError_t e = cudaSuccess;
  with_activation(p.act, [&](auto act) {
    e = launch_ex(gated_backward_kernel<decltype(act)::value>, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))),
                  dim3(256), 0, st, 1, p);
  });
  return e;
}

cudaError_t launch_gated_down_backward(const GatedDownBackward &p, const OpContext &c) {
  const dim3 grid((unsigned)((p.b.T + kTile - 1) / kTile), (unsigned)((p.b.F + kTile - 1) / kTile));
  cudaError_t e = cudaSuccess;
  with_activation(p.b.act, [&](auto act) {
    e = launch_ex(gated_down_backward_kernel<decltype(act)::value>, grid, dim3(256), 0, c.st, 1, p);
  });
  return e;
}

}  // namespace gb300
