// gated_tail.cu -- the split tail of the gated feed-forward block's tensor-core
// kernel: the sums of a last, partly filled round's tiles, split in K so that
// they fill it, are added in split order, and the gate or its gradient is taken
// from them.  A thread has four columns of a row, eight lanes a block of the
// checkpoint; the partial sums' bytes, mostly in L2, bound it.
#include "gate_math.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

// Adds up four columns of the compact partials.
__device__ __forceinline__ float4 tail_sum(const GatedTcParams &p, const float *src, int64_t plane) {
  float4 s = *reinterpret_cast<const float4 *>(src);
  for (int k = 1; k < p.tail_splits; ++k) {
    const float4 v = *reinterpret_cast<const float4 *>(src + k * plane);
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  return s;
}

// tile_f: features of a tile, bn: columns of its partials.
template <bool FORWARD>
__global__ void __launch_bounds__(256)
    gated_tail_kernel(const GatedTcParams p, int tile_m, int tile_f, int bn, int64_t groups) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= groups) return;  // whole warps: groups is a multiple of 32
  const int per_row = tile_f / 4;
  const int64_t prow = t / per_row;
  const int pc = (int)(t - prow * per_row) * 4;
  const int slot = (int)(prow / tile_m);
  int tm, tn;
  raster_tile(p.tail_first + slot, p.tiles_m, p.tiles_n, p.group_m, &tm, &tn);
  const int64_t row = (int64_t)tm * tile_m + (prow - (int64_t)slot * tile_m);
  const int col = tn * tile_f + pc;
  const int n = row < p.T ? max(0, min(4, p.F - col)) : 0;
  const int64_t plane = (int64_t)(p.tiles_m * p.tiles_n - p.tail_first) * tile_m * bn;
  const float *src = p.ws + prow * bn + pc;
  const float4 s4 = tail_sum(p, src, plane);
  const float s[4] = {s4.x, s4.y, s4.z, s4.w};
  if constexpr (FORWARD) {
    const float4 u4 = tail_sum(p, src + tile_f, plane);
    const float u[4] = {u4.x, u4.y, u4.z, u4.w};
    float h[4];
    with_activation(p.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = gate<decltype(act)::value, false>(s[i]).a * u[i];
    });
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) {
        store_value<bf16>(p.out[0], row * p.ldout[0] + col + i, h[i]);
        if (p.out[1]) {
          store_value<bf16>(p.out[1], row * p.ldout[1] + col + i, s[i]);
          store_value<bf16>(p.out[2], row * p.ldout[2] + col + i, u[i]);
        }
      }
  } else {
    float g[4], u[4], h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[i] = i < n ? load_value<bf16>(p.gate, row * p.ldgate + col + i) : 0.f;
      u[i] = i < n ? load_value<bf16>(p.up, row * p.ldup + col + i) : 0.f;
    }
    with_activation(p.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const GateValue v = gate<decltype(act)::value, true>(g[i]);
        h[i] = v.a * u[i];
        g[i] = s[i] * u[i] * v.slope;
        u[i] = s[i] * v.a;
      }
    });
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) {
        store_value<bf16>(p.out[0], row * p.ldout[0] + col + i, g[i]);
        store_value<bf16>(p.out[1], row * p.ldout[1] + col + i, u[i]);
      }
    if (!p.ck.q) return;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(h[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t e = q8_exponent(top);
    const float inverse = q8_inverse(e);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p.ck.q[row * p.ck.ldq + col + i] = (int8_t)q8_byte(h[i], inverse, e);
    if (n > 0 && (col & 31) == 0) p.ck.e[row * p.ck.lde + (col >> 5)] = (uint8_t)e;
  }
}

}  // namespace

cudaError_t launch_gated_tail(const GatedTile &tile, bool forward, const GatedTcParams &p, cudaStream_t st) {
  const int tile_m = tile.pair ? 2 * kBM : kBM, tile_f = forward ? tile.bn / 2 : tile.bn;
  const int64_t tail = (int64_t)p.tiles_m * p.tiles_n - p.tail_first;
  const int64_t groups = tail * tile_m * (tile_f / 4);
  return launch_ex(forward ? gated_tail_kernel<true> : gated_tail_kernel<false>, dim3((unsigned)((groups + 255) / 256)),
                   dim3(256), 0, st, 1, p, tile_m, tile_f, tile.bn, groups);
}

}  // namespace gb300
