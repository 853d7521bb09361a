// layer_gate.cu -- the gated feed-forward block's gate: planning and staging of
// the kernel that takes it with the projections (gated_tc.cuh), and the kernel
// of its gradient alone.
#include <atomic>
#include <cmath>

#include "gate_math.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ------------------------------------------------------- the gradient alone

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

// --------------------------------------------- with a product: tiles, staging

// Modelled cost of a tile shape: microseconds per k-block of 64 and per tile
// besides.
struct TileCost {
  GatedTile tile;
  double kb_us, tile_us;
};
constexpr TileCost kForwardTiles[] = {{{true, 256}, 0.36, 2.0}, {{false, 128}, 0.33, 1.2}};
constexpr TileCost kBackwardTiles[] = {{{true, 256}, 0.36, 3.0}, {{false, 128}, 0.33, 2.0}, {{false, 64}, 0.30, 1.5}};

struct GatedPlan {
  GatedTile tile;
  int tiles_m, tiles_n, grid;
};
template <size_t N>
GatedPlan plan_gated(const TileCost (&tiles)[N], int64_t T, int64_t K, int64_t F, bool forward, int sms, int pairs) {
  GatedPlan best{};
  double best_us = -1;
  const int64_t num_kb = ceil_div64(K, kBK);
  for (const TileCost &c : tiles) {
    const int64_t slots = c.tile.pair ? pairs : sms;
    if (slots <= 0) continue;
    const int64_t tm = ceil_div64(T, c.tile.pair ? 2 * kBM : kBM), tn = ceil_div64(F, forward ? c.tile.bn / 2 : c.tile.bn);
    const int64_t rounds = ceil_div64(tm * tn, slots);
    const double us = rounds * (num_kb * c.kb_us + c.tile_us);
    if (best_us >= 0 && us >= best_us) continue;
    best_us = us;
    best.tile = c.tile;
    best.tiles_m = (int)tm;
    best.tiles_n = (int)tn;
    best.grid = (int)(tm * tn < slots ? tm * tn : slots) * (c.tile.pair ? 2 : 1);
  }
  return best;
}

// An operand as TMA can read it: as it is, or (rows off 16 bytes) copied into
// the stream's scratch at `at`.
struct Operand {
  const uint16_t *p;
  int64_t rows, cols, ld;
  bool pack() const { return !rows_on(p, ld, 2, 16); }
  int64_t packed_ld() const { return (cols + 7) / 8 * 8; }
  size_t bytes() const { return pack() ? align256((size_t)rows * packed_ld() * 2) : 0; }
};
cudaError_t stage(Operand &o, uint8_t *&at, const OpContext &c) {
  if (!o.pack()) return cudaSuccess;
  uint16_t *dst = reinterpret_cast<uint16_t *>(at);
  at += o.bytes();
  count_launches(1);
  const cudaError_t e = launch_pack_u16(o.p, o.rows, o.cols, o.ld, dst, o.packed_ld(), c.sms, c.st);
  o.ld = o.packed_ld();
  o.p = dst;
  return e;
}

// Stages the n operands (the first is A, the others weights of layout km),
// makes their maps and the outputs', and launches.
gemm_status_t run_gated(const GatedPlan &pl, Operand *o, int n, bool km, bool forward, GatedTcParams &p,
                        const OpContext &c) {
  if (pl.grid <= 0) return GEMM_ERR_CUDA;
  size_t need = 0;
  for (int i = 0; i < n; ++i) need += o[i].bytes();
  void *ws = nullptr;
  if (need) {
    const gemm_status_t s = op_workspace(need, c.st, &ws);
    if (s != GEMM_OK) return s;
  }
  uint8_t *at = static_cast<uint8_t *>(ws);
  for (int i = 0; i < n; ++i)
    if (stage(o[i], at, c) != cudaSuccess) return GEMM_ERR_CUDA;
  GatedMaps m;
  if (!bf16_box_map(&m.a, o[0].p, (uint64_t)o[0].cols, (uint64_t)o[0].rows, (uint64_t)o[0].ld, kBK, kBM))
    return GEMM_ERR_CUDA;
  const int cta_n = pl.tile.pair ? pl.tile.bn / 2 : pl.tile.bn;
  const uint32_t part = (uint32_t)(forward && !pl.tile.pair ? cta_n / 2 : cta_n);
  for (int i = 1; i < n; ++i)
    if (!bf16_box_map(&m.b[i - 1], o[i].p, (uint64_t)o[i].cols, (uint64_t)o[i].rows, (uint64_t)o[i].ld, km ? kBK : 64,
                      km ? part : kBK))
      return GEMM_ERR_CUDA;
  if (n < 3) m.b[1] = m.b[0];
  // outputs through TMA where their rows are whole 16-byte pieces (a clipped
  // store would write into a row's padding), and G and U, read in such pieces
  // then, likewise
  p.tma = tma_store_enabled() && p.F % 8 == 0;
  for (int i = 0; i < 3; ++i)
    if (p.out[i]) p.tma = p.tma && rows_on(p.out[i], p.ldout[i], 2, 16);
  if (p.gate) p.tma = p.tma && rows_on(p.gate, p.ldgate, 2, 16) && rows_on(p.up, p.ldup, 2, 16);
  for (int i = 0; i < 3; ++i) {
    m.out[i] = m.a;
    if (p.tma && p.out[i] &&
        !float_out_map(&m.out[i], true, p.out[i], (uint64_t)p.F, (uint64_t)p.T, (uint64_t)p.ldout[i], 1))
      return GEMM_ERR_CUDA;
  }
  p.tiles_m = pl.tiles_m;
  p.tiles_n = pl.tiles_n;
  p.num_kb = (int)ceil_div64(p.K, kBK);
  p.group_m = 8;
  p.q_vec = p.ck.q && rows_on(p.ck.q, p.ck.ldq, 1, 16);
  p.err = c.err;
  p.wait_limit_ns = c.wait_limit_ns;
  count_launches(1);
  const cudaError_t e = forward ? launch_gated_tc_fwd(pl.tile, km, m, p, pl.grid, c.st)
                                : launch_gated_tc_bwd(pl.tile, km, m, p, pl.grid, c.st);
  return e == cudaSuccess ? GEMM_OK : GEMM_ERR_CUDA;
}

}  // namespace

gemm_status_t gated_forward(const GatedForward &p, const OpContext &c) {
  if (p.K == 0) {
    uint16_t *out[3] = {p.h, p.g, p.u};
    const int64_t ld[3] = {p.ldh, p.ldg, p.ldu};
    for (int i = 0; i < 3; ++i) {
      if (!out[i]) continue;
      count_launches(1);
      if (launch_zero_fill(out[i], p.T, p.F, ld[i], 2, c.sms, c.st) != cudaSuccess) return GEMM_ERR_CUDA;
    }
    return GEMM_OK;
  }
  const int64_t wr = p.w_kmajor ? p.F : p.K, wc = p.w_kmajor ? p.K : p.F;
  Operand o[3] = {{p.x, p.T, p.K, p.ldx}, {p.wg, wr, wc, p.ldwg}, {p.wu, wr, wc, p.ldwu}};
  GatedTcParams t{};
  t.T = (int)p.T, t.F = p.F, t.K = p.K, t.act = p.act;
  t.out[0] = p.h, t.out[1] = p.g, t.out[2] = p.u;
  t.ldout[0] = p.ldh, t.ldout[1] = p.ldg, t.ldout[2] = p.ldu;
  return run_gated(plan_gated(kForwardTiles, p.T, p.K, p.F, true, c.sms, pair_slots()), o, 3, p.w_kmajor, true, t, c);
}

gemm_status_t gated_down_backward(const GatedDownBackward &p, const OpContext &c) {
  const GatedBackward &b = p.b;
  const int64_t wr = p.w_kmajor ? b.F : p.N, wc = p.w_kmajor ? p.N : b.F;
  Operand o[2] = {{p.d, b.T, p.N, p.ldd}, {p.w, wr, wc, p.ldw}};
  GatedTcParams t{};
  t.T = (int)b.T, t.F = b.F, t.K = p.N, t.act = b.act;
  t.out[0] = b.dg, t.out[1] = b.du;
  t.ldout[0] = b.lddg, t.ldout[1] = b.lddu;
  t.gate = b.g, t.up = b.u, t.ldgate = b.ldg, t.ldup = b.ldu;
  t.ck = b.ck;
  return run_gated(plan_gated(kBackwardTiles, b.T, p.N, b.F, false, c.sms, pair_slots()), o, 2, p.w_kmajor, false, t,
                   c);
}

cudaError_t launch_gated_backward(const GatedBackward &p, cudaStream_t st) {
  const int64_t blocks = (p.T * ((p.F + 31) / 32) + 7) / 8;
  const auto kern = p.act == GEMM_ACT_SILU        ? gated_backward_kernel<GEMM_ACT_SILU>
                    : p.act == GEMM_ACT_GELU      ? gated_backward_kernel<GEMM_ACT_GELU>
                    : p.act == GEMM_ACT_GELU_TANH ? gated_backward_kernel<GEMM_ACT_GELU_TANH>
                                                  : gated_backward_kernel<GEMM_ACT_RELU>;
  return launch_ex(kern, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(256), 0, st, 1, p);
}

}  // namespace gb300
