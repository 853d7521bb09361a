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

constexpr int kThreads = 256;

// A thread takes half a block of the checkpoint: 16 consecutive values of a
// row, its neighbouring lane the other half; they exchange the largest
// magnitude with one shuffle.  VEC: all rows start on 16 bytes; else values are
// shifted between registers and the 16-byte pieces of memory that they lie in.
template <int ACT, bool VEC>
__global__ void __launch_bounds__(kThreads) gated_backward_kernel(const GatedBackward p, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t halves = (cols + 31) / 32 * 2, items = p.T * halves, step = (int64_t)gridDim.x * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t h0 = (int64_t)blockIdx.x * kThreads; h0 < items; h0 += step) {
    // items is even, so both lanes of a block are in range or neither is
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    int64_t r, c;
    half_block(live ? h : items - 1, halves, &r, &c);
    const int n = !live || c >= cols ? 0 : (int)min((int64_t)16, cols - c);
    const auto load = [&](const uint16_t *m, int64_t ld) {
      const uint16_t *row = m + r * ld;
      Chunk<bf16, 16> v;
      if (n < 16)
        v.load_part(row, c, n);
      else if constexpr (VEC)
        v.load(row, c);
      else
        load_half(row + c, c == 0, (cols - c - 16) * 2, v.w);
      return v;
    };
    Chunk<bf16, 16> d;
    if (p.dh)
      d = load(p.dh, p.lddh);
    else
      d.load_part(nullptr, 0, 0);
    const Chunk<bf16, 16> g = load(p.g, p.ldg), u = load(p.u, p.ldu);
    uint32_t dg[8], du[8];
    float2 v[8];  // act(g) * u
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 di = d.get2(i), gi = g.get2(i), ui = u.get2(i);
      const GateValue a = gate<ACT, true>(gi.x), b = gate<ACT, true>(gi.y);
      dg[i] = pack_bf16x2(di.x * ui.x * a.slope, di.y * ui.y * b.slope);
      du[i] = pack_bf16x2(di.x * a.a, di.y * b.a);
      v[i] = make_float2(a.a * ui.x, b.a * ui.y);
      top = max(top, max(__float_as_uint(v[i].x) & 0x7FFFFFFFu, __float_as_uint(v[i].y) & 0x7FFFFFFFu));
    }
    const auto store = [&](uint16_t *m, int64_t ld, const uint32_t(&w)[8]) {
      uint16_t *row = m + r * ld;
      if constexpr (VEC) {
        if (n == 16) store_32_bytes(row + c, w);
      } else {
        store_shifted<4>(row + c, n == 16, lane > 0 && c > 0, lane < 31 && c + 32 <= cols, w);
      }
      if (n < 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i < n) row[c + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
      }
    };
    store(p.dg, p.lddg, dg);
    store(p.du, p.lddu, du);
    if (!p.ck.q) continue;
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t e = q8_exponent(top);
    float2 lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) lo[j] = v[j], hi[j] = v[4 + j];
    const uint2 wl = q8_pack8(lo, e), wh = q8_pack8(hi, e);
    const uint32_t w[4] = {wl.x, wl.y, wh.x, wh.y};
    int8_t *q = p.ck.q + r * p.ck.ldq + c;
    if constexpr (VEC) {
      if (n == 16) *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      store_shifted<4>(q, n == 16, lane > 0 && c > 0, lane < 31 && c + 32 <= cols, w);
    }
    if (n < 16) store_bytes(q, w, n);
    if (live && (h & 1) == 0) p.ck.e[r * p.ck.lde + (c >> 5)] = (uint8_t)e;
  }
}

template <bool VEC>
auto backward_kernel(int act) {
  return act == GEMM_ACT_SILU        ? gated_backward_kernel<GEMM_ACT_SILU, VEC>
         : act == GEMM_ACT_GELU      ? gated_backward_kernel<GEMM_ACT_GELU, VEC>
         : act == GEMM_ACT_GELU_TANH ? gated_backward_kernel<GEMM_ACT_GELU_TANH, VEC>
                                     : gated_backward_kernel<GEMM_ACT_RELU, VEC>;
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
// makes their maps, and launches.
gemm_status_t run_gated(const GatedPlan &pl, Operand *o, int n, bool km, bool forward, GatedTcParams &p,
                        const OpContext &c) {
  const bool few = forward && p.T <= kFewTokens;
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
  if (!bf16_box_map(&m.a, o[0].p, (uint64_t)o[0].cols, (uint64_t)o[0].rows, (uint64_t)o[0].ld, kBK,
                    few ? (uint32_t)gated_few_columns(p.T) : kBM))
    return GEMM_ERR_CUDA;
  const int cta_n = pl.tile.pair ? pl.tile.bn / 2 : pl.tile.bn;
  const uint32_t part = few ? 64u : (uint32_t)(forward && !pl.tile.pair ? cta_n / 2 : cta_n);
  for (int i = 1; i < n; ++i)
    if (!bf16_box_map(&m.b[i - 1], o[i].p, (uint64_t)o[i].cols, (uint64_t)o[i].rows, (uint64_t)o[i].ld, km ? kBK : 64,
                      km ? part : kBK))
      return GEMM_ERR_CUDA;
  if (n < 3) m.b[1] = m.b[0];
  p.num_kb = (int)ceil_div64(p.K, kBK);
  p.err = c.err;
  p.wait_limit_ns = c.wait_limit_ns;
  if (few) {
    count_launches(1);
    return launch_gated_few(km, m, p, c.sms, c.st) == cudaSuccess ? GEMM_OK : GEMM_ERR_CUDA;
  }
  p.vec = p.F % 8 == 0 && (!p.gate || (rows_on(p.gate, p.ldgate, 2, 16) && rows_on(p.up, p.ldup, 2, 16)));
  for (int i = 0; i < 3; ++i)
    if (p.out[i]) p.vec = p.vec && rows_on(p.out[i], p.ldout[i], 2, 16);
  p.tiles_m = pl.tiles_m;
  p.tiles_n = pl.tiles_n;
  p.group_m = 8;
  p.q_vec = p.ck.q && rows_on(p.ck.q, p.ck.ldq, 1, 16);
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
  const auto on16 = [&](const void *m, int64_t ld) { return rows_on(m, ld, 2, 16); };
  const bool vec = (!p.dh || on16(p.dh, p.lddh)) && on16(p.g, p.ldg) && on16(p.u, p.ldu) && on16(p.dg, p.lddg) &&
                   on16(p.du, p.lddu) && (!p.ck.q || rows_on(p.ck.q, p.ck.ldq, 1, 16));
  const int64_t blocks = ceil_div64(p.T * (ceil_div64(p.F, 32) * 2), kThreads);
  return launch_ex(vec ? backward_kernel<true>(p.act) : backward_kernel<false>(p.act),
                   dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(kThreads), 0, st, 1, p, (int64_t)p.F);
}

}  // namespace gb300
