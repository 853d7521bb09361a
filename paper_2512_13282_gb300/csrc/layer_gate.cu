// layer_gate.cu -- the gated feed-forward block's gate: planning and staging of
// the kernel that takes it with the projections (gated_tc.cuh), and the kernel
// of its gradient alone.
#include <cstdio>

#include "gate_math.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ------------------------------------------------------- the gradient alone

constexpr int kThreads = 256;

// A thread takes V = 16 or 8 consecutive values of a row, two or four
// neighbouring lanes a block of the checkpoint; they exchange its largest
// magnitude with shuffles.  VEC: all rows start on 16 bytes (the checkpoint's on
// 8); else values are shifted between registers and the 16-byte pieces of memory
// that they lie in.
// The bytes bound many values (8192 x 11008 silu with the checkpoint: 141 us, 7.1
// TB/s), a thread's own chain of instructions few, for which V is 8.
template <int ACT, bool VEC, int V>
__global__ void __launch_bounds__(kThreads) gated_backward_kernel(const GatedBackward p, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  constexpr int kLanes = 32 / V;  // of a block
  const int64_t pieces = (cols + 31) / 32 * kLanes, items = p.T * pieces, step = (int64_t)gridDim.x * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t h0 = (int64_t)blockIdx.x * kThreads; h0 < items; h0 += step) {
    // items is a multiple of kLanes, so the lanes of a block are all in range or none
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    int64_t r, c;
    row_piece<V>(live ? h : items - 1, pieces, &r, &c);
    const int n = !live || c >= cols ? 0 : (int)min((int64_t)V, cols - c);
    const auto load = [&](const uint16_t *m, int64_t ld) {
      const uint16_t *row = m + r * ld;
      Chunk<bf16, V> v;
      if (n < V)
        v.load_part(row, c, n);
      else if constexpr (VEC)
        v.load(row, c);
      else
        load_half(row + c, c == 0, (cols - c - V) * 2, v.w);
      return v;
    };
    Chunk<bf16, V> d;
    if (p.dh)
      d = load(p.dh, p.lddh);
    else
      d.load_part(nullptr, 0, 0);
    const Chunk<bf16, V> g = load(p.g, p.ldg), u = load(p.u, p.ldu);
    uint32_t dg[V / 2], du[V / 2];
    float2 v[V / 2];  // act(g) * u
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float2 di = d.get2(i), gi = g.get2(i), ui = u.get2(i);
      const GateValue a = gate<ACT, true>(gi.x), b = gate<ACT, true>(gi.y);
      dg[i] = pack_bf16x2(di.x * ui.x * a.slope, di.y * ui.y * b.slope);
      du[i] = pack_bf16x2(di.x * a.a, di.y * b.a);
      v[i] = make_float2(a.a * ui.x, b.a * ui.y);
      top = max(top, max(__float_as_uint(v[i].x) & 0x7FFFFFFFu, __float_as_uint(v[i].y) & 0x7FFFFFFFu));
    }
    const bool joined = lane > 0 && c > 0, taken = lane < 31 && c + 2 * V <= cols;
    const auto store = [&](uint16_t *m, int64_t ld, const uint32_t(&w)[V / 2]) {
      uint16_t *row = m + r * ld;
      if constexpr (!VEC) {
        store_shifted<4>(row + c, n == V, joined, taken, w);
      } else if (n == V) {
        if constexpr (V == 16)
          store_32_bytes(row + c, w);
        else
          *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if (n < V) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < n) row[c + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
      }
    };
    store(p.dg, p.lddg, dg);
    store(p.du, p.lddu, du);
    if (!p.ck.q) continue;
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t e = q8_exponent(top);
    uint32_t w[V / 4];
#pragma unroll
    for (int k = 0; k < V / 8; ++k) {
      const float2 eight[4] = {v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
      const uint2 q = q8_pack8(eight, e);
      w[2 * k] = q.x, w[2 * k + 1] = q.y;
    }
    int8_t *q = p.ck.q + r * p.ck.ldq + c;
    if constexpr (!VEC) {
      store_shifted<V / 4>(q, n == V, joined, taken, w);
    } else if (n == V) {
      if (V == 16 && (reinterpret_cast<uintptr_t>(q) & 15) == 0) {
        *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[V / 4 - 2], w[V / 4 - 1]);
      } else {
#pragma unroll
        for (int k = 0; k < V / 8; ++k) reinterpret_cast<uint2 *>(q)[k] = make_uint2(w[2 * k], w[2 * k + 1]);
      }
    }
    if (n < V) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) q[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
    }
    if (live && (c & 31) == 0) p.ck.e[r * p.ck.lde + (c >> 5)] = (uint8_t)e;
  }
}

template <bool VEC, int V>
auto backward_kernel(int act) {
  return act == GEMM_ACT_SILU        ? gated_backward_kernel<GEMM_ACT_SILU, VEC, V>
         : act == GEMM_ACT_GELU      ? gated_backward_kernel<GEMM_ACT_GELU, VEC, V>
         : act == GEMM_ACT_GELU_TANH ? gated_backward_kernel<GEMM_ACT_GELU_TANH, VEC, V>
                                     : gated_backward_kernel<GEMM_ACT_RELU, VEC, V>;
}

// --------------------------------------------- with a product: tiles, staging

// Modelled cost of a tile shape: microseconds per k-block of 64, per unit
// besides, and of the last unit's epilogue, which nothing hides.  Fitted to
// forced plans on GB300 (19 sizes a direction).  Against all forced plans of 90
// random sizes a direction (65 to 8192 tokens, reductions of 256 to 8192, 256 to
// 12288 features; in graphs, on rotating operands) what the model picks is off the
// fastest by 0.6 % forward and 2.5 % backward on average, by 11 and 22 % at most.
struct TileCost {
  GatedTile tile;
  double kb_us, unit_us, last_us;
};
constexpr TileCost kForwardTiles[] = {{{true, 256}, 0.345, 0.5, 5.0}, {{false, 128}, 0.31, 0.5, 3.0}};
constexpr TileCost kBackwardTiles[] = {
    {{true, 256}, 0.345, 4.5, 12.0}, {{false, 128}, 0.31, 2.0, 6.0}, {{false, 64}, 0.28, 1.5, 4.0}};
// A split tail besides: the reduction's launch, the partials written and read.
// After whole rounds its units wait for the slowest of them; where the tail is
// all there is they start at once, and backward the reduction takes the
// epilogue too, on all SMs.  2048 tokens 4096 x 11008 forward: 214 us whole, 204
// with a tail; one round of tiles, whole and split: 80 tokens 2048 x 1024 forward
// 12.6, 9.5, backward of 256 tokens 2048 x 1024 15.4, 10.2, 512 tokens 4096 x
// 2048 25.2, 20.9.
constexpr double kTailFixedUs = 6.0, kTailAloneForwardUs = 2.0, kTailAloneBackwardUs = 0.0, kTailUsPerMB = 0.36;

struct GatedPlan {
  GatedTile tile;
  int tiles_m, tiles_n, grid;
  int tail_first, tail_splits, tail_kb_per;
  int tile_m() const { return tile.pair ? 2 * kBM : kBM; }
  size_t partial_bytes() const {
    return (size_t)tail_splits * ((size_t)tiles_m * tiles_n - tail_first) * tile_m() * tile.bn * 4;
  }
};
// Tile shape, split tail and grid of the least modelled time, among those that
// the planner overrides leave: first with a forced tail (a split of 2 or more
// where the plan has a round to split), then without, then without a forced tile
// that is not compiled.
template <size_t N>
GatedPlan plan_gated(const TileCost (&tiles)[N], int64_t T, int64_t K, int64_t F, bool forward, int sms, int pairs) {
  GatedPlan best{};
  double best_us = -1;
  const int64_t num_kb = ceil_div64(K, kBK);
  const TileOverrides ovr = tile_overrides();
  for (int pass = ovr.tail_splits >= 2 ? 0 : 1; pass < 3 && best_us < 0; ++pass) {
    for (const TileCost &c : tiles) {
      if (pass < 2 && ((ovr.bn > 0 && ovr.bn != c.tile.bn) || (ovr.pair >= 0 && (ovr.pair != 0) != c.tile.pair))) continue;
      const int64_t slots = c.tile.pair ? pairs : sms;
      if (slots <= 0) continue;
      const int tile_m = c.tile.pair ? 2 * kBM : kBM;
      const int64_t tm = ceil_div64(T, tile_m), tn = ceil_div64(F, forward ? c.tile.bn / 2 : c.tile.bn), all = tm * tn;
      const int64_t full = all / slots, rem = all % slots;
      const double whole = num_kb * c.kb_us + c.unit_us;
      const int64_t first = pass == 0 ? ovr.tail_splits : 1, last = pass == 0 ? first : ovr.tail_splits == 0 ? 1 : 16;
      for (int64_t s = first; s <= last; ++s) {
        int64_t kb_per = num_kb, parts = 1;
        if (s > 1) {
          if (rem == 0 || rem * s > slots) break;
          kb_per = ceil_div64(num_kb, s);
          parts = ceil_div64(num_kb, kb_per);  // no part is empty
          if (parts != s || kb_per < 4) continue;
        }
        double us = full * whole;
        if (rem > 0) us += kb_per * c.kb_us + c.unit_us;
        us += c.last_us;
        const double tail_us = full > 0 ? kTailFixedUs : forward ? kTailAloneForwardUs : kTailAloneBackwardUs;
        if (parts > 1) us += tail_us + kTailUsPerMB * (double)parts * rem * tile_m * c.tile.bn * 4e-6;
        if (best_us >= 0 && us >= best_us) continue;
        best_us = us;
        best.tile = c.tile;
        best.tiles_m = (int)tm;
        best.tiles_n = (int)tn;
        best.tail_first = parts > 1 ? (int)(full * slots) : 0;
        best.tail_splits = parts > 1 ? (int)parts : 0;
        best.tail_kb_per = parts > 1 ? (int)kb_per : 0;
        const int64_t units = parts > 1 ? full * slots + rem * parts : all;
        best.grid = (int)(units < slots ? units : slots) * (c.tile.pair ? 2 : 1);
      }
    }
  }
  if (ovr.debug)
    std::fprintf(stderr, "[gb300_gemm] gated %s %lldx%lldx%lld: %s %d, %dx%d tiles, %d in whole, tail split in %d\n",
                 forward ? "forward" : "backward", (long long)T, (long long)K, (long long)F,
                 best.tile.pair ? "pair" : "single", best.tile.bn, best.tiles_m, best.tiles_n,
                 best.tail_splits ? best.tail_first : best.tiles_m * best.tiles_n, best.tail_splits);
  return best;
}

// An operand as TMA can read it: as it is, or (rows off 16 bytes) copied into
// the stream's scratch.
struct Operand {
  const uint16_t *p;
  int64_t rows, cols, ld;
  bool pack() const { return !rows_on(p, ld, 2, 16); }
  int64_t packed_ld() const { return (cols + 7) / 8 * 8; }
  size_t bytes() const { return pack() ? align256((size_t)rows * packed_ld() * 2) : 0; }
};

// The copies of up to three operands in one launch: a thread writes eight
// values (16 bytes), read in the 16-byte pieces of memory that they lie in.  The
// bytes bound it (two 4096 x 4096: 25 us, 5.4 TB/s read and written; four pieces a
// thread took twice as long).
struct PackJobs {
  struct {
    const uint16_t *src;
    uint16_t *dst;
    int64_t rows, cols, ld, ld_dst;
  } job[3];
  int jobs;
};
__global__ void __launch_bounds__(kThreads) gated_pack_kernel(const PackJobs j, int64_t items) {
  griddep_launch_dependents();
  griddep_wait();
  for (int64_t t0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; t0 < items; t0 += (int64_t)gridDim.x * kThreads) {
    int64_t t = t0;
    int i = 0;
    for (; i + 1 < j.jobs; ++i) {
      const int64_t n = j.job[i].rows * (j.job[i].ld_dst / 8);
      if (t < n) break;
      t -= n;
    }
    const auto &o = j.job[i];
    const int64_t per = o.ld_dst / 8;
    const int64_t r = t <= 0xFFFFFFFFll ? (int64_t)((uint32_t)t / (uint32_t)per) : t / per, c = (t - r * per) * 8;
    const uint16_t *row = o.src + r * o.ld;
    Chunk<bf16, 8> v;
    if (c + 8 <= o.cols)
      load_half(row + c, c == 0, (o.cols - c - 8) * 2, v.w);
    else
      v.load_part(row, c, (int)(o.cols - c));
    *reinterpret_cast<uint4 *>(o.dst + r * o.ld_dst + c) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  }
}
cudaError_t pack_operands(Operand *o, int n, uint8_t *at, const OpContext &c) {
  PackJobs j{};
  int64_t items = 0;
  for (int i = 0; i < n; ++i) {
    if (!o[i].pack()) continue;
    uint16_t *dst = reinterpret_cast<uint16_t *>(at);
    at += o[i].bytes();
    j.job[j.jobs++] = {o[i].p, dst, o[i].rows, o[i].cols, o[i].ld, o[i].packed_ld()};
    items += o[i].rows * (o[i].packed_ld() / 8);
    o[i].ld = o[i].packed_ld();
    o[i].p = dst;
  }
  if (j.jobs == 0) return cudaSuccess;
  count_launches(1);
  const int64_t blocks = ceil_div64(items, kThreads);
  return launch_ex(gated_pack_kernel, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(kThreads), 0, c.st,
                   1, j, items);
}

// Packs what has to be of the n operands (the first is A, the others weights of
// layout km), makes their maps, and launches: the kernel of few tokens, or the plan.
gemm_status_t run_gated(const GatedPlan &pl, Operand *o, int n, bool km, bool forward, GatedTcParams &p,
                        const OpContext &c) {
  const bool few = p.T <= kFewTokens;
  if (!few && pl.grid <= 0) return GEMM_ERR_CUDA;
  size_t packed = 0;
  for (int i = 0; i < n; ++i) packed += o[i].bytes();
  const size_t need = packed + (few ? 0 : pl.partial_bytes());
  void *ws = nullptr;
  if (need) {
    const gemm_status_t s = op_workspace(need, c.st, &ws);
    if (s != GEMM_OK) return s;
  }
  if (pack_operands(o, n, static_cast<uint8_t *>(ws), c) != cudaSuccess) return GEMM_ERR_CUDA;
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
  p.num_kb = (int)ceil_div64(o[0].cols, kBK);
  p.err = c.err;
  p.wait_limit_ns = c.wait_limit_ns;
  if (few) {
    count_launches(1);
    return launch_gated_few(forward, km, m, p, c.sms, c.st) == cudaSuccess ? GEMM_OK : GEMM_ERR_CUDA;
  }
  p.vec = p.F % 8 == 0 && (!p.gate || (rows_on(p.gate, p.ldgate, 2, 16) && rows_on(p.up, p.ldup, 2, 16)));
  for (int i = 0; i < 3; ++i)
    if (p.out[i]) p.vec = p.vec && rows_on(p.out[i], p.ldout[i], 2, 16);
  p.q_align = !p.ck.q ? 1 : rows_on(p.ck.q, p.ck.ldq, 1, 16) ? 16 : rows_on(p.ck.q, p.ck.ldq, 1, 8) ? 8 : 1;
  p.tiles_m = pl.tiles_m;
  p.tiles_n = pl.tiles_n;
  p.group_m = 8;
  p.tail_first = pl.tail_first;
  p.tail_splits = pl.tail_splits;
  p.tail_kb_per = pl.tail_kb_per;
  p.ws = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + packed);
  count_launches(1);
  const cudaError_t e = forward ? launch_gated_tc_fwd(pl.tile, km, m, p, pl.grid, c.st)
                                : launch_gated_tc_bwd(pl.tile, km, m, p, pl.grid, c.st);
  if (e != cudaSuccess) return GEMM_ERR_CUDA;
  if (pl.tail_splits > 0) {
    count_launches(1);
    if (launch_gated_tail(pl.tile, forward, p, c.st) != cudaSuccess) return GEMM_ERR_CUDA;
  }
  return GEMM_OK;
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
  t.T = (int)p.T, t.F = p.F, t.act = p.act;
  t.out[0] = p.h, t.out[1] = p.g, t.out[2] = p.u;
  t.ldout[0] = p.ldh, t.ldout[1] = p.ldg, t.ldout[2] = p.ldu;
  const GatedPlan pl =
      p.T > kFewTokens ? plan_gated(kForwardTiles, p.T, p.K, p.F, true, c.sms, pair_slots()) : GatedPlan{};
  return run_gated(pl, o, 3, p.w_kmajor, true, t, c);
}

gemm_status_t gated_down_backward(const GatedDownBackward &p, const OpContext &c) {
  const GatedBackward &b = p.b;
  const int64_t wr = p.w_kmajor ? b.F : p.N, wc = p.w_kmajor ? p.N : b.F;
  Operand o[2] = {{p.d, b.T, p.N, p.ldd}, {p.w, wr, wc, p.ldw}};
  GatedTcParams t{};
  t.T = (int)b.T, t.F = b.F, t.act = b.act;
  t.out[0] = b.dg, t.out[1] = b.du;
  t.ldout[0] = b.lddg, t.ldout[1] = b.lddu;
  t.gate = b.g, t.up = b.u, t.ldgate = b.ldg, t.ldup = b.ldu;
  t.ck = b.ck;
  const GatedPlan pl =
      b.T > kFewTokens ? plan_gated(kBackwardTiles, b.T, p.N, b.F, false, c.sms, pair_slots()) : GatedPlan{};
  return run_gated(pl, o, 2, p.w_kmajor, false, t, c);
}

cudaError_t launch_gated_backward(const GatedBackward &p, const OpContext &c) {
  const auto on16 = [&](const void *m, int64_t ld) { return rows_on(m, ld, 2, 16); };
  const bool vec = (!p.dh || on16(p.dh, p.lddh)) && on16(p.g, p.ldg) && on16(p.u, p.ldu) && on16(p.dg, p.lddg) &&
                   on16(p.du, p.lddu) && (!p.ck.q || rows_on(p.ck.q, p.ck.ldq, 1, 8));
  // eight values a thread while each has one piece: 100 x 1024 1.9 us (16: 2.25),
  // 2928 x 776 the same.  Unaligned, whose pieces overlap, only for very few: 56 x
  // 290 4.3 us (16: 5.5), 1000 x 1501 11.3 (8.4)
  const bool small = p.T * ceil_div64(p.F, 32) * 4 <= (int64_t)c.sms * (vec ? 2048 : 256);
  const int64_t blocks = ceil_div64(p.T * ceil_div64(p.F, 32) * (small ? 4 : 2), kThreads);
  const auto kern = small ? vec ? backward_kernel<true, 8>(p.act) : backward_kernel<false, 8>(p.act)
                          : vec ? backward_kernel<true, 16>(p.act) : backward_kernel<false, 16>(p.act);
  return launch_ex(kern, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(kThreads), 0, c.st, 1, p,
                   (int64_t)p.F);
}

}  // namespace gb300
