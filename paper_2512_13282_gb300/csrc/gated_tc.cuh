// gated_tc.cuh -- the persistent tcgen05 kernel of the gated feed-forward block,
// forward (H = act(X Wg) * (X Wu)) and backward (the gate's gradient from
// dH = dO Wd^T).
//
// Both are C = A . B with A row-major and a B of either layout, and run as
// gemm_tc2.cuh does (PAIR: a CTA pair per 256-row tile, each CTA holding 128
// rows of A and half of B; else one CTA per 128-row tile): a TMA producer, an
// MMA issuer and epilogue warps (four forward, eight backward), two accumulators
// in TMEM.  What differs:
//
// Forward.  A tile's BN columns are BN / 2 of the gate's projection and the
// same BN / 2 of the up projection's, so that one lane of the epilogue finds g
// and u of an element in its own TMEM lane, BN / 2 columns apart, and H leaves
// the kernel without G and U having been stored.  In a pair, one CTA's half of
// B is Wg's, the other's Wu's.
//
// Backward.  The epilogue warps bring blocks of G and U (32 x 32) into shared
// memory, take the gradient from dH and leave dG and dU in their place, from
// where they store them; and the checkpoint of act(G) U: a lane holds 32
// consecutive values of a row, which is one block of the checkpoint, so that
// needs no exchange between lanes.  dH is never stored: 8192 x 11008 would cost
// 360 MB of traffic, 53 us.
//
// The tensor cores bound both: 8192 tokens 4096 x 11008 forward with G and U kept
// 813 us in bursts (1.82 PFLOP/s), 917 back to back under the power cap; backward
// 480 and 530, a round of tiles 25 us where a plain GEMM's takes 21, since what the
// epilogue moves competes with the operands on their way from L2.
#pragma once
#include "gate_math.cuh"
#include "layer_rows.cuh"
#include "gemm_tc2.cuh"

namespace gb300 {

template <int BN, bool PAIR, bool BWD>
struct GatedCfg {
  static constexpr int kTileM = PAIR ? 2 * kBM : kBM;
  static constexpr int kTileF = BWD ? BN : BN / 2;   // features of a tile
  static constexpr int kCtaN = PAIR ? BN / 2 : BN;   // columns of B a CTA loads
  static constexpr int kPartN = BWD || PAIR ? kCtaN : kCtaN / 2;  // ... of one weight
  static_assert(kPartN % 64 == 0 && BN <= 256, "operands are assembled from 64-wide boxes");
  static constexpr int kEpiWarps = !BWD || BN == 64 ? 4 : 8;
  static constexpr int kThreads = (2 + kEpiWarps) * 32;
  static constexpr uint32_t kBBytes = kCtaN * kRowBytes;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  // a 32 x 32 block of each output; backward, of G and U, which become dG and dU
  static constexpr uint32_t kEpiWarpBytes = (BWD ? 2 : 3) * 2048u;
  static constexpr int kStages =
      (int)((232448u - 1024u - 256u - kEpiWarps * kEpiWarpBytes) / kStageBytes);
  static constexpr uint32_t kTmemCols = pow2_at_least(2 * BN);
  static constexpr int kChunks = kTileF / 32 / (kEpiWarps / 4);  // 32-column blocks of an epilogue warp
  static_assert(kChunks >= 1, "each warpgroup has a block");
  static constexpr uint32_t kEpiOffset = kStages * kStageBytes;
  static constexpr uint32_t kBarOffset = kEpiOffset + kEpiWarps * kEpiWarpBytes;
  static constexpr uint32_t kNumBars = 2 * kStages + 4 + 1;
  static constexpr uint32_t kSmemBytes = kBarOffset + kNumBars * 8 + 16 + 1024;
  static_assert(kNumBars * 8 + 16 <= 256 && kSmemBytes <= 232448, "shared memory per CTA is 227 KB");
  static_assert(kTmemCols <= 512, "TMEM has 512 columns");
};

// Blocks of 32 x 32 bf16 in an epilogue warp's shared memory: rows of 64 bytes,
// chunk j (16 bytes) of row r at chunk j ^ ((r / 2) % 4), so that neither a
// lane's row nor a warp's eight rows of four chunks meet in a bank.
__device__ __forceinline__ uint32_t block_chunk(uint32_t buf, int row, int j) {
  return buf + row * 64 + ((j ^ ((row >> 1) & 3)) << 4);
}
__device__ __forceinline__ uint32_t block_element(uint32_t buf, int row, int col) {
  return block_chunk(buf, row, col >> 3) + (col & 7) * 2;
}
__device__ __forceinline__ void put_row(uint32_t buf, int lane, const uint32_t (&h)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    st_shared_v4(block_chunk(buf, lane, j), h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
}
// A lane's 16 values from column 16 * k on.
__device__ __forceinline__ void get_row16(uint32_t buf, int lane, int k, uint32_t (&h)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint4 v = ld_shared_v4(block_chunk(buf, lane, 2 * k + j));
    h[4 * j] = v.x, h[4 * j + 1] = v.y, h[4 * j + 2] = v.z, h[4 * j + 3] = v.w;
  }
}
__device__ __forceinline__ void put_row16(uint32_t buf, int lane, int k, const uint32_t (&h)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
    st_shared_v4(block_chunk(buf, lane, 2 * k + j), h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
}
__device__ __forceinline__ void st_shared_u16(uint32_t addr, uint16_t v) {
  asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"(v) : "memory");
}
__device__ __forceinline__ uint16_t ld_shared_u16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t ld_shared_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// The block at (y0, x) between memory and shared memory, along rows: a lane's
// own row would be 32 lines touched by every access.  By the warps and not by
// TMA, whose engine the operands keep busy: blocks through it stretched a
// 256 x 256 tile of 4096 deep from 20.9 to 25 us (G, U, dG and dU; prefetches
// into L2 by it, to 33 to 40 us).
//
// Rows on 16 bytes, F a multiple of 8: 16-byte pieces, four lanes a row.
// block_fetch only asks for them (zero past the matrix); block_arrived waits.
__device__ __forceinline__ void block_fetch(const uint16_t *m, int64_t ld, uint32_t buf, int lane, int y0, int x, int T,
                                            int F) {
  const int j = lane & 3, c = x + 8 * j;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 2);
    const bool in = y0 + row < T && c < F;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(block_chunk(buf, row, j)),
                 "l"(__cvta_generic_to_global(in ? m + (int64_t)(y0 + row) * ld + c : m)), "r"(in ? 16 : 0)
                 : "memory");
  }
}
__device__ __forceinline__ void block_arrived() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
}
__device__ __forceinline__ void block_store(uint16_t *m, int64_t ld, uint32_t buf, int lane, int y0, int x, int T,
                                            int F) {
  const int j = lane & 3, c = x + 8 * j;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 2);
    const uint4 v = ld_shared_v4(block_chunk(buf, row, j));
    if (y0 + row < T && c < F) *reinterpret_cast<uint4 *>(m + (int64_t)(y0 + row) * ld + c) = v;
  }
}
// Any alignment: element by element, lane = column; both matrices in one batch
// of loads.
__device__ __forceinline__ void block_fetch_any(const uint16_t *m0, int64_t ld0, const uint16_t *m1, int64_t ld1,
                                                uint32_t buf0, uint32_t buf1, int lane, int y0, int x, int T, int F) {
  const int c = x + lane, rows = c < F ? min(32, T - y0) : 0;
  m0 += (int64_t)y0 * ld0 + c;
  m1 += (int64_t)y0 * ld1 + c;
  uint16_t v[32], w[32];
#pragma unroll
  for (int i = 0; i < 32; ++i, m0 += ld0, m1 += ld1) {
    v[i] = i < rows ? *m0 : (uint16_t)0;
    w[i] = i < rows ? *m1 : (uint16_t)0;
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    st_shared_u16(block_element(buf0, i, lane), v[i]);
    st_shared_u16(block_element(buf1, i, lane), w[i]);
  }
}
__device__ __forceinline__ void block_store_any(uint16_t *m, int64_t ld, uint32_t buf, int lane, int y0, int x, int T,
                                                int F) {
  const int c = x + lane, rows = min(32, T - y0);
  if (c >= F) return;
  m += (int64_t)y0 * ld + c;
#pragma unroll 8
  for (int i = 0; i < rows; ++i, m += ld) *m = ld_shared_u16(block_element(buf, i, lane));
}
__device__ __forceinline__ float bf16_at(const uint32_t (&w)[8], int i) {
  return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}

// Gradient of 16 elements of a row from dh (float32 bits): g and u become dg
// and du, dh becomes act(g) * u.
template <int ACT>
__device__ __forceinline__ void gate_backward16(uint32_t (&dh)[16], uint32_t (&g)[8], uint32_t (&u)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float dg[2], du[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float d = __uint_as_float(dh[2 * i + k]), uu = bf16_at(u, 2 * i + k);
      const GateValue v = gate<ACT, true>(bf16_at(g, 2 * i + k));
      dg[k] = d * uu * v.slope;
      du[k] = d * v.a;
      dh[2 * i + k] = __float_as_uint(v.a * uu);
    }
    g[i] = pack_bf16x2(dg[0], dg[1]);
    u[i] = pack_bf16x2(du[0], du[1]);
  }
}

// The checkpoint of 32 float32 values: their bytes, and the exponent.
__device__ __forceinline__ uint32_t q8_block32(const uint32_t (&h)[32], uint32_t (&q)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max(top, h[i] & 0x7FFFFFFFu);
  const uint32_t e = q8_exponent(top);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = make_float2(__uint_as_float(h[8 * j + 2 * i]), __uint_as_float(h[8 * j + 2 * i + 1]));
    const uint2 w = q8_pack8(v, e);
    q[2 * j] = w.x, q[2 * j + 1] = w.y;
  }
  return e;
}

// Work unit u -> tile, k-blocks, and whether its sums are partial ones.
struct GatedUnit {
  int tm, tn, kb0, kb1, split, slot;
  bool part;
};
__device__ __forceinline__ int gated_units(const GatedTcParams &p) {
  const int tiles = p.tiles_m * p.tiles_n;
  return p.tail_splits > 0 ? p.tail_first + (tiles - p.tail_first) * p.tail_splits : tiles;
}
__device__ __forceinline__ GatedUnit gated_unit(const GatedTcParams &p, int u) {
  GatedUnit w{0, 0, 0, p.num_kb, 0, 0, false};
  if (p.tail_splits > 0 && u >= p.tail_first) {
    const int tail = p.tiles_m * p.tiles_n - p.tail_first, v = u - p.tail_first;
    w.part = true;
    w.split = v / tail;
    w.slot = v - w.split * tail;
    w.kb0 = w.split * p.tail_kb_per;
    w.kb1 = min(p.num_kb, w.kb0 + p.tail_kb_per);
    u = p.tail_first + w.slot;
  }
  raster_tile(u, p.tiles_m, p.tiles_n, p.group_m, &w.tm, &w.tn);
  return w;
}

// A lane's 32 sums to its row of a partial block (128 bytes, a whole line).
__device__ __forceinline__ void store_partials(float *at, const uint32_t (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w[8] = {v[8 * j],     v[8 * j + 1], v[8 * j + 2], v[8 * j + 3],
                           v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]};
    store_32_bytes(at + 8 * j, w);
  }
}

template <int BN, bool PAIR, bool KM, bool BWD>
__global__ void __launch_bounds__(GatedCfg<BN, PAIR, BWD>::kThreads, 1)
    gated_tc_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB0,
                    const __grid_constant__ CUtensorMap tmB1, const GatedTcParams p) {
  using Cfg = GatedCfg<BN, PAIR, BWD>;
  constexpr int STAGES = Cfg::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;  // swizzle atoms need 1024-byte alignment
  uint8_t *base_ptr = smem_raw + (base - raw);
  const uint32_t sA = base;
  const uint32_t sB = base + STAGES * kABytes;
  const uint32_t bars = base + Cfg::kBarOffset;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(base_ptr + Cfg::kBarOffset + Cfg::kNumBars * 8);
  volatile uint32_t *abort_flag = tmem_slot + 1;

  auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bars + 8u * (STAGES + s); };
  auto accf_bar = [&](uint32_t b) { return bars + 8u * (2 * STAGES + b); };
  auto acce_bar = [&](uint32_t b) { return bars + 8u * (2 * STAGES + 2 + b); };
  const uint32_t drain_bar = bars + 8u * (2 * STAGES + 4);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const bool leader = rank == 0;
  const int first_unit = PAIR ? blockIdx.x >> 1 : blockIdx.x;
  const int unit_step = PAIR ? gridDim.x >> 1 : gridDim.x;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), (PAIR ? 2 : 1) * Cfg::kEpiWarps * 32);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0u;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB0);
    if (!BWD) tma_prefetch_desc(&tmB1);
  }
  __syncwarp();
  if (warp == 1) {
    if constexpr (PAIR)
      tmem_alloc_pair<Cfg::kTmemCols>(smem_addr(tmem_slot));
    else
      tmem_alloc<Cfg::kTmemCols>(smem_addr(tmem_slot));
  }
  tc_fence_before_sync();
  if constexpr (PAIR)
    cluster_sync_all();  // barriers of both CTAs initialised, TMEM allocated
  else
    __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // Nothing above touched global memory, so it may overlap the previous
  // kernel of the stream.
  griddep_wait();

  const int num_units = gated_units(p);
  constexpr uint64_t kDrainNs = 200ull * 1000 * 1000;

  if (warp == 0) {
    // -------------------------------------------------------- TMA producer
    if (lane == 0) {
      uint32_t g = 0;
      bool ok = true;
      for (int t = first_unit; ok && t < num_units; t += unit_step) {
        const GatedUnit w = gated_unit(p, t);
        const int m0 = w.tm * Cfg::kTileM + (int)rank * kBM;
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          const uint32_t s = g % STAGES, ph = (g / STAGES) & 1u;
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, p.err, p.wait_limit_ns)) {
            ok = false;
            break;
          }
          if (leader) mbar_arrive_expect_tx(full_bar(s), (PAIR ? 2 : 1) * Cfg::kStageBytes);
          const uint32_t fb = PAIR ? mapa_shared(full_bar(s), 0) : full_bar(s);
          const auto load = [&](uint32_t dst, const CUtensorMap *m, int c0, int c1) {
            if constexpr (PAIR)
              tma_load_2d_pair(dst, m, c0, c1, fb);
            else
              tma_load_2d(dst, m, c0, c1, fb);
          };
          load(sA + s * kABytes, &tmA, kb * kBK, m0);
          // kPartN columns of a weight from feature f0 on
          const auto load_b = [&](uint32_t dst, const CUtensorMap *m, int f0) {
            if constexpr (KM) {
              load(dst, m, kb * kBK, f0);
            } else {
#pragma unroll
              for (int j = 0; j < Cfg::kPartN / 64; ++j) load(dst + j * (kBK * 128), m, f0 + 64 * j, kb * kBK);
            }
          };
          const uint32_t b_dst = sB + s * Cfg::kBBytes;
          const int f0 = w.tn * Cfg::kTileF;
          if constexpr (BWD) {
            load_b(b_dst, &tmB0, f0 + (int)rank * Cfg::kCtaN);
          } else if constexpr (PAIR) {
            load_b(b_dst, leader ? &tmB0 : &tmB1, f0);
          } else {
            load_b(b_dst, &tmB0, f0);
            load_b(b_dst + Cfg::kPartN * kRowBytes, &tmB1, f0);
          }
          ++g;
        }
      }
      // Every load has landed before the CTA may exit (the peer's loads
      // complete on the leader's barriers: it waits until their stages have
      // been released).
      const uint32_t first = g > (uint32_t)STAGES ? g - STAGES : 0u;
      for (uint32_t i = first; i < g; ++i)
        mbar_wait_drain(leader ? full_bar(i % STAGES) : empty_bar(i % STAGES), (i / STAGES) & 1u, kDrainNs);
    }
    __syncwarp();
  } else if (warp == 1) {
    // -------------------------------------------------- MMA issuer (leader)
    if (lane == 0 && leader) {
      constexpr uint32_t idesc = idesc_bf16_f32(Cfg::kTileM, BN, !KM);
      uint32_t g = 0, acc_cnt = 0;
      bool ok = true;
      for (int t = first_unit; ok && t < num_units; t += unit_step) {
        const GatedUnit w = gated_unit(p, t);
        const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
        if (!mbar_wait(acce_bar(b), aph ^ 1u, abort_flag, p.err, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + b * BN;
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          const uint32_t s = g % STAGES, ph = (g / STAGES) & 1u;
          if (!mbar_wait(full_bar(s), ph, abort_flag, p.err, p.wait_limit_ns)) {
            ok = false;
            break;
          }
          tc_fence_after_sync();
          const uint32_t a0 = sA + s * kABytes;
          const uint32_t b0 = sB + s * Cfg::kBBytes;
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) {
            const uint64_t ad = smem_desc_sw128(a0 + k * 32, 16, 1024);
            const uint64_t bd = KM ? smem_desc_sw128(b0 + k * 32, 16, 1024)
                                   : smem_desc_sw128(b0 + k * 2048, kBK * 128, 1024);
            const uint32_t acc = (kb > w.kb0 || k > 0) ? 1u : 0u;
            if constexpr (PAIR)
              tc_mma_bf16_pair(d_tmem, ad, bd, idesc, acc);
            else
              tc_mma_bf16(d_tmem, ad, bd, idesc, acc);
          }
          if constexpr (PAIR)
            tc_commit_pair_multicast(empty_bar(s));
          else
            tc_commit(empty_bar(s));
          ++g;
        }
        if (!ok) break;
        if constexpr (PAIR)
          tc_commit_pair_multicast(accf_bar(b));
        else
          tc_commit(accf_bar(b));
        ++acc_cnt;
      }
      // all MMAs complete before TMEM is released
      if constexpr (PAIR)
        tc_commit_pair_multicast(drain_bar);
      else
        tc_commit(drain_bar);
      mbar_wait_drain(drain_bar, 0, kDrainNs);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    const int ew = warp - 2;
    const int quad = warp & 3;  // a warp may only touch TMEM lanes 32*(warp%4) ..
    const int colpart = ew >> 2;
    const uint32_t ebuf = base + Cfg::kEpiOffset + ew * Cfg::kEpiWarpBytes;
    uint32_t acc_cnt = 0;
    const auto store = [&](uint16_t *m, int64_t ld, uint32_t buf, int y, int x) {
      if (p.vec)
        block_store(m, ld, buf, lane, y, x, p.T, p.F);
      else
        block_store_any(m, ld, buf, lane, y, x, p.T, p.F);
    };
    // backward: blocks of G and U are asked for in the order in which they are
    // taken, those that exist; next_t, next_c: the next one
    int next_t = first_unit, next_c = 0;
    const auto ask = [&]() {
      while (next_t < num_units) {
        const GatedUnit w = gated_unit(p, next_t);
        const int y = w.tm * Cfg::kTileM + (int)rank * kBM + quad * 32;
        const int x = w.tn * Cfg::kTileF + (colpart * Cfg::kChunks + next_c) * 32;
        const bool here = !w.part && y < p.T && x < p.F;
        if (++next_c == Cfg::kChunks || !here) {
          next_c = 0;
          next_t += unit_step;
        }
        if (!here) continue;
        if (p.vec) {
          block_fetch(p.gate, p.ldgate, ebuf, lane, y, x, p.T, p.F);
          block_fetch(p.up, p.ldup, ebuf + 2048, lane, y, x, p.T, p.F);
        } else {
          block_fetch_any(p.gate, p.ldgate, p.up, p.ldup, ebuf, ebuf + 2048, lane, y, x, p.T, p.F);
        }
        return;
      }
    };
    if (BWD) ask();
    for (int t = first_unit; t < num_units; t += unit_step) {
      const GatedUnit w = gated_unit(p, t);
      const int y0 = w.tm * Cfg::kTileM + (int)rank * kBM + quad * 32;  // first row of this warp
      const int y = y0 + lane;
      const int col0 = colpart * (Cfg::kChunks * 32);
      const int x0 = w.tn * Cfg::kTileF + col0;
      const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
      const uint32_t t0 = tmem_base + b * BN + ((uint32_t)(quad * 32) << 16) + col0;
      if (!__all_sync(0xffffffffu, mbar_wait(accf_bar(b), aph, abort_flag, p.err, p.wait_limit_ns))) break;
      tc_fence_after_sync();
      if (w.part) {
        // all BN columns, as they are
        constexpr int kCols = BN / (Cfg::kEpiWarps / 4);
        const int64_t tail_rows = (int64_t)(p.tiles_m * p.tiles_n - p.tail_first) * Cfg::kTileM;
        const int row = w.slot * Cfg::kTileM + (int)rank * kBM + quad * 32 + lane;
        float *at = p.ws + (w.split * tail_rows + row) * BN + colpart * kCols;
#pragma unroll 1
        for (int c = 0; c < kCols; c += 32) {
          uint32_t v[32];
          tmem_ld_32x32b_x32(t0 - col0 + colpart * kCols + c, v);
          tmem_ld_wait();
          store_partials(at + c, v);
        }
      } else if constexpr (!BWD) {
#pragma unroll 1
        for (int c = 0; c < Cfg::kChunks; ++c) {
          const int x = x0 + c * 32;
          uint32_t g[32], u[32], h[16];
          tmem_ld_32x32b_x32(t0 + c * 32, g);
          tmem_ld_32x32b_x32(t0 + Cfg::kTileF + c * 32, u);
          tmem_ld_wait();
          if (y0 >= p.T || x >= p.F) continue;
          with_activation(p.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              h[i] = pack_bf16x2(gate<ACT, false>(__uint_as_float(g[2 * i])).a * __uint_as_float(u[2 * i]),
                                 gate<ACT, false>(__uint_as_float(g[2 * i + 1])).a * __uint_as_float(u[2 * i + 1]));
          });
          put_row(ebuf, lane, h);
          if (p.out[1]) {
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = pack_bf16x2(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1]));
            put_row(ebuf + 2048, lane, h);
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = pack_bf16x2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
            put_row(ebuf + 4096, lane, h);
          }
          __syncwarp();
          store(p.out[0], p.ldout[0], ebuf, y0, x);
          if (p.out[1]) {
            store(p.out[1], p.ldout[1], ebuf + 2048, y0, x);
            store(p.out[2], p.ldout[2], ebuf + 4096, y0, x);
          }
          __syncwarp();
        }
      } else {
        const bool live = y < p.T;
        uint32_t es = 0;  // exponents of the row's blocks
#pragma unroll 1
        for (int c = 0; c < Cfg::kChunks; ++c) {
          const int x = x0 + c * 32;
          if (y0 >= p.T || x >= p.F) break;
          uint32_t h[32];  // act(G) U of the block
          block_arrived();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t dh[16], g[8], u[8];
            tmem_ld_32x32b_x16(t0 + c * 32 + k * 16, dh);
            get_row16(ebuf, lane, k, g);
            get_row16(ebuf + 2048, lane, k, u);
            tmem_ld_wait();
            with_activation(p.act, [&](auto act) { gate_backward16<decltype(act)::value>(dh, g, u); });
            put_row16(ebuf, lane, k, g);
            put_row16(ebuf + 2048, lane, k, u);
#pragma unroll
            for (int i = 0; i < 16; ++i) h[16 * k + i] = dh[i];
          }
          __syncwarp();
          store(p.out[0], p.ldout[0], ebuf, y0, x);
          store(p.out[1], p.ldout[1], ebuf + 2048, y0, x);
          __syncwarp();
          const bool q_bytes = p.ck.q && !(p.vec && p.q_align >= 8);
          if (!q_bytes) ask();  // into the block just stored
          if (p.ck.q) {
            uint32_t q[8];
            es |= q8_block32(h, q) << (8 * c);
            int8_t *to = p.ck.q + (int64_t)y * p.ck.ldq + x;
            if (q_bytes) {
              // byte by byte along rows, through the block just stored
              st_shared_v4(ebuf + lane * 32, q[0], q[1], q[2], q[3]);
              st_shared_v4(ebuf + lane * 32 + 16, q[4], q[5], q[6], q[7]);
              __syncwarp();
              if (x + lane < p.F) {
                const int rows = min(32, p.T - y0);
                int8_t *col = p.ck.q + (int64_t)y0 * p.ck.ldq + x + lane;
#pragma unroll 8
                for (int i = 0; i < rows; ++i, col += p.ck.ldq) *col = (int8_t)ld_shared_u8(ebuf + i * 32 + lane);
              }
              __syncwarp();
              ask();
            } else if (p.q_align == 16 && x + 32 <= p.F) {
              if (live) store_32_bytes(to, q);
            } else {  // F is a multiple of 8
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (live && x + 8 * j < p.F) *reinterpret_cast<uint2 *>(to + 8 * j) = make_uint2(q[2 * j], q[2 * j + 1]);
            }
          }
        }
        if (p.ck.q && live) {
          uint8_t *e = p.ck.e + (int64_t)y * p.ck.lde + (x0 >> 5);
          constexpr int kMost = Cfg::kChunks;
          const int n = min(kMost, (p.F - x0 + 31) >> 5);  // blocks that exist (may be below 1)
          if (kMost == 4 && n == 4 && (reinterpret_cast<uintptr_t>(e) & 3) == 0) {
            *reinterpret_cast<uint32_t *>(e) = es;
          } else {
#pragma unroll
            for (int i = 0; i < kMost; ++i)
              if (i < n) e[i] = (uint8_t)(es >> (8 * i));
          }
        }
      }
      tc_fence_before_sync();
      if constexpr (PAIR)
        mbar_arrive_cluster(mapa_shared(acce_bar(b), 0));
      else
        mbar_arrive(acce_bar(b));
      ++acc_cnt;
    }
    block_arrived();  // a block asked for and not taken (after giving up only) has landed
  }

  griddep_launch_dependents();
  __syncwarp();
  tc_fence_before_sync();
  if constexpr (PAIR)
    cluster_sync_all();  // no remote arrival or load may target a CTA that has left
  else
    __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    if constexpr (PAIR)
      tmem_dealloc_pair<Cfg::kTmemCols>(tmem_base);
    else
      tmem_dealloc<Cfg::kTmemCols>(tmem_base);
  }
}

}  // namespace gb300
