// wgrad_tc.cuh -- persistent tcgen05 kernel of the weight gradient,
//     C[m][n] = base[m][n] + sum_t A[t][m] * B[t][n],
// A (T x M) and B (T x N) bf16 with the reduction index t outermost.
//
// Against C = A . B of gemm_tc.cuh / gemm_tc2.cuh both operands are
// transposed: a weight gradient reduces over the tokens, which are the rows
// of the activation and of the gradient.  The tensor core takes either
// operand with its M or N index contiguous ("MN-major"), so nothing is
// transposed in memory: boxes of 64 columns x 64 tokens land in shared memory
// with the 128-byte swizzle, and the matrix descriptors say which way to read
// them.  Roles, rings, accumulators and the pairing of two CTAs are those of
// gemm_tc2.cuh (PAIR: 256 x BN tiles, each CTA holding 128 rows of A^T and
// half of B) and gemm_tc.cuh (one CTA, 128 x BN tiles).
//
// Results are summed in slabs of p.tc.slab_kb k-blocks: the tensor core
// accumulates a slab in TMEM, and the epilogue warps add the slabs' sums in
// registers with round-to-nearest.  The tensor core's own additions cut what
// lies below 2^-25 of the larger of the sum and the products, so that a chain's
// error grows with its length; slabs bound the chain.  bf16 results, whose last
// rounding is far coarser, take longer slabs.
//
// The tensor cores bound it for many tokens (8192 tokens, 4096 x 11008,
// float32: 417 us alone, 1.77 PFLOP/s; 475 us back to back with X's restore,
// under the power cap), the output's bytes for few (128 tokens, 4096 x 4096
// float32 with base: 27 us for 136 MB), and between the two the rounds of
// tiles over 76 pairs (2048 tokens, 4096 x 4096: 256 tiles are 3.4 rounds, run
// as 4).
#pragma once
#include "gemm_tc2.cuh"
#include "layer_internal.h"

namespace gb300 {

constexpr int kWgEpiWarps = 8;
// Warps 0 (TMA) and 1 (MMA) of the first warpgroup work, the epilogue is the
// other two warpgroups.
constexpr int kWgThreads = (4 + kWgEpiWarps) * 32;
constexpr uint32_t kWgBoxBytes = 64 * kBK * 2;  // one 64-column x 64-token box

// Registers a thread when the sums of slabs are kept in them: the block is
// launched with 384 x 168; the first warpgroup gives up all but 40 of its own,
// and the epilogue's threads (128 sums each) take them: 128 x 40 + 256 x 232 =
// 384 x 168.
constexpr int kWgLaunchRegs = 168, kWgIssueRegs = 40, kWgEpiRegs = 232;
static_assert(128 * kWgIssueRegs + kWgEpiWarps * 32 * kWgEpiRegs <= kWgThreads * kWgLaunchRegs, "the shares fit");
template <int N>
__device__ __forceinline__ void regs_give() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_take() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// Blocks of base (32 x 32) in flight per epilogue warp of a kernel that brings
// base in by TMA.
constexpr int kBaseBlocks = 2;

// BASE: the kernel has shared memory for blocks of base.
template <int BN, bool PAIR, bool BASE>
struct WgCfg {
  static constexpr int kTileM = PAIR ? 2 * kBM : kBM;
  static constexpr int kCtaN = PAIR ? BN / 2 : BN;  // columns of B a CTA loads
  static_assert(kCtaN % 64 == 0 && BN <= 256, "operands are assembled from 64-wide boxes");
  static constexpr uint32_t kBBytes = kCtaN * kRowBytes;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  static constexpr uint32_t kBaseBytes = BASE ? kWgEpiWarps * kBaseBlocks * 4096u : 0u;
  static constexpr int kBaseBars = BASE ? kWgEpiWarps * kBaseBlocks : 0;
  // the deepest ring that the rest leaves room for
  static constexpr int kStages =
      tc_max_stages(kCtaN, kWgEpiWarps, 1) - (int)((kBaseBytes + kBaseBars * 8 + kStageBytes - 1) / kStageBytes);
  static constexpr uint32_t kTmemCols = pow2_at_least(2 * BN);
  static constexpr int kColsPerThread = BN / (kWgEpiWarps / 4);
  static_assert(kColsPerThread % 32 == 0, "the epilogue moves 32 columns at a time");
  static constexpr uint32_t kEpiOffset = kStages * kStageBytes;
  static constexpr uint32_t kBaseOffset = kEpiOffset + kWgEpiWarps * 4096;
  static constexpr uint32_t kBarOffset = kBaseOffset + kBaseBytes;
  static constexpr uint32_t kNumBars = 2 * kStages + 4 + 1 + kBaseBars;
  static constexpr uint32_t kSmemBytes = kBarOffset + kNumBars * 8 + 16 + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory per CTA is 227 KB");
  static_assert(kTmemCols <= 512, "TMEM has 512 columns");
};

// Where a base is added, and where C's rows rule TMA out, a 32 x 32 block of
// results is turned in the epilogue warp's shared memory, so that the lanes
// read base and write C along rows: a lane's own row would be 32 lines touched
// by every access of the warp, along rows it is four (16-byte pieces) or one
// or two (elements).

// Base's values that this lane adds to the block at (y0, x) by elements (lane =
// column): word i is row y0 + i.
__device__ __forceinline__ void fetch_base_elements(const WgradParams &p, int64_t y0, int x, int lane, uint4 (&b)[8]) {
  const int c = x + lane;
  if (c >= p.tc.N) return;
  uint32_t w[32] = {};
  const int rows = (int)min((int64_t)32, p.tc.M - y0);
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < rows) {
      const int64_t at = (y0 + i) * p.ldbase + c;
      w[i] = p.out_bf16 ? (uint32_t) static_cast<const uint16_t *>(p.base)[at] << 16
                        : static_cast<const uint32_t *>(p.base)[at];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// The same in 16-byte pieces (base's rows come in whole ones): four words of
// bf16, eight of float32.
__device__ __forceinline__ void fetch_base(const WgradParams &p, int64_t y0, int x, int lane, uint4 (&b)[8]) {
  if (p.out_bf16) {
    const int c = x + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = y0 + i * 8 + (lane >> 2);
      if (r < p.tc.M && c < p.tc.N)
        b[i] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.base) + r * p.ldbase + c);
    }
  } else {
    const int c = x + (lane & 7) * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = y0 + i * 4 + (lane >> 3);
      if (r < p.tc.M && c < p.tc.N)
        b[i] = *reinterpret_cast<const uint4 *>(static_cast<const float *>(p.base) + r * p.ldbase + c);
    }
  }
}

__device__ __forceinline__ float4 as_float4(uint4 v) {
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ float4 operator+(float4 a, float4 b) {
  return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}
__device__ __forceinline__ uint32_t block_piece(uint32_t buf, int row, int j) {
  return buf + row * 128 + ((j ^ (row & 7)) << 4);
}
// A block of sums (lane = row, 32 columns) into the warp's shared memory, in
// the layout of TMA's 128-byte swizzle.
__device__ __forceinline__ void stage_block(uint32_t buf, int lane, const uint32_t (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    st_shared_v4(block_piece(buf, lane, j), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}

// The block at (y0, x): base added, rounded once, stored by TMA.  AHEAD: b is
// as fetch_base left it; else base is fetched here, once v's registers are
// free.
template <bool AHEAD>
__device__ __forceinline__ void tma_out_with_base(const WgradParams &p, const CUtensorMap *tm, uint32_t buf, int lane,
                                                  const uint32_t (&v)[32], uint4 (&b)[8], int y0, int x) {
  if (lane == 0) bulk_wait_read_all();
  __syncwarp();
  stage_block(buf, lane, v);
  if (!AHEAD) fetch_base(p, y0, x, lane, b);
  __syncwarp();
  if (p.out_bf16) {
    const int j = lane & 3;
    uint4 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + (lane >> 2);
      const float4 lo = as_float4(ld_shared_v4(block_piece(buf, row, 2 * j))) +
                        make_float4(__uint_as_float(b[i].x << 16), __uint_as_float(b[i].x & 0xFFFF0000u),
                                    __uint_as_float(b[i].y << 16), __uint_as_float(b[i].y & 0xFFFF0000u));
      const float4 hi = as_float4(ld_shared_v4(block_piece(buf, row, 2 * j + 1))) +
                        make_float4(__uint_as_float(b[i].z << 16), __uint_as_float(b[i].z & 0xFFFF0000u),
                                    __uint_as_float(b[i].w << 16), __uint_as_float(b[i].w & 0xFFFF0000u));
      o[i] = make_uint4(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y),
                        pack_bf16x2(hi.z, hi.w));
    }
    __syncwarp();
    // 64-byte rows, 64-byte swizzle: chunk j of row r at chunk j ^ ((r / 2) % 4)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + (lane >> 2);
      st_shared_v4(buf + row * 64 + ((j ^ ((row >> 1) & 3)) << 4), o[i].x, o[i].y, o[i].z, o[i].w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = block_piece(buf, i * 4 + (lane >> 3), lane & 7);
      const float4 f = as_float4(ld_shared_v4(at)) + as_float4(b[i]);
      st_shared_v4(at, __float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w));
    }
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_2d(tm, buf, x, y0);
    bulk_commit();
  }
}

// A block of base in shared memory, as TMA brought it (the lane's row; 128-byte
// swizzle for float32, 64-byte for bf16), added to v.
__device__ __forceinline__ void add_base_block(uint32_t buf, int lane, bool bf, uint32_t (&v)[32]) {
  if (bf) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 w = ld_shared_v4(buf + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4));
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t &lo = v[8 * j + 2 * k], &hi = v[8 * j + 2 * k + 1];
        lo = __float_as_uint(__uint_as_float(lo) + __uint_as_float(u[k] << 16));
        hi = __float_as_uint(__uint_as_float(hi) + __uint_as_float(u[k] & 0xFFFF0000u));
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float4 w = as_float4(ld_shared_v4(block_piece(buf, lane, j)));
      const float u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) v[4 * j + k] = __float_as_uint(__uint_as_float(v[4 * j + k]) + u[k]);
    }
  }
}

// The block at (y0, x) with any base and C: base added, rounded once, stored
// element by element along rows (lane = column).  AHEAD: b is as
// fetch_base_elements left it.
template <bool AHEAD>
__device__ __forceinline__ void store_elements(const WgradParams &p, uint32_t buf, int lane, const uint32_t (&v)[32],
                                               const uint4 (&b)[8], int y0, int x) {
  if (lane == 0) bulk_wait_read_all();  // partials may still be leaving the buffer
  __syncwarp();
  stage_block(buf, lane, v);
  __syncwarp();
  const int c = x + lane, rows = min(32, p.tc.M - y0);
  if (c >= p.tc.N) return;
  // base may be C itself, so loads cannot move above stores by themselves: a
  // batch of rows is read before the first of them is written
  constexpr int kBatch = AHEAD ? 32 : 8;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += kBatch) {
    if (r0 >= rows) break;
    float f[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      f[i] = __uint_as_float(ld_shared_u32(block_piece(buf, r0 + i, lane >> 2) + (lane & 3) * 4));
    if (p.base) {
      float o[kBatch] = {};
      if constexpr (AHEAD) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 l = as_float4(b[i]);
          o[4 * i] = l.x, o[4 * i + 1] = l.y, o[4 * i + 2] = l.z, o[4 * i + 3] = l.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (r0 + i < rows) {
            const int64_t at = (int64_t)(y0 + r0 + i) * p.ldbase + c;
            o[i] = p.out_bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(p.base)[at] << 16)
                              : static_cast<const float *>(p.base)[at];
          }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) f[i] += o[i];
    }
    if (p.out_bf16) {
      __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(p.tc.C) + (int64_t)(y0 + r0) * p.tc.ldc + c;
#pragma unroll
      for (int i = 0; i < kBatch; ++i, dst += p.tc.ldc)
        if (r0 + i < rows) *dst = __float2bfloat16_rn(f[i]);
    } else {
      float *dst = static_cast<float *>(p.tc.C) + (int64_t)(y0 + r0) * p.tc.ldc + c;
#pragma unroll
      for (int i = 0; i < kBatch; ++i, dst += p.tc.ldc)
        if (r0 + i < rows) *dst = f[i];
    }
  }
}

// SLABS: the sums of several slabs are added in registers (the reduction is
// longer than one slab); else every unit is one slab.
// BASE (without SLABS): base and C are TMA's; each epilogue warp keeps
// kBaseBlocks blocks of base on their way in shared memory, the next unit's
// among them, since with few tokens base and C are all the traffic and
// registers hold base no further ahead than the unit (128 tokens, 4096 x 4096
// float32: 36.0 us with registers, 27.4 so).
template <int BN, bool PAIR, bool SLABS, bool BASE>
__global__ void __launch_bounds__(kWgThreads, 1)
    wgrad_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                 const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmWs,
                 const __grid_constant__ CUtensorMap tmBase, const WgradParams wp) {
  static_assert(!(SLABS && BASE), "slabs add base in registers");
  using Cfg = WgCfg<BN, PAIR, BASE>;
  constexpr int STAGES = Cfg::kStages;
  const TcParams &p = wp.tc;
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
  const uint32_t base_bars = drain_bar + 8u;

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
      mbar_init(acce_bar(b), (PAIR ? 2 : 1) * kWgEpiWarps * 32);
    }
    mbar_init(drain_bar, 1);
    for (int b = 0; b < Cfg::kBaseBars; ++b) mbar_init(base_bars + 8u * b, 1);
    *abort_flag = 0u;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (p.out_tma == kOutTmaC) tma_prefetch_desc(&tmOut);
    if (BASE) tma_prefetch_desc(&tmBase);
    if (p.tail_splits > 0) tma_prefetch_desc(&tmWs);
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
  // kernel of the stream (which wrote A).
  griddep_wait();

  const int num_units = tc_num_units(p);
  constexpr uint64_t kDrainNs = 200ull * 1000 * 1000;

  if (warp < 4) {
    if constexpr (SLABS) regs_give<kWgIssueRegs>();
    if (warp == 0) {
      // ------------------------------------------------------ TMA producer
      if (lane == 0) {
        uint32_t g = 0;
        bool ok = true;
        for (int u = first_unit; ok && u < num_units; u += unit_step) {
          const Unit w = decode_unit(p, u);
          const int m0 = w.tm * Cfg::kTileM + (int)rank * kBM;
          const int n0 = w.tn * BN + (int)rank * Cfg::kCtaN;
          for (int kb = w.kb0; kb < w.kb1; ++kb) {
            const uint32_t s = g % STAGES, ph = (g / STAGES) & 1u;
            if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, p.err, p.wait_limit_ns)) {
              ok = false;
              break;
            }
            if (leader) mbar_arrive_expect_tx(full_bar(s), (PAIR ? 2 : 1) * Cfg::kStageBytes);
            const uint32_t a_dst = sA + s * kABytes, b_dst = sB + s * Cfg::kBBytes;
            if constexpr (PAIR) {
              const uint32_t fb = mapa_shared(full_bar(s), 0);
#pragma unroll
              for (int j = 0; j < kBM / 64; ++j)
                tma_load_2d_pair(a_dst + j * kWgBoxBytes, &tmA, m0 + 64 * j, kb * kBK, fb);
#pragma unroll
              for (int j = 0; j < Cfg::kCtaN / 64; ++j)
                tma_load_2d_pair(b_dst + j * kWgBoxBytes, &tmB, n0 + 64 * j, kb * kBK, fb);
            } else {
#pragma unroll
              for (int j = 0; j < kBM / 64; ++j)
                tma_load_2d(a_dst + j * kWgBoxBytes, &tmA, m0 + 64 * j, kb * kBK, full_bar(s));
#pragma unroll
              for (int j = 0; j < Cfg::kCtaN / 64; ++j)
                tma_load_2d(b_dst + j * kWgBoxBytes, &tmB, n0 + 64 * j, kb * kBK, full_bar(s));
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
      // ------------------------------------------------ MMA issuer (leader)
      if (lane == 0 && leader) {
        // both operands MN-major: bit 15 is A's, bit 16 B's
        constexpr uint32_t idesc = idesc_bf16_f32(Cfg::kTileM, BN, true) | (1u << 15);
        uint32_t g = 0, acc_cnt = 0;
        bool ok = true;
        for (int u = first_unit; ok && u < num_units; u += unit_step) {
          const Unit w = decode_unit(p, u);
          for (int kb_s = w.kb0; ok && kb_s < w.kb1; kb_s += p.slab_kb) {
            const int kb_e = min(w.kb1, kb_s + p.slab_kb);
            const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
            if (!mbar_wait(acce_bar(b), aph ^ 1u, abort_flag, p.err, p.wait_limit_ns)) {
              ok = false;
              break;
            }
            tc_fence_after_sync();
            const uint32_t d_tmem = tmem_base + b * BN;
            for (int kb = kb_s; kb < kb_e; ++kb) {
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
                // 64-wide chunks one box apart (LBO), groups of 8 tokens 1024
                // bytes apart (SBO); a step of 16 tokens is 2048 bytes
                const uint64_t ad = smem_desc_sw128(a0 + k * 2048, kWgBoxBytes, 1024);
                const uint64_t bd = smem_desc_sw128(b0 + k * 2048, kWgBoxBytes, 1024);
                const uint32_t acc = (kb > kb_s || k > 0) ? 1u : 0u;
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
        }
        // all MMAs complete before TMEM is released
        if constexpr (PAIR)
          tc_commit_pair_multicast(drain_bar);
        else
          tc_commit(drain_bar);
        mbar_wait_drain(drain_bar, 0, kDrainNs);
      }
      __syncwarp();
    }
  } else {
    if constexpr (SLABS) regs_take<kWgEpiRegs>();
    // --------------------------------------------------------- epilogue
    constexpr int CPT = Cfg::kColsPerThread;
    const int ew = warp - 4;
    const int quad = warp & 3;  // a warp may only touch TMEM lanes 32*(warp%4) ..
    const int colpart = ew >> 2;
    const uint32_t ebuf = base + Cfg::kEpiOffset + ew * 4096u;
    uint32_t acc_cnt = 0;
    bool ok = true;
    // BASE: blocks of base in the order in which they are added, those that
    // exist; next_u, next_c: the next one to ask for
    constexpr int kChunks = CPT / 32;
    const uint32_t base_buf = base + Cfg::kBaseOffset + ew * (kBaseBlocks * 4096u);
    const uint32_t base_bar = base_bars + 8u * (ew * kBaseBlocks);
    uint32_t asked = 0, added = 0;
    int next_u = first_unit, next_c = 0;
    const auto ask = [&]() {
      while (next_u < num_units) {
        const Unit w = decode_unit(p, next_u);
        const int y = w.tm * Cfg::kTileM + (int)rank * kBM + quad * 32, x = w.tn * BN + colpart * CPT + next_c * 32;
        const bool here = w.part == 0 && y < p.M && x < p.N;
        if (++next_c == kChunks || w.part != 0 || y >= p.M) {
          next_c = 0;
          next_u += unit_step;
        }
        if (!here) continue;
        if (lane == 0) {
          const uint32_t k = asked % kBaseBlocks;
          mbar_arrive_expect_tx(base_bar + 8u * k, wp.out_bf16 ? 2048u : 4096u);
          tma_load_2d(base_buf + k * 4096u, &tmBase, x, y, base_bar + 8u * k);
        }
        ++asked;
        return;
      }
    };
    if constexpr (BASE) {
      for (int i = 0; i < kBaseBlocks; ++i) ask();
    }
    for (int u = first_unit; ok && u < num_units; u += unit_step) {
      const Unit w = decode_unit(p, u);
      const bool split = w.part != 0;  // partials of a split-tail tile, not C
      const int y0 = w.tm * Cfg::kTileM + (int)rank * kBM + quad * 32;  // first row of this warp
      const int col0 = w.tn * BN + colpart * CPT;
      const bool with_base = !BASE && wp.base != nullptr && !split && y0 < p.M;
      // Writes 32 columns of sums: of C, or of a tail tile's partials (compact
      // blocks: tile `slot`, row pitch BN).
      auto emit = [&](uint32_t(&v)[32], uint4(&base_words)[8], int c) {
        const int x = col0 + c * 32;
        const bool in_range = y0 < p.M && x < p.N;
        if (split) {
          tma_out_words32<true>(&tmWs, ebuf, lane, v, colpart * CPT + c * 32,
                                w.slot * Cfg::kTileM + (int)rank * kBM + quad * 32, w.split, true);
        } else if (!BASE && p.out_tma == kOutTmaC && wp.base) {
          if (in_range) tma_out_with_base<!SLABS>(wp, &tmOut, ebuf, lane, v, base_words, y0, x);
        } else if (BASE || p.out_tma == kOutTmaC) {
          if (BASE && in_range) {
            const uint32_t k = added % kBaseBlocks;
            ok = __all_sync(0xffffffffu, mbar_wait(base_bar + 8u * k, (added / kBaseBlocks) & 1u, abort_flag, p.err,
                                                   p.wait_limit_ns));
            if (!ok) return;
            ++added;
            add_base_block(base_buf + k * 4096u, lane, wp.out_bf16 != 0, v);
            fence_proxy_async_smem();
            __syncwarp();
            ask();  // into the block just read
          }
          if (wp.out_bf16)
            tma_out_bf16x32(&tmOut, ebuf, lane, v, x, y0, in_range);
          else
            tma_out_words32<false>(&tmOut, ebuf, lane, v, x, y0, 0, in_range);
        } else if (in_range) {
          store_elements<!SLABS>(wp, ebuf, lane, v, base_words, y0, x);
        }
      };
      auto release = [&](uint32_t b) {
        tc_fence_before_sync();
        if constexpr (PAIR)
          mbar_arrive_cluster(mapa_shared(acce_bar(b), 0));
        else
          mbar_arrive(acce_bar(b));
        ++acc_cnt;
      };
      const uint32_t t_lane = (uint32_t)(quad * 32) << 16;
      if constexpr (!SLABS) {
        // one slab: its sums are the result, streamed 32 columns at a time, base
        // (without BASE) two blocks ahead in registers
        constexpr int kAhead = kChunks < 2 ? kChunks : 2;
        uint4 ahead[kAhead][8] = {};
        const auto fetch = [&](int x, uint4(&o)[8]) {
          if (p.out_tma == kOutTmaC)
            fetch_base(wp, y0, x, lane, o);
          else
            fetch_base_elements(wp, y0, x, lane, o);
        };
#pragma unroll
        for (int c = 0; c < kAhead; ++c)
          if (with_base) fetch(col0 + c * 32, ahead[c]);
        const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
        if (!__all_sync(0xffffffffu, mbar_wait(accf_bar(b), aph, abort_flag, p.err, p.wait_limit_ns))) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          uint32_t v[32];
          tmem_ld<32>(tmem_base + b * BN + t_lane + colpart * CPT + c * 32, v);
          tmem_ld_wait();
          emit(v, ahead[c % kAhead], c);
          if (!ok) break;
          if (with_base && c + kAhead < kChunks) fetch(col0 + (c + kAhead) * 32, ahead[c % kAhead]);
        }
        if (!ok) break;
        release(b);
      } else {
        float acc[CPT];
#pragma unroll
        for (int i = 0; i < CPT; ++i) acc[i] = 0.f;
        for (int kb_s = w.kb0; kb_s < w.kb1; kb_s += p.slab_kb) {
          const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
          if (!__all_sync(0xffffffffu, mbar_wait(accf_bar(b), aph, abort_flag, p.err, p.wait_limit_ns))) {
            ok = false;
            break;
          }
          tc_fence_after_sync();
#pragma unroll
          for (int c = 0; c < CPT / 16; ++c) {
            uint32_t v[16];
            tmem_ld<16>(tmem_base + b * BN + t_lane + colpart * CPT + c * 16, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c * 16 + i] += __uint_as_float(v[i]);
          }
          release(b);
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < CPT / 32; ++c) {
          uint32_t v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(acc[c * 32 + i]);
          uint4 base_words[8];
          emit(v, base_words, c);
        }
      }
    }
    if (lane == 0) {
      // blocks of base asked for and not added (after giving up only) have landed
      for (; BASE && added < asked; ++added)
        mbar_wait_drain(base_bar + 8u * (added % kBaseBlocks), (added / kBaseBlocks) & 1u, kDrainNs);
      bulk_wait_all();  // this warp's TMA stores have landed
    }
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
