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
// Float32 results are summed in slabs of p.tc.slab_kb k-blocks: the tensor
// core accumulates a slab in TMEM, and the epilogue warps add the slabs'
// sums in registers with round-to-nearest.  The tensor core's own additions
// lose low bits in one direction, so that a chain's error grows with its
// length; slabs bound the chain.  bf16 results, whose last rounding is far
// coarser, take the whole sum as one slab.
#pragma once
#include "gemm_tc2.cuh"
#include "layer_internal.h"

namespace gb300 {

constexpr int kWgEpiWarps = 8;
constexpr int kWgThreads = (2 + kWgEpiWarps) * 32;
constexpr uint32_t kWgBoxBytes = 64 * kBK * 2;  // one 64-column x 64-token box

template <int BN, bool PAIR>
struct WgCfg {
  static constexpr int kTileM = PAIR ? 2 * kBM : kBM;
  static constexpr int kCtaN = PAIR ? BN / 2 : BN;  // columns of B a CTA loads
  static_assert(kCtaN % 64 == 0 && BN <= 256, "operands are assembled from 64-wide boxes");
  static constexpr uint32_t kBBytes = kCtaN * kRowBytes;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = tc_max_stages(kCtaN, kWgEpiWarps, 1);
  static constexpr uint32_t kTmemCols = pow2_at_least(2 * BN);
  static constexpr int kColsPerThread = BN / (kWgEpiWarps / 4);
  static_assert(kColsPerThread % 32 == 0, "the epilogue moves 32 columns at a time");
  static constexpr uint32_t kEpiOffset = kStages * kStageBytes;
  static constexpr uint32_t kBarOffset = kEpiOffset + kWgEpiWarps * 4096;
  static constexpr uint32_t kNumBars = 2 * kStages + 4 + 1;
  static constexpr uint32_t kSmemBytes = kBarOffset + kNumBars * 8 + 16 + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory per CTA is 227 KB");
  static_assert(kTmemCols <= 512, "TMEM has 512 columns");
};

// 32 columns of one row of base added to v; clipped at column N.  base may be
// the result itself, so these are plain loads; this thread's block of C is
// written after them.
__device__ __forceinline__ void add_base32(const WgradParams &p, int64_t row, int col, uint32_t (&v)[32]) {
  if (p.out_bf16) {
    const uint16_t *src = static_cast<const uint16_t *>(p.base) + row * p.ldbase + col;
    if (col + 32 <= p.tc.N && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 w = reinterpret_cast<const uint4 *>(src)[i];
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[8 * i + 2 * j] = __float_as_uint(__uint_as_float(v[8 * i + 2 * j]) + __uint_as_float(u[j] << 16));
          v[8 * i + 2 * j + 1] =
              __float_as_uint(__uint_as_float(v[8 * i + 2 * j + 1]) + __uint_as_float(u[j] & 0xFFFF0000u));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (col + i < p.tc.N)
          v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float((uint32_t)src[i] << 16));
    }
  } else {
    const float *src = static_cast<const float *>(p.base) + row * p.ldbase + col;
    if (col + 32 <= p.tc.N && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 w = reinterpret_cast<const float4 *>(src)[i];
        v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + w.x);
        v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + w.y);
        v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + w.z);
        v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + w.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (col + i < p.tc.N) v[i] = __float_as_uint(__uint_as_float(v[i]) + src[i]);
    }
  }
}

// Launch with cluster dimensions (2,1,1) and an even grid when PAIR.
template <int BN, bool PAIR>
__global__ void __launch_bounds__(kWgThreads, 1)
    wgrad_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                 const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmWs,
                 const WgradParams wp) {
  using Cfg = WgCfg<BN, PAIR>;
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
    *abort_flag = 0u;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (p.out_tma != kOutDirect) tma_prefetch_desc(&tmOut);
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
  } else {
    // --------------------------------------------------------- epilogue
    constexpr int CPT = Cfg::kColsPerThread;
    const int ew = warp - 2;
    const int quad = warp & 3;  // a warp may only touch TMEM lanes 32*(warp%4) ..
    const int colpart = ew >> 2;
    const uint32_t ebuf = base + Cfg::kEpiOffset + ew * 4096u;
    uint32_t acc_cnt = 0;
    bool ok = true;
    for (int u = first_unit; ok && u < num_units; u += unit_step) {
      const Unit w = decode_unit(p, u);
      const bool split = w.part != 0;  // partials of a split-tail tile, not C
      const int y0 = w.tm * Cfg::kTileM + (int)rank * kBM + quad * 32;  // first row of this warp
      const int64_t row = (int64_t)y0 + lane;
      const bool row_ok = row < p.M;
      const int col0 = w.tn * BN + colpart * CPT;
      // Writes 32 columns of sums, with base added and rounded once: of C
      // through TMA where its rows allow, else directly; of the partials
      // (compact blocks: tail tile `slot`, row pitch BN) through TMA.
      auto emit = [&](uint32_t(&v)[32], int c) {
        const int x = col0 + c * 32;
        if (split) {
          tma_out_words32<true>(&tmWs, ebuf, lane, v, colpart * CPT + c * 32,
                                w.slot * Cfg::kTileM + (int)rank * kBM + quad * 32, w.split, true);
          return;
        }
        if (wp.base && row_ok && x < p.N) add_base32(wp, row, x, v);
        const bool in_range = y0 < p.M && x < p.N;
        if (p.out_tma == kOutTmaC) {
          if (wp.out_bf16)
            tma_out_bf16x32(&tmOut, ebuf, lane, v, x, y0, in_range);
          else
            tma_out_words32<false>(&tmOut, ebuf, lane, v, x, y0, 0, in_range);
        } else if (row_ok) {
          if (wp.out_bf16)
            store_bf16<32>(static_cast<uint16_t *>(p.C) + row * p.ldc, x, p.N, true, v);
          else
            store_words<32>(static_cast<uint32_t *>(p.C) + row * p.ldc, x, p.N, true, v);
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
      if (w.kb1 - w.kb0 <= p.slab_kb) {
        // one slab: its sums are the result, streamed 32 columns at a time
        const uint32_t b = acc_cnt & 1u, aph = (acc_cnt >> 1) & 1u;
        if (!__all_sync(0xffffffffu, mbar_wait(accf_bar(b), aph, abort_flag, p.err, p.wait_limit_ns))) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
#pragma unroll 1
        for (int c = 0; c < CPT / 32; ++c) {
          uint32_t v[32];
          tmem_ld<32>(tmem_base + b * BN + t_lane + colpart * CPT + c * 32, v);
          tmem_ld_wait();
          emit(v, c);
        }
        release(b);
        continue;
      }
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
        for (int c = 0; c < CPT / 32; ++c) {
          uint32_t v[32];
          tmem_ld<32>(tmem_base + b * BN + t_lane + colpart * CPT + c * 32, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[c * 32 + i] += __uint_as_float(v[i]);
        }
        release(b);
      }
      if (!ok) break;
#pragma unroll
      for (int c = 0; c < CPT / 32; ++c) {
        uint32_t v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(acc[c * 32 + i]);
        emit(v, c);
      }
    }
    if (lane == 0) bulk_wait_all();  // this warp's TMA stores have landed
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
