// gated_few.cu -- the gated feed-forward block's projections for few tokens (a
// batch of sequences a token each): H = act(X Wg) * (X Wu), T <= 128.
//
// The weights' bytes bound it (4 K F, read once), so the tile is turned round:
// the tensor core's 128 rows are 64 gate and the same 64 up features, streamed
// by TMA in either layout of the weights, and its columns are the tokens, 16 to
// 128 of them.  A cluster of up to eight CTAs shares a tile's reduction, so that
// a layer with few tiles still fills the device; their sums meet in distributed
// shared memory, added in the order of the CTAs, and the gate is taken there:
// one launch, no scratch, no atomics.
#include <atomic>

#include "gate_math.cuh"
#include "gemm_tc2.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kFewThreads = 192;  // warp 0: TMA, warp 1: MMA, warps 2-5: TMEM lanes
constexpr int kFewF = 64;         // features of a tile
constexpr uint32_t kWBytes = 2 * kFewF * kRowBytes;

template <int TN>
struct FewCfg {
  static constexpr uint32_t kStageBytes = kWBytes + TN * kRowBytes;
  static constexpr int kCtasPerSm = TN <= 64 ? 3 : 2;
  // shared memory of an SM (228 KB, 1 KB a CTA taken) among its CTAs
  static constexpr int kStages = (int)((227u * 1024u / kCtasPerSm - 3072u) / kStageBytes);
  static constexpr uint32_t kTmemCols = pow2_at_least(TN);
  static constexpr uint32_t kRingBytes = kStages * kStageBytes;
  static_assert(kRingBytes >= 128 * TN * 4, "the sums are laid over the ring");
  static constexpr uint32_t kSmemBytes = kRingBytes + (2 * kStages + 1) * 8 + 16 + 1024;
};

struct FewParams {
  GatedTcParams g;
  int splits;  // CTAs of a cluster
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared_f32(uint32_t addr, uint32_t v) { st_shared_u32(addr, v); }

template <int TN, bool KM>
__global__ void __launch_bounds__(kFewThreads, FewCfg<TN>::kCtasPerSm)
    gated_few_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmG,
                     const __grid_constant__ CUtensorMap tmU, const FewParams fp) {
  using Cfg = FewCfg<TN>;
  constexpr int STAGES = Cfg::kStages;
  const GatedTcParams &p = fp.g;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;  // swizzle atoms need 1024-byte alignment
  uint8_t *ring_ptr = smem_raw + (ring - raw);
  const uint32_t bars = ring + Cfg::kRingBytes;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(ring_ptr + Cfg::kRingBytes + (2 * STAGES + 1) * 8);
  volatile uint32_t *abort_flag = tmem_slot + 1;
  auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bars + 8u * (STAGES + s); };
  const uint32_t acc_bar = bars + 8u * (2 * STAGES);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int f0 = (int)(blockIdx.x / (unsigned)fp.splits) * kFewF;
  const int kb0 = (int)((int64_t)p.num_kb * rank / fp.splits), kb1 = (int)((int64_t)p.num_kb * (rank + 1) / fp.splits);

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(acc_bar, 1);
    *abort_flag = 0u;
    fence_mbar_init();
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmG);
    tma_prefetch_desc(&tmU);
  }
  __syncwarp();
  if (warp == 1) tmem_alloc<Cfg::kTmemCols>(smem_addr(tmem_slot));
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();
  constexpr uint64_t kDrainNs = 200ull * 1000 * 1000;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t g = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++g) {
        const uint32_t s = g % STAGES, ph = (g / STAGES) & 1u;
        if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, p.err, p.wait_limit_ns)) break;
        mbar_arrive_expect_tx(full_bar(s), Cfg::kStageBytes);
        const uint32_t w = ring + s * Cfg::kStageBytes;
        const int x = KM ? kb * kBK : f0, y = KM ? f0 : kb * kBK;
        tma_load_2d(w, &tmG, x, y, full_bar(s));
        tma_load_2d(w + kWBytes / 2, &tmU, x, y, full_bar(s));
        tma_load_2d(w + kWBytes, &tmX, kb * kBK, 0, full_bar(s));
      }
      // every load has landed before the CTA may exit
      const uint32_t first = g > (uint32_t)STAGES ? g - STAGES : 0u;
      for (uint32_t i = first; i < g; ++i) mbar_wait_drain(full_bar(i % STAGES), (i / STAGES) & 1u, kDrainNs);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_bf16_f32(128, TN, false) | (KM ? 0u : 1u << 15);
      uint32_t g = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++g) {
        const uint32_t s = g % STAGES, ph = (g / STAGES) & 1u;
        if (!mbar_wait(full_bar(s), ph, abort_flag, p.err, p.wait_limit_ns)) break;
        tc_fence_after_sync();
        const uint32_t w = ring + s * Cfg::kStageBytes, x = w + kWBytes;
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k) {
          const uint64_t ad = KM ? smem_desc_sw128(w + k * 32, 16, 1024)
                                 : smem_desc_sw128(w + k * 2048, kWBytes / 2, 1024);
          tc_mma_bf16(tmem_base, ad, smem_desc_sw128(x + k * 32, 16, 1024), idesc, (g > 0 || k > 0) ? 1u : 0u);
        }
        tc_commit(empty_bar(s));
      }
      tc_commit(acc_bar);  // all MMAs, which have read every stage
      mbar_wait_drain(acc_bar, 0, kDrainNs);
    }
    __syncwarp();
  } else {
    // this CTA's sums, token by token, over the ring: sums[token][feature]
    const int quad = warp & 3;
    if (__all_sync(0xffffffffu, mbar_wait(acc_bar, 0, abort_flag, p.err, p.wait_limit_ns))) {
      tc_fence_after_sync();
      const uint32_t at = ring + (quad * 32 + lane) * 4;
#pragma unroll
      for (int c = 0; c < TN / 16; ++c) {
        uint32_t v[16];
        tmem_ld_32x32b_x16(tmem_base + ((uint32_t)(quad * 32) << 16) + c * 16, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) st_shared_f32(at + (c * 16 + i) * 512, v[i]);
      }
    }
    tc_fence_before_sync();
  }
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc<Cfg::kTmemCols>(tmem_base);
  }
  // the cluster's CTAs share the tokens out: sums of all of them, the gate, H
  const int t0 = (int)((int64_t)p.T * rank / fp.splits), t1 = (int)((int64_t)p.T * (rank + 1) / fp.splits);
  const int f = (int)threadIdx.x & (kFewF - 1);
  if (f0 + f < p.F) {
    for (int t = t0 + ((int)threadIdx.x >> 6); t < t1; t += kFewThreads / kFewF) {
      const uint32_t at = ring + t * 512 + f * 4;
      float g = 0.f, u = 0.f;
      for (int s = 0; s < fp.splits; ++s) {
        const uint32_t from = mapa_shared(at, s);
        g += ld_cluster_f32(from);
        u += ld_cluster_f32(from + kFewF * 4);
      }
      float h = 0.f;
      with_activation(p.act, [&](auto act) { h = gate<decltype(act)::value, false>(g).a * u; });
      store_value<bf16>(p.out[0], t * p.ldout[0] + f0 + f, h);
      if (p.out[1]) {
        store_value<bf16>(p.out[1], t * p.ldout[1] + f0 + f, g);
        store_value<bf16>(p.out[2], t * p.ldout[2] + f0 + f, u);
      }
    }
  }
  cluster_sync_all();  // no CTA leaves while another reads its sums
}

template <int TN, bool KM>
cudaError_t launch(const GatedMaps &m, const FewParams &p, int grid, cudaStream_t st) {
  using Cfg = FewCfg<TN>;
  auto kern = gated_few_kernel<TN, KM>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3((unsigned)grid), dim3(kFewThreads), Cfg::kSmemBytes, st, p.splits, m.a, m.b[0], m.b[1], p);
}
template <bool KM>
cudaError_t launch_tokens(int tn, const GatedMaps &m, const FewParams &p, int grid, cudaStream_t st) {
  return tn == 16   ? launch<16, KM>(m, p, grid, st)
         : tn == 32 ? launch<32, KM>(m, p, grid, st)
         : tn == 64 ? launch<64, KM>(m, p, grid, st)
                    : launch<128, KM>(m, p, grid, st);
}

}  // namespace

int gated_few_columns(int64_t T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128; }

cudaError_t launch_gated_few(bool km, const GatedMaps &m, const GatedTcParams &p, int sms, cudaStream_t st) {
  const int tn = gated_few_columns(p.T), tiles = (p.F + kFewF - 1) / kFewF;
  const int slots = sms * (tn <= 64 ? 3 : 2);
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= slots && p.num_kb >= splits * 8) splits *= 2;
  const FewParams fp{p, splits};
  return km ? launch_tokens<true>(tn, m, fp, tiles * splits, st) : launch_tokens<false>(tn, m, fp, tiles * splits, st);
}

}  // namespace gb300
