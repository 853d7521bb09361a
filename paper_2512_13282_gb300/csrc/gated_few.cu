// gated_few.cu -- the gated feed-forward block for few tokens (a batch of
// sequences a token each), T <= 64: H = act(X Wg) * (X Wu), and the gate's
// gradient from dH = dO Wd^T.
//
// The weights' bytes bound both (4 K F or 2 N F, read once), so the tile is
// turned round: the tensor core's 128 rows are features -- 64 gate and the same
// 64 up features, or 128 of Wd's -- streamed by TMA in either layout of the
// weights, and its columns are the tokens, 16 to 64 of them.  A cluster of up
// to eight CTAs shares a tile's reduction, so that a layer with few tiles still
// fills the device; their sums meet in distributed shared memory, added in the
// order of the CTAs, and the gate or its gradient is taken there: one launch, no
// scratch, no atomics.  1 token, 4096 x 11008: 31.4 us (180 MB at 5.7 TB/s).
#include <atomic>

#include "gate_math.cuh"
#include "gemm_tc2.cuh"
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kFewThreads = 192;  // warp 0: TMA, warp 1: MMA, warps 2-5: TMEM lanes
constexpr int kFewRows = 128;     // features (forward: gate and up values) of a tile
constexpr uint32_t kWBytes = kFewRows * kRowBytes;

template <int TN>
struct FewCfg {
  static constexpr uint32_t kStageBytes = kWBytes + TN * kRowBytes;
  static constexpr int kCtasPerSm = 3;
  // shared memory of an SM (228 KB, 1 KB a CTA taken) among its CTAs
  static constexpr int kStages = (int)((227u * 1024u / kCtasPerSm - 3u * 1024u) / kStageBytes);
  static constexpr uint32_t kTmemCols = pow2_at_least(TN);
  static constexpr uint32_t kRingBytes = kStages * kStageBytes;
  static_assert(kRingBytes >= kFewRows * TN * 4, "the sums are laid over the ring");
  static constexpr uint32_t kSmemBytes = kRingBytes + (2 * kStages + 1) * 8 + 16 + 1024;
};

struct FewParams {
  GatedTcParams g;
  int splits;  // CTAs of a cluster
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

template <int TN, bool KM, bool BWD>
__global__ void __launch_bounds__(kFewThreads, FewCfg<TN>::kCtasPerSm)
    gated_few_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmG,
                     const __grid_constant__ CUtensorMap tmU, const FewParams fp) {
  using Cfg = FewCfg<TN>;
  constexpr int STAGES = Cfg::kStages;
  constexpr int kTileF = BWD ? kFewRows : kFewRows / 2;
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
  const int f0 = (int)(blockIdx.x / (unsigned)fp.splits) * kTileF;
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
    if (!BWD) tma_prefetch_desc(&tmU);
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
        // two boxes of 64 features: a weight's each, or one weight's
        const int f1 = BWD ? f0 + kFewRows / 2 : f0;
        tma_load_2d(w, &tmG, KM ? kb * kBK : f0, KM ? f0 : kb * kBK, full_bar(s));
        tma_load_2d(w + kWBytes / 2, BWD ? &tmG : &tmU, KM ? kb * kBK : f1, KM ? f1 : kb * kBK, full_bar(s));
        tma_load_2d(w + kWBytes, &tmX, kb * kBK, 0, full_bar(s));
      }
      // every load has landed before the CTA may exit
      const uint32_t first = g > (uint32_t)STAGES ? g - STAGES : 0u;
      for (uint32_t i = first; i < g; ++i) mbar_wait_drain(full_bar(i % STAGES), (i / STAGES) & 1u, kDrainNs);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_bf16_f32(kFewRows, TN, false) | (KM ? 0u : 1u << 15);
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
        for (int i = 0; i < 16; ++i) st_shared_u32(at + (c * 16 + i) * (kFewRows * 4), v[i]);
      }
    }
    tc_fence_before_sync();
  }
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc<Cfg::kTmemCols>(tmem_base);
  }
  // The cluster's CTAs share the tokens out: sums of all of them, the gate,
  // results.  A warp takes 32 features of a token, kBatch of these at a time so
  // that their loads overlap.
  constexpr int kGroups = kTileF / 32, kBatch = 4, kWarps = kFewThreads / 32;
  const int t0 = (int)((int64_t)p.T * rank / fp.splits), t1 = (int)((int64_t)p.T * (rank + 1) / fp.splits);
  const int items = (t1 - t0) * kGroups;
  for (int i0 = warp; i0 < items; i0 += kBatch * kWarps) {
    float a[kBatch] = {}, b[kBatch] = {};  // the sums: of g and u, or of dh
    float gate_in[kBatch], up_in[kBatch];
    uint32_t at[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = min(i0 + j * kWarps, items - 1), t = t0 + i / kGroups, f = (i % kGroups) * 32 + lane, c = f0 + f;
      at[j] = ring + t * (kFewRows * 4) + f * 4;
      if constexpr (BWD) {
        gate_in[j] = c < p.F ? load_value<bf16>(p.gate, t * p.ldgate + c) : 0.f;
        up_in[j] = c < p.F ? load_value<bf16>(p.up, t * p.ldup + c) : 0.f;
      }
    }
    for (int s = 0; s < fp.splits; ++s) {
      float v[kBatch], w[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t from = mapa_shared(at[j], s);
        v[j] = ld_cluster_f32(from);
        w[j] = BWD ? 0.f : ld_cluster_f32(from + kTileF * 4);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) a[j] += v[j], b[j] += w[j];
    }
    // act and the checkpoint's exponents of the batch together: chains that
    // would take 0.4 us an item one after the other
    if constexpr (!BWD) {
      float h[kBatch];
      with_activation(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) h[j] = gate<decltype(act)::value, false>(a[j]).a * b[j];
      });
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = i0 + j * kWarps, t = t0 + i / kGroups, c = f0 + (i % kGroups) * 32 + lane;
        if (i >= items || c >= p.F) continue;
        store_value<bf16>(p.out[0], t * p.ldout[0] + c, h[j]);
        if (p.out[1]) {
          store_value<bf16>(p.out[1], t * p.ldout[1] + c, a[j]);
          store_value<bf16>(p.out[2], t * p.ldout[2] + c, b[j]);
        }
      }
    } else {
      float h[kBatch], g[kBatch], u[kBatch];  // act(G) U (0 past F), dG, dU
      uint32_t top[kBatch];
      with_activation(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const GateValue v = gate<decltype(act)::value, true>(gate_in[j]);
          h[j] = v.a * up_in[j];
          g[j] = a[j] * up_in[j] * v.slope;
          u[j] = a[j] * v.a;
          top[j] = __float_as_uint(h[j]) & 0x7FFFFFFFu;
        }
      });
      if (p.ck.q) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
          for (int j = 0; j < kBatch; ++j) top[j] = max(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = i0 + j * kWarps, t = t0 + i / kGroups, c = f0 + (i % kGroups) * 32 + lane;
        if (i >= items || c >= p.F) continue;
        store_value<bf16>(p.out[0], t * p.ldout[0] + c, g[j]);
        store_value<bf16>(p.out[1], t * p.ldout[1] + c, u[j]);
        if (!p.ck.q) continue;
        const uint32_t e = q8_exponent(top[j]);
        p.ck.q[t * p.ck.ldq + c] = (int8_t)q8_byte(h[j], q8_inverse(e), e);
        if (lane == 0) p.ck.e[t * p.ck.lde + (c >> 5)] = (uint8_t)e;
      }
    }
  }
  cluster_sync_all();  // no CTA leaves while another reads its sums
}

template <int TN, bool KM, bool BWD>
cudaError_t launch(const GatedMaps &m, const FewParams &p, int grid, cudaStream_t st) {
  using Cfg = FewCfg<TN>;
  auto kern = gated_few_kernel<TN, KM, BWD>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3((unsigned)grid), dim3(kFewThreads), Cfg::kSmemBytes, st, p.splits, m.a, m.b[0], m.b[1], p);
}
template <bool KM, bool BWD>
cudaError_t launch_tokens(int tn, const GatedMaps &m, const FewParams &p, int grid, cudaStream_t st) {
  return tn == 16   ? launch<16, KM, BWD>(m, p, grid, st)
         : tn == 32 ? launch<32, KM, BWD>(m, p, grid, st)
                    : launch<64, KM, BWD>(m, p, grid, st);
}

}  // namespace

int gated_few_columns(int64_t T) { return T <= 16 ? 16 : T <= 32 ? 32 : 64; }

cudaError_t launch_gated_few(bool forward, bool km, const GatedMaps &m, const GatedTcParams &p, int sms,
                             cudaStream_t st) {
  const int tn = gated_few_columns(p.T), tile_f = forward ? kFewRows / 2 : kFewRows, tiles = (p.F + tile_f - 1) / tile_f;
  // The split: up to a CTA an SM or a quarter more, at least one k-block each
  // (eight CTAs of a cluster: eight); where that leaves 32 k-blocks or more to
  // each, twice as many, as long as all are resident at once (three an SM).
  // Forward in us by 1, 2, 4 and 8: 16 tokens 4096 x 2048 (32 tiles) 20.4, 11.7,
  // 7.9, 9.7; 64 tokens 768 x 4096 (64) 8.5, 6.4, 8.5, 15.6; 48 tokens 4096 x
  // 11008 (172) 40, 34.6, 39, 49.
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= sms * 5 / 4 && p.num_kb >= (splits == 4 ? 64 : splits * 2)) splits *= 2;
  if (splits < 8 && p.num_kb >= splits * 32 && tiles * splits * 2 <= sms * 3) splits *= 2;
  const FewParams fp{p, splits};
  const int grid = tiles * splits;
  if (forward) return km ? launch_tokens<true, false>(tn, m, fp, grid, st) : launch_tokens<false, false>(tn, m, fp, grid, st);
  return km ? launch_tokens<true, true>(tn, m, fp, grid, st) : launch_tokens<false, true>(tn, m, fp, grid, st);
}

}  // namespace gb300
