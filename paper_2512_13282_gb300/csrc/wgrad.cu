// wgrad.cu -- planning and launches of the weight gradient's tensor-core
// kernel (wgrad_tc.cuh), and the reduction of its split tail.
#include <atomic>
#include <cmath>

#include "layer_rows.cuh"
#include "wgrad_tc.cuh"

namespace gb300 {

namespace {

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Longest chain of tensor-core additions of a float32 result, in k-blocks
// of 64 tokens.  Measured error of dW against 64 bits (2-norm, 1000 tokens of
// 777 x 1501): 8.1e-8, 1.1e-7, 2.2e-7 and 5.1e-7 with slabs of 2, 4, 8 and 16
// k-blocks; with 16 an element of random products is off by more than 2^-20 of
// their magnitudes' sum.  (The header's bound is of 8.)
constexpr int kSlabKb = 8;
// The same of a bf16 result: 8192 tokens, whose additions lose at most a tenth
// of what its last rounding may (without a limit, millions of tokens lost more
// than that).  4096 x 4096: 16384 tokens 329 us, in one chain 327; 32768 tokens
// 665 and 671.
constexpr int kSlabKbBf16 = 128;

// Most k-blocks for which base comes through shared memory: its blocks displace
// two stages of operands, which longer reductions miss.  4096 x 4096 bf16 with
// base, through registers / through shared memory: 768 tokens 34.7 / 33.4 us,
// 1024 37.1 / 39.0, 2048 56.4 / 65.9.
constexpr int kBaseKb = 12;

template <int BN, bool PAIR, bool SLABS, bool BASE>
cudaError_t launch_kernel(const WgradMaps &m, const WgradParams &p, int grid, cudaStream_t st) {
  using Cfg = WgCfg<BN, PAIR, BASE>;
  auto kern = wgrad_kernel<BN, PAIR, SLABS, BASE>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, Cfg::kSmemBytes, allowed);
  if (e != cudaSuccess) return e;
  if (SLABS) {
    // its epilogue takes registers over from the other warps, and would wait
    // for ever if the block were launched with fewer than that adds up to
    static std::atomic<int> regs{0};
    if (regs.load() == 0) {
      cudaFuncAttributes attr;
      const cudaError_t f = cudaFuncGetAttributes(&attr, kern);
      if (f != cudaSuccess) return f;
      regs.store(attr.numRegs);
    }
    if (regs.load() < kWgLaunchRegs) return cudaErrorLaunchOutOfResources;
  }
  return launch_ex(kern, dim3((unsigned)grid), dim3(kWgThreads), Cfg::kSmemBytes, st, PAIR ? 2 : 1, m.a, m.b, m.out,
                   m.partials, m.base, p);
}

template <int BN, bool PAIR>
cudaError_t launch_tile(const WgradMaps &m, const WgradParams &p, int grid, cudaStream_t st) {
  if (p.tc.num_kb > p.tc.slab_kb) return launch_kernel<BN, PAIR, true, false>(m, p, grid, st);
  if (p.base && p.tc.out_tma == kOutTmaC && p.tc.num_kb <= kBaseKb)
    return launch_kernel<BN, PAIR, false, true>(m, p, grid, st);
  return launch_kernel<BN, PAIR, false, false>(m, p, grid, st);
}

// Split tail: element group t (4 columns of a row) of the compact partials,
// over the tail tiles' rows; the partials' bytes, mostly in L2, bound it (four
// tiles split 16 ways: 6 us, launch included).
__global__ void __launch_bounds__(256) wgrad_reduce_kernel(const WgradParams wp, int bn, int tile_m, int64_t groups) {
  griddep_launch_dependents();
  griddep_wait();
  const TcParams &p = wp.tc;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= groups) return;
  const int per_row = bn / 4;
  const int64_t prow = t / per_row;
  const int pc = (int)(t - prow * per_row) * 4;
  const int slot = (int)(prow / tile_m);
  int tm, tn;
  raster_tile(p.tail_first + slot, p.tiles_m, p.tiles_n, p.group_m, &tm, &tn);
  const int64_t row = (int64_t)tm * tile_m + (prow - (int64_t)slot * tile_m);
  const int64_t col = (int64_t)tn * bn + pc;
  if (row >= p.M || col >= p.N) return;
  const int64_t plane = (int64_t)(p.tiles_m * p.tiles_n - p.tail_first) * tile_m * bn;
  const float *src = static_cast<const float *>(p.ws) + prow * bn + pc;
  float4 s = *reinterpret_cast<const float4 *>(src);
  for (int k = 1; k < p.tail_splits; ++k) {
    const float4 v = *reinterpret_cast<const float4 *>(src + k * plane);
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (col + i >= p.N) break;
    float r = v[i];
    if (wp.out_bf16) {
      if (wp.base)
        r += __bfloat162float(static_cast<const __nv_bfloat16 *>(wp.base)[row * wp.ldbase + col + i]);
      static_cast<__nv_bfloat16 *>(p.C)[row * p.ldc + col + i] = __float2bfloat16_rn(r);
    } else {
      if (wp.base) r += static_cast<const float *>(wp.base)[row * wp.ldbase + col + i];
      static_cast<float *>(p.C)[row * p.ldc + col + i] = r;
    }
  }
}

// 32-bit words that hold the bytes from p on, p any address: BYTES / 4 of
// them, from aligned words (one more than that is read where p is not
// aligned: up to 3 bytes before p and after the last byte asked for).
template <int BYTES>
__device__ __forceinline__ void load_shifted(const void *p, uint32_t (&w)[BYTES / 4]) {
  const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 3u;
  const uint32_t *a = reinterpret_cast<const uint32_t *>(reinterpret_cast<uintptr_t>(p) - off);
  uint32_t v[BYTES / 4 + 1];
#pragma unroll
  for (int i = 0; i < BYTES / 4; ++i) v[i] = a[i];
  v[BYTES / 4] = off ? a[BYTES / 4] : 0;
#pragma unroll
  for (int i = 0; i < BYTES / 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], off * 8);
}

// A thread writes 8 values (16 bytes) of a row of the restored X or, past
// them, of the copied gradient (1000 x 777 and 1000 x 1501: 5 us for both; two
// launches with element accesses took 14).  The source's words are read aligned and
// shifted into place; within 8 values of a row's ends, where such a word may
// reach outside the matrix, its elements are read one by one.
__global__ void __launch_bounds__(256)
    wgrad_stage_kernel(Q8Ref ck, int64_t T, int64_t K, uint16_t *x, int64_t ldx, const uint16_t *g, int64_t ldg,
                       int64_t N, uint16_t *gx, int64_t ldgx) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t xe = ldx / 8, ge = g ? ldgx / 8 : 0, x_items = T * xe, items = x_items + T * ge;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < items; t += (int64_t)gridDim.x * 256) {
    const bool is_x = t < x_items;
    const int64_t u = is_x ? t : t - x_items, per = is_x ? xe : ge;
    const int64_t r = u <= 0xFFFFFFFFll ? (int64_t)((uint32_t)u / (uint32_t)per) : u / per;
    const int64_t c = (u - r * per) * 8, cols = is_x ? K : N;
    const bool inside = c >= 8 && c + 16 <= cols;
    const int n = (int)min((int64_t)8, cols - c);
    uint32_t o[4];
    if (is_x) {
      const int8_t *src = ck.q + r * ck.ldq + c;
      uint32_t w[2] = {0, 0};
      if (inside) {
        load_shifted<8>(src, w);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) w[i / 4] |= (uint32_t)(uint8_t)src[i] << (8 * (i & 3));
      }
      const __nv_bfloat162 s = __float2bfloat162_rn(q8_scale(ck.e[r * ck.lde + (c >> 5)]));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s8x4_to_bf16x4(w[i], o[2 * i], o[2 * i + 1]);
        o[2 * i] = scale_bf16x2(o[2 * i], s);
        o[2 * i + 1] = scale_bf16x2(o[2 * i + 1], s);
      }
    } else {
      const uint16_t *src = g + r * ldg + c;
      if (inside) {
        load_shifted<16>(src, o);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) o[i / 2] |= (uint32_t)src[i] << (16 * (i & 1));
      }
    }
    *reinterpret_cast<uint4 *>((is_x ? x + r * ldx : gx + r * ldgx) + c) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// T == 0: C = base, or zero.
__global__ void __launch_bounds__(256) wgrad_base_kernel(const WgradParams wp) {
  griddep_launch_dependents();
  griddep_wait();
  const TcParams &p = wp.tc;
  const int64_t n = (int64_t)p.M * p.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / p.N, c = i - r * p.N;
    if (wp.out_bf16)
      static_cast<uint16_t *>(p.C)[r * p.ldc + c] =
          wp.base ? static_cast<const uint16_t *>(wp.base)[r * wp.ldbase + c] : (uint16_t)0;
    else
      static_cast<float *>(p.C)[r * p.ldc + c] =
          wp.base ? static_cast<const float *>(wp.base)[r * wp.ldbase + c] : 0.f;
  }
}

// Modelled cost of a tile shape, fitted to forced plans on GB300 (T from 16
// to 8192, K and N from 256 to 12288, every shape and split): microseconds per
// k-block of 64 tokens and per unit besides, and what a unit takes at least to
// write its tile (and read base's): its latency, and the bytes at a slot's
// share of the memory.  The narrow tiles move twice and four times the operand
// bytes a flop, which shared memory paces; with few tokens, where the output
// sets the time, they fill the device in rounds that leave less of it idle
// (128 tokens, 4096 x 4096 float32 with base: 27.2 us, pairs 34.0; 2048 tokens:
// 88 us, pairs 76; without base 83 and 61).  192-wide pairs take as long a k-block as 256-wide
// ones and are not compiled.
struct TileCost {
  WgradTile tile;
  double kb_us, unit_us, least_us, bytes_per_us;
};
constexpr TileCost kTiles[] = {{{true, 256}, 0.36, 1.2, 3.2, 65e3},
                               {{false, 128}, 0.33, 0.5, 1.45, 35e3},
                               {{false, 64}, 0.30, 0.4, 0.9, 35e3}};
// A split tail's reduction: its launch, and the partials written and read.
constexpr double kTailFixedUs = 3.5, kTailUsPerMB = 0.36;

}  // namespace

WgradPlan plan_wgrad(int64_t M, int64_t N, int64_t T, int out_bytes, bool base, int sms, int pairs) {
  WgradPlan best{};
  double best_us = -1;
  const int64_t num_kb = ceil_div64(T, kBK);
  for (const TileCost &tc : kTiles) {
    const int64_t slots = tc.tile.pair ? pairs : sms;
    if (slots <= 0) continue;
    const int tile_m = tc.tile.pair ? 2 * kBM : kBM;
    const int64_t tiles_m = ceil_div64(M, tile_m), tiles_n = ceil_div64(N, tc.tile.bn), tiles = tiles_m * tiles_n;
    const int64_t full = tiles / slots, rem = tiles % slots;
    const double tile_bytes = (double)tile_m * tc.tile.bn;
    const auto unit_us = [&](int64_t kb, double bytes) {
      return fmax(kb * tc.kb_us + tc.unit_us, fmax(tc.least_us, bytes / tc.bytes_per_us));
    };
    const double out = tile_bytes * out_bytes * (base ? 2 : 1), whole = unit_us(num_kb, out);
    for (int64_t s = 1; s <= 16; ++s) {
      int64_t kb_per = num_kb, parts = 1;
      if (s > 1) {
        if (rem == 0 || rem * s > slots) break;
        kb_per = ceil_div64(num_kb, s);
        parts = ceil_div64(num_kb, kb_per);  // no part is empty
        if (parts != s || kb_per < 4) continue;
      }
      double us = full * whole;
      if (rem > 0) us += parts > 1 ? unit_us(kb_per, tile_bytes * 4) : whole;
      if (parts > 1) us += kTailFixedUs + kTailUsPerMB * (double)parts * rem * tile_bytes * 4e-6;
      if (best_us < 0 || us < best_us) {
        best_us = us;
        best.tile = tc.tile;
        best.tiles_m = (int)tiles_m;
        best.tiles_n = (int)tiles_n;
        best.num_kb = (int)num_kb;
        best.tail_first = parts > 1 ? (int)(full * slots) : 0;
        best.tail_splits = parts > 1 ? (int)parts : 0;
        best.tail_kb_per = parts > 1 ? (int)kb_per : 0;
        const int64_t units = parts > 1 ? full * slots + rem * parts : tiles;
        best.grid = (int)(units < slots ? units : slots) * (tc.tile.pair ? 2 : 1);
      }
    }
  }
  return best;
}

size_t wgrad_partial_bytes(const WgradPlan &pl) {
  if (pl.tail_splits < 2) return 0;
  const size_t tail = (size_t)pl.tiles_m * pl.tiles_n - pl.tail_first;
  return (size_t)pl.tail_splits * tail * (pl.tile.pair ? 2 * kBM : kBM) * pl.tile.bn * 4;
}

cudaError_t launch_wgrad(const WgradTile &tile, const WgradMaps &m, const WgradParams &p, int grid, cudaStream_t st) {
  WgradParams q = p;
  q.tc.slab_kb = p.out_bf16 ? kSlabKbBf16 : kSlabKb;
  if (tile.pair) return launch_tile<256, true>(m, q, grid, st);
  return tile.bn == 128 ? launch_tile<128, false>(m, q, grid, st) : launch_tile<64, false>(m, q, grid, st);
}

cudaError_t launch_wgrad_stage(const Q8Ref &ck, int64_t T, int64_t K, uint16_t *x, int64_t ldx, const uint16_t *g,
                               int64_t ldg, int64_t N, uint16_t *gx, int64_t ldgx, cudaStream_t st) {
  const int64_t blocks = ceil_div64(T * (ldx / 8 + (g ? ldgx / 8 : 0)), 256);
  return launch_ex(wgrad_stage_kernel, dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30))), dim3(256), 0, st, 1,
                   ck, T, K, x, ldx, g, ldg, N, gx, ldgx);
}

cudaError_t launch_wgrad_base(const WgradParams &p, int sms, cudaStream_t st) {
  const int64_t want = ceil_div64((int64_t)p.tc.M * p.tc.N, 1024), cap = (int64_t)sms * 8;
  return launch_ex(wgrad_base_kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(256), 0, st, 1, p);
}

cudaError_t launch_wgrad_reduce(const WgradTile &tile, const WgradParams &p, cudaStream_t st) {
  const int tile_m = tile.pair ? 2 * kBM : kBM;
  const int64_t tail = (int64_t)p.tc.tiles_m * p.tc.tiles_n - p.tc.tail_first;
  const int64_t groups = tail * tile_m * (tile.bn / 4);
  return launch_ex(wgrad_reduce_kernel, dim3((unsigned)ceil_div64(groups, 256)), dim3(256), 0, st, 1, p, tile.bn,
                   tile_m, groups);
}

}  // namespace gb300
