// layer_ln_fwd.cu -- layer norm forward, optionally with the result's 8-bit
// checkpoint:
//     y = (x - mu) * rstd * gamma + beta,  rstd = 1 / sqrt(var + eps),
// mu and var of a row, var from the differences x - mu (a second sum over the
// row, held in registers).  Sums are float32; y is rounded once, to its type.
//
// A mean far above the deviations costs no digits: the sum of x times 1/n, m,
// is off by roundings of the size of |x|, and where that exceeds the
// deviations (far_mean) a third sum, over d = x - m, takes them out again.  Its
// average c is off by roundings of the size of the deviations only, and
//     mu = m + c,  x - mu = d - c,  var = avg(d^2) - c^2.
//
// HBM bounds it: each value read once and written once, 4 bytes in bf16, and 1
// more for the checkpoint.  Measured, back to back, bf16, against a plain copy
// of as many bytes: 8192 x 4096 28.6 us (4.7 TB/s; copy 23.1), with the
// checkpoint 38.6 us; 32768 x 4096 97 us (5.5 TB/s; copy 82).  What is left is
// a row's two block-wide sums, one after the other: neither issue (64 % of the
// cycles with the checkpoint) nor the HBM is full.
#include <atomic>

#include <type_traits>

#include "layer_rows.cuh"

namespace gb300 {

namespace {

// Whether a row's mean is more than two standard deviations from zero, so that
// its roundings matter beside those of the deviations (`squares`: the average
// of d^2).  False for a row with a NaN.  Taking the average of d for every row,
// in the same sum as d^2, cost 9 % (32768 x 1024 bf16: 33.0 us, without 30.3).
__device__ __forceinline__ bool far_mean(float mean, float squares) { return mean * mean > 4.f * squares; }
// avg(d^2) - c^2, not below zero by roundings (a NaN stays one).
__device__ __forceinline__ float variance(float squares, float c) {
  const float v = fmaf(-c, c, squares);
  return v < 0.f ? 0.f : v;
}

constexpr int kAnyThreads = 256, kAnyBlocks = 8;  // blocks an SM

// Any width, pitch and alignment: a block per row, the row read three times
// (mean, variance, result), the second and third time from L1 or L2.  For rows
// above 16384 values and unaligned ones below 64 only: 8192 x 4096 with its
// checkpoint takes 300 us here.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kAnyThreads, kAnyBlocks) ln_forward_any_kernel(const LnForward p) {
  __shared__ float2 sm[2][32];
  griddep_launch_dependents();
  griddep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float inv_n = 1.0f / (float)p.cols;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const TX *x = static_cast<const TX *>(p.x) + r * p.ldx;
    float s = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kAnyThreads) s += load_value<TX>(x, c);
    const float mean = block_sum2(s, 0.f, sm, 0).x * inv_n;
    float v = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kAnyThreads) {
      const float d = load_value<TX>(x, c) - mean;
      v = fmaf(d, d, v);
    }
    float var = block_sum2(v, 0.f, sm, 1).x * inv_n, rest = 0.f;
    if (far_mean(mean, var)) {
      float t = 0.f;
      for (int c = threadIdx.x; c < p.cols; c += kAnyThreads) t += load_value<TX>(x, c) - mean;
      // (the buffer's last reads came before the barrier of the sum between)
      rest = block_sum2(t, 0.f, sm, 0).x * inv_n;
      var = variance(var, rest);
      __syncthreads();  // the next row writes the same buffer
    }
    const float rstd = rsqrtf(var + p.eps), shift = -rest * rstd;
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[r] = mean + rest;
      if (p.rstd) p.rstd[r] = rstd;
    }
    TY *y = static_cast<TY *>(p.y) + r * p.ldy;
    // each warp takes whole blocks of 32 columns, so that a checkpoint block
    // is the warp's 32 lanes
    for (int c0 = warp * 32; c0 < p.cols; c0 += kAnyThreads) {
      const int c = c0 + lane;
      float out = 0.f;
      if (c < p.cols) {
        out = fmaf(fmaf(load_value<TX>(x, c) - mean, rstd, shift), load_param(p.gamma, p.param_type, c, 1.f),
                   load_param(p.beta, p.param_type, c, 0.f));
        store_value<TY>(y, c, out);
      }
      if (p.ck.q) {
        out = as_stored<TY>(out);
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(out) & 0x7FFFFFFFu);
        const uint32_t e = q8_exponent(top);
        if (c < p.cols) p.ck.q[r * p.ck.ldq + c] = (int8_t)q8_byte(out, q8_inverse(e), e);
        if (lane == 0) p.ck.e[r * p.ck.lde + (c0 >> 5)] = (uint8_t)e;
      }
    }
  }
}


// A lane's 8 consecutive results (zero past the row's end), rounded to y's type
// and stored, and their part of the checkpoint of y as stored (four lanes hold
// a block).  All lanes of the warp call it, also those past the row's end.
template <typename TY, bool SHIFT>
__device__ __forceinline__ void store_eighth(TY *y, const Q8Ref &ck, int64_t r, int c, int cols, const float2 (&v)[4]) {
  const bool in = c < cols;
  float2 o[4];
  uint32_t top = 0, h[2 * sizeof(TY)];
  if constexpr (sizeof(TY) == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = pack_bf16x2(v[j].x, v[j].y);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) h[2 * j] = __float_as_uint(v[j].x), h[2 * j + 1] = __float_as_uint(v[j].y);
  }
  store_group<TY, SHIFT>(y, c, cols, h);
  if (!ck.q) return;
  if constexpr (sizeof(TY) == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = make_float2(__uint_as_float(h[j] << 16), __uint_as_float(h[j] & 0xFFFF0000u));
    top = max_magnitude_bf16<4>(h);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[j] = v[j];
      top = max(top, max(h[2 * j] & 0x7FFFFFFFu, h[2 * j + 1] & 0x7FFFFFFFu));
    }
  }
  if (!in) top = 0;  // not in the block
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t e = q8_exponent(top);
  const uint2 q = q8_pack8(o, e);
  if (!SHIFT && !in) return;
  const uint32_t w[2] = {q.x, q.y};
  store_group<int8_t, SHIFT>(ck.q + r * ck.ldq, c, cols, w);
  if (in && (c & 31) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)e;
}

// Rows of up to THREADS * NV * 8 values, at least 64 where V is not 8, read once and
// kept in registers until they are written.  A block of threads walks rows
// gridDim.x apart, which come through a ring of slots that bulk copies fill
// (SlotRow); one row ahead in registers instead was not enough in flight (3
// blocks of 8 KB rows an SM: 24 KB, where the copy rate times the latency asks
// for 40).  The first of a row's two barriers, the sums for its mean and its
// variance (a third with far_mean), frees its slot.  gamma and beta stay in registers (NV = 1), else in
// shared memory as float32 where the rings leave room (params_shared), so that
// 1024 threads share an SM whatever the width: with 16 parameters a thread in
// registers half as many fit (8192 x 8192 with checkpoint: 77.4 us, from shared
// memory 72.4).
template <typename TX, typename TY, int NV, int THREADS, int V>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
    ln_forward_ring_kernel(const LnForward p, const int stages, const uint32_t x_bytes, const int params_shared,
                           uint32_t *err, const uint64_t wait_limit_ns) {
  constexpr bool kKeep = NV == 1;
  static_assert(kKeep || V != 1, "parameters in shared memory are for groups of eight");
  using Row = std::conditional_t<V == kShifted, ShiftedRow<TX>, SlotRow<TX, V == 1 ? 1 : 8, THREADS>>;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) float sm[3][32];
  __shared__ __align__(8) uint64_t bars[kMaxStages];
  __shared__ volatile uint32_t abort_flag;
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_addr(slots), bar0 = smem_addr(bars);
  const int param_cols = (p.cols + 7) / 8 * 8;
  float *shared_gamma = reinterpret_cast<float *>(slots + stages * x_bytes), *shared_beta = shared_gamma + param_cols;
  RingPlace use, put;  // put: thread 0's
  const float inv_n = 1.0f / (float)p.cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 32) sm[0][threadIdx.x] = sm[1][threadIdx.x] = sm[2][threadIdx.x] = 0.f;
  __syncthreads();
  griddep_wait();
  const int64_t mine = (p.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;  // rows of this block, at least one
  const auto row_of = [&](int64_t i) { return (int64_t)blockIdx.x + i * gridDim.x; };
  const auto x_row = [&](int64_t i) { return static_cast<const TX *>(p.x) + row_of(i) * p.ldx; };
  const auto fill = [&](int64_t i) {
    const uint32_t dst = ring + put.slot * x_bytes, bar = bar0 + 8u * put.slot;
    put.advance(stages);
    const uint32_t bytes = Row::copy_bytes(x_row(i), p.cols);
    mbar_arrive_expect_tx(bar, bytes);
    Row::copy(dst, x_row(i), bytes, bar);
  };
  int64_t filled = mine < stages ? mine : stages;
  if (threadIdx.x == 0)
    for (int64_t i = 0; i < filled; ++i) fill(i);
  Row xr;
  if constexpr (V == kShifted) {
    // a row's ends go into its slot while the row before is worked on
    xr.fetch_ends(x_row(0), p.cols);
    xr.put_ends(slots, xr.offset(x_row(0)), p.cols);
    if (mine > 1) xr.fetch_ends(x_row(1), p.cols);
    __syncthreads();
  } else {
    xr.init(p.cols);
    xr.fetch_ends(x_row(0));
  }
  const auto gamma_at = [&](int c) { return c < p.cols ? load_param(p.gamma, p.param_type, c, 1.f) : 0.f; };
  // place of column c's parameters in shared memory: the first four of every
  // eight and then the others, so that a warp's 16-byte reads follow one another
  const auto param_at = [&](int c) { return ((c >> 2) & 1) * (param_cols / 2) + (c >> 3) * 4 + (c & 3); };
  const auto beta_at = [&](int c) { return c < p.cols ? load_param(p.beta, p.param_type, c, 0.f) : 0.f; };
  float2 gamma[kKeep ? NV * 4 : 1], beta[kKeep ? NV * 4 : 1];
  if constexpr (kKeep) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = group_col<V, THREADS>(v, 2 * j), d = group_col<V, THREADS>(v, 2 * j + 1);
        gamma[v * 4 + j] = make_float2(gamma_at(c), gamma_at(d));
        beta[v * 4 + j] = make_float2(beta_at(c), beta_at(d));
      }
  } else if (params_shared) {
    // read past the first row's barriers; eight columns in flight a thread
    for (int c0 = threadIdx.x; c0 < param_cols; c0 += 8 * blockDim.x) {
      float g[8], b[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        g[k] = gamma_at(c0 + k * blockDim.x);
        b[k] = beta_at(c0 + k * blockDim.x);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int c = c0 + k * (int)blockDim.x;
        if (c < param_cols) shared_gamma[param_at(c)] = g[k], shared_beta[param_at(c)] = b[k];
      }
    }
  }
  bool ok = true;
  int64_t done = 0;
  for (int64_t i = 0; i < mine; done = ++i, use.advance(stages)) {
    const int64_t r = row_of(i);
    ok = mbar_wait(bar0 + 8u * use.slot, use.parity, &abort_flag, err, wait_limit_ns);
    uint8_t *slot = slots + use.slot * x_bytes;
    const uint32_t off = xr.offset(x_row(i));
    if constexpr (V == 1) {
      if (ok) xr.put_ends(slot, off);
      if (i + 1 < mine) xr.fetch_ends(x_row(i + 1));
    }
    if constexpr (V == kShifted) {
      // (that slot's last reads came before the barrier of the row before)
      RingPlace next = use;
      next.advance(stages);
      if (i + 1 < mine) xr.put_ends(slots + next.slot * x_bytes, xr.offset(x_row(i + 1)), p.cols);
      if (i + 2 < mine) xr.fetch_ends(x_row(i + 2), p.cols);
    }
    float2 x[NV * 4], s2 = both(0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float2 e[4], t = both(0.f);
      xr.load(slot, off, v, p.cols, e);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[v * 4 + j] = e[j];
        t = add2(t, e[j]);
      }
      s2 = add2(s2, V == 1 || group_col<V, THREADS>(v, 0) < p.cols ? t : both(0.f));
    }
    const float s = warp_sum(s2.x + s2.y);
    if (lane == 0) sm[0][warp] = s;
    // every wait of the block succeeded, or the block gives up together
    if (!__syncthreads_and(ok)) {
      ok = false;
      break;
    }
    if (threadIdx.x == 0 && filled < mine) fill(filled++);  // this row's slot
    const float mean = sum_over_warps<THREADS / 32>(sm[0]) * inv_n;
    float2 v2 = both(0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float2 t = both(0.f), d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] = add2(x[v * 4 + j], both(-mean));
        if constexpr (V == 1) {
          if (group_col<V, THREADS>(v, 2 * j) >= p.cols) d[j].x = 0.f;
          if (group_col<V, THREADS>(v, 2 * j + 1) >= p.cols) d[j].y = 0.f;
        }
      }
      if (V == kShifted && group_col<V, THREADS>(v, 8) > p.cols) zero_from(d, p.cols - group_col<V, THREADS>(v, 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[v * 4 + j] = d[j];
        t = fma2(d[j], d[j], t);
      }
      v2 = add2(v2, V == 1 || group_col<V, THREADS>(v, 0) < p.cols ? t : both(0.f));
    }
    const float squares = warp_sum(v2.x + v2.y);
    if (lane == 0) sm[1][warp] = squares;
    __syncthreads();
    float var = sum_over_warps<THREADS / 32>(sm[1]) * inv_n, rest = 0.f;
    if (far_mean(mean, var)) {  // the same for every thread
      float2 c2 = both(0.f);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const float2 t = add2(add2(x[v * 4], x[v * 4 + 1]), add2(x[v * 4 + 2], x[v * 4 + 3]));
        c2 = add2(c2, V == 1 || group_col<V, THREADS>(v, 0) < p.cols ? t : both(0.f));
      }
      const float c = warp_sum(c2.x + c2.y);
      if (lane == 0) sm[2][warp] = c;
      __syncthreads();
      rest = sum_over_warps<THREADS / 32>(sm[2]) * inv_n;
      var = variance(var, rest);
    }
    const float rstd = rsqrtf(var + p.eps);
    const float2 shift = both(-rest * rstd);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[r] = mean + rest;
      if (p.rstd) p.rstd[r] = rstd;
    }
    TY *y = static_cast<TY *>(p.y) + r * p.ldy;
    int8_t *q_row = p.ck.q + r * p.ck.ldq;
    uint8_t *e_row = p.ck.e + r * p.ck.lde;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c0 = group_col<V, THREADS>(v, 0);
      float2 g[4], b[4], o[4];
      if constexpr (kKeep) {
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] = gamma[v * 4 + j], b[j] = beta[v * 4 + j];
      } else {
        if (params_shared) {
          const int at = c0 < p.cols ? param_at(c0) : 0, half = param_cols / 2;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float4 gq = *reinterpret_cast<const float4 *>(shared_gamma + at + h * half);
            const float4 bq = *reinterpret_cast<const float4 *>(shared_beta + at + h * half);
            g[2 * h] = make_float2(gq.x, gq.y), g[2 * h + 1] = make_float2(gq.z, gq.w);
            b[2 * h] = make_float2(bq.x, bq.y), b[2 * h + 1] = make_float2(bq.z, bq.w);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            g[j] = make_float2(gamma_at(c0 + 2 * j), gamma_at(c0 + 2 * j + 1));
            b[j] = make_float2(beta_at(c0 + 2 * j), beta_at(c0 + 2 * j + 1));
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fma2(fma2(x[v * 4 + j], both(rstd), shift), g[j], b[j]);
      if constexpr (V != 1) {
        store_eighth<TY, V == kShifted>(y, p.ck, r, c0, p.cols, o);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = group_col<V, THREADS>(v, k);
          const float w = (k & 1) ? o[k >> 1].y : o[k >> 1].x;
          if (c < p.cols) store_value<TY>(y, c, w);
          if (p.ck.q && c - lane < p.cols) {  // the warp's 32 columns are a block
            const float h = c < p.cols ? as_stored<TY>(w) : 0.f;
            const uint32_t e = q8_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7FFFFFFFu));
            if (c < p.cols) q_row[c] = (int8_t)q8_byte(h, q8_inverse(e), e);
            if (lane == 0) e_row[c >> 5] = (uint8_t)e;
          }
        }
      }
    }
  }
  if (!ok && threadIdx.x == 0) ring_drain(bar0, stages, use, filled - done);
}

// Blocks of a kernel that an SM holds at once, asked once a kernel, block
// shape and shared memory size (the devices served are all the same).
template <typename K>
int blocks_per_sm(K kern, int threads, size_t smem, std::atomic<uint64_t> &known) {
  const uint64_t key = (uint64_t)smem << 24 | (uint64_t)threads << 8;
  const uint64_t k = known.load(std::memory_order_relaxed);
  if ((k & ~(uint64_t)0xFF) == key && (k & 0xFF)) return (int)(k & 0xFF);
  int n = 0;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, threads, smem) != cudaSuccess || n < 1) n = 1;
  known.store(key | (uint64_t)n, std::memory_order_relaxed);
  return n;
}

// Blocks that fill the device once, no more than there are rows.
unsigned persistent_grid(int per_sm, int64_t rows, int sms) {
  const int64_t most = (int64_t)sms * per_sm;
  return (unsigned)(rows < most ? rows : most);
}

template <typename TX, typename TY, int NV, int THREADS, int V>
cudaError_t run_ring(const LnForward &p, const OpContext &c) {
  static std::atomic<uint64_t> known{0};
  const auto kern = ln_forward_ring_kernel<TX, TY, NV, THREADS, V>;
  const int eights = (p.cols + 7) / 8, threads = V == 1 ? THREADS : ((eights + NV - 1) / NV + 31) / 32 * 32;
  const uint32_t x_bytes =
      V == kShifted ? shifted_slot_bytes(p.cols, sizeof(TX)) : slot_bytes(p.cols, sizeof(TX), V == 8);
  // the rings of the blocks that registers allow share the memory, with the
  // parameters where those stay in it; fewer blocks where two slots would not
  // fit beside them (8192 x 4096 float32: 98 us with four blocks that read the
  // parameters from global memory for every row, 45.4 with three)
  int want = 1024 / threads;
  if (want > 16) want = 16;
  int64_t param_bytes = NV > 1 ? 64 * (int64_t)eights : 0;
  while (want > 1 && param_bytes && kRingBytes / want - param_bytes < 2 * (int64_t)x_bytes) --want;
  const int64_t room = kRingBytes / want;
  if (room - param_bytes < 2 * (int64_t)x_bytes) param_bytes = 0;
  int64_t stages = (room - param_bytes) / x_bytes;
  stages = stages < 2 ? 2 : stages > kMaxStages ? kMaxStages : stages;
  const size_t smem = (size_t)(stages * x_bytes + param_bytes);
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, kRingBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(persistent_grid(blocks_per_sm(kern, threads, smem, known), p.rows, c.sms)), dim3(threads),
                   smem, c.st, 1, p, (int)stages, x_bytes, param_bytes ? 1 : 0, c.err, c.wait_limit_ns);
}

// Rows of up to 128 eights, at any alignment, are a value a lane at a time (V =
// 1: 2560 x 777 bf16 7.1 us, shifted 9.0), wider ones shifted (3543 x 5690 bf16,
// with checkpoint: 42 us, 69; shifted 35.5, 51; float32 without one 42 and 48).
template <typename TX, typename TY, int V>
cudaError_t run_width(const LnForward &p, const OpContext &c) {
  const int eights = (p.cols + 7) / 8;
  if (V == 1 && eights <= 32) return run_ring<TX, TY, 1, 32, 1>(p, c);
  if (V == 1 && eights <= 64) return run_ring<TX, TY, 1, 64, 1>(p, c);
  if (eights <= 128) return run_ring<TX, TY, 1, 128, V>(p, c);
  constexpr int W = V == 1 ? kShifted : V;
  if (eights <= 512) return run_ring<TX, TY, 2, 256, W>(p, c);
  return eights <= 1024 ? run_ring<TX, TY, 2, 512, W>(p, c) : run_ring<TX, TY, 2, 1024, W>(p, c);
}

template <typename TX, typename TY>
cudaError_t run_types(const LnForward &p, const OpContext &c) {
  const bool vec = p.cols % 8 == 0 && rows_on(p.x, p.ldx, sizeof(TX), 16) && rows_on(p.y, p.ldy, sizeof(TY), 16) &&
                   (!p.ck.q || rows_on(p.ck.q, p.ck.ldq, 1, 8));
  if (p.cols > 16384 || (!vec && p.cols < 64)) {
    const int64_t most = (int64_t)c.sms * kAnyBlocks;
    return launch_ex(ln_forward_any_kernel<TX, TY>, dim3((unsigned)(p.rows < most ? p.rows : most)), dim3(kAnyThreads),
                     0, c.st, 1, p);
  }
  return vec ? run_width<TX, TY, 8>(p, c) : run_width<TX, TY, 1>(p, c);
}

}  // namespace

cudaError_t launch_ln_forward(const LnForward &p, const OpContext &c) {
  const bool xb = p.x_type == GEMM_TYPE_BF16, yb = p.y_type == GEMM_TYPE_BF16;
  if (xb) return yb ? run_types<bf16, bf16>(p, c) : run_types<bf16, float>(p, c);
  return yb ? run_types<float, bf16>(p, c) : run_types<float, float>(p, c);
}

}  // namespace gb300
