// layer_ln_fwd.cu -- layer norm forward, optionally with the result's 8-bit
// checkpoint.
#include <atomic>

#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kAnyThreads = 256;
constexpr int kMaxThreads = 512;

// Any width, pitch and alignment: a block per row, the row read three times
// (mean, variance, result), the second and third time from L1 or L2.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kAnyThreads) ln_forward_any_kernel(const LnForward p) {
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
    const float rstd = rsqrtf(block_sum2(v, 0.f, sm, 1).x * inv_n + p.eps);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[r] = mean;
      if (p.rstd) p.rstd[r] = rstd;
    }
    TY *y = static_cast<TY *>(p.y) + r * p.ldy;
    // each warp takes whole blocks of 32 columns, so that a checkpoint block
    // is the warp's 32 lanes
    for (int c0 = warp * 32; c0 < p.cols; c0 += kAnyThreads) {
      const int c = c0 + lane;
      float out = 0.f;
      if (c < p.cols) {
        out = fmaf((load_value<TX>(x, c) - mean) * rstd, load_param(p.gamma, p.param_type, c, 1.f),
                   load_param(p.beta, p.param_type, c, 0.f));
        store_value<TY>(y, c, out);
      }
      if (p.ck.q) {
        out = as_stored<TY>(out);
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(out) & 0x7FFFFFFFu);
        const uint32_t e = q8_exponent(top);
        if (c < p.cols) p.ck.q[r * p.ck.ldq + c] = (int8_t)q8_quantise(out, q8_inverse(e), e);
        if (lane == 0) p.ck.e[r * p.ck.lde + (c0 >> 5)] = (uint8_t)e;
      }
    }
  }
}


// A lane's 8 consecutive results (the first n of them), rounded to y's type
// and stored, and their part of the checkpoint of y as stored (four lanes hold
// a block).  All lanes of the warp call it.
template <typename TY>
__device__ __forceinline__ void store_eighth(TY *y, const Q8Ref &ck, int64_t r, int c, const float2 (&v)[4], int n) {
  float2 o[4];
  uint32_t top;
  if constexpr (sizeof(TY) == 2) {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = pack_bf16x2(v[j].x, v[j].y);
    if (n == 8) {
      *reinterpret_cast<uint4 *>(y + c) = make_uint4(h[0], h[1], h[2], h[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i < n)
          reinterpret_cast<uint16_t *>(y)[c + i] = (uint16_t)(h[i / 2] >> (16 * (i & 1)));
        else
          h[i / 2] &= (i & 1) ? 0x0000FFFFu : 0xFFFF0000u;  // not in the block
      }
    }
    if (!ck.q) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = make_float2(__uint_as_float(h[j] << 16), __uint_as_float(h[j] & 0xFFFF0000u));
    top = max_magnitude_bf16<4>(h);
  } else {
    float w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[2 * j] = v[j].x, w[2 * j + 1] = v[j].y;
    store_chunk<TY, 8>(y, c, w, n);
    if (!ck.q) return;
    top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[j] = make_float2(2 * j < n ? v[j].x : 0.f, 2 * j + 1 < n ? v[j].y : 0.f);
      top = max(top, max(__float_as_uint(o[j].x) & 0x7FFFFFFFu, __float_as_uint(o[j].y) & 0x7FFFFFFFu));
    }
  }
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t e = q8_exponent(top);
  const uint2 w = q8_pack8(o, e);
  int8_t *q = ck.q + r * ck.ldq + c;
  if (n == 8) {
    *reinterpret_cast<uint2 *>(q) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) q[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
  }
  if (n > 0 && (c & 31) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)e;
}

// Rows of up to 512 * NV * 8 values, kept in registers from their one read to
// their one write: a block of T threads walks rows gridDim.x apart, the next
// row's values on their way (as they are in memory) while this row is
// reduced, so that the loads never wait for the two block-wide sums.  gamma
// and beta stay in registers where they fit (NV <= 2).
//
// A thread holds NV * 8 / V chunks of V consecutive values, chunk k at column
// (k * T + t) * V: V = 8 where every row of x, y and q starts on 16 (q: 8)
// bytes, else V = 1, which any alignment allows and which still fills whole
// sectors, as the lanes of a warp are neighbours.  A checkpoint block is 4
// lanes' chunks (V = 8) or the warp's 32 lanes (V = 1).
template <typename TX, typename TY, int NV, int V>
__global__ void __launch_bounds__(kMaxThreads, NV == 1 ? 2 : 1) ln_forward_kernel(const LnForward p) {
  constexpr int C = NV * 8 / V;  // chunks per thread
  constexpr bool kKeep = NV <= 2;
  __shared__ float sm[2][32];
  griddep_launch_dependents();
  const int T = blockDim.x;
  int64_t r = blockIdx.x;
  const float inv_n = 1.0f / (float)p.cols;
  const auto col = [&](int k) { return (k * T + (int)threadIdx.x) * V; };
  // valid values of chunk k
  const auto valid = [&](int k) { return max(0, min(V, p.cols - col(k))); };
  const auto fetch = [&](Chunk<TX, V>(&raw)[C], int64_t row) {
    const TX *x = static_cast<const TX *>(p.x) + row * p.ldx;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int n = valid(k);
      if (n == V)
        raw[k].load(x, col(k));
      else
        raw[k].load_part(x, col(k), n);
    }
  };
  griddep_wait();
  Chunk<TX, V> raw[C];
  fetch(raw, r);
  float gamma[kKeep ? C * V : 1], beta[kKeep ? C * V : 1];
  if constexpr (kKeep) {
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = col(k) + i < p.cols;
        gamma[k * V + i] = in ? load_param(p.gamma, p.param_type, col(k) + i, 1.f) : 0.f;
        beta[k * V + i] = in ? load_param(p.beta, p.param_type, col(k) + i, 0.f) : 0.f;
      }
  }
  for (; r < p.rows; r += gridDim.x) {
    float x[C * V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k * V + i] = raw[k].get(i);
        s += x[k * V + i];  // zero past the row's end
      }
    if (r + gridDim.x < p.rows) fetch(raw, r + gridDim.x);
    const float mean = block_sum(s, sm[0]) * inv_n;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int n = valid(k);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k * V + i] -= mean;
        if (i < n) v = fmaf(x[k * V + i], x[k * V + i], v);
      }
    }
    const float rstd = rsqrtf(block_sum(v, sm[1]) * inv_n + p.eps);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[r] = mean;
      if (p.rstd) p.rstd[r] = rstd;
    }
    TY *y = static_cast<TY *>(p.y) + r * p.ldy;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int n = valid(k), c = col(k);
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float g = kKeep ? gamma[k * V + i] : i < n ? load_param(p.gamma, p.param_type, c + i, 1.f) : 0.f;
        const float b = kKeep ? beta[k * V + i] : i < n ? load_param(p.beta, p.param_type, c + i, 0.f) : 0.f;
        o[i] = fmaf(x[k * V + i] * rstd, g, b);
      }
      if constexpr (V == 8) {
        const float2 w[4] = {{o[0], o[1]}, {o[2], o[3]}, {o[4], o[5]}, {o[6], o[7]}};
        store_eighth<TY>(y, p.ck, r, c, w, n);
      } else {
        store_chunk<TY, V>(y, c, o, n);
        if (!p.ck.q) continue;
        o[0] = n > 0 ? as_stored<TY>(o[0]) : 0.f;
        const uint32_t e = q8_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(o[0]) & 0x7FFFFFFFu));
        if (n > 0) p.ck.q[r * p.ck.ldq + c] = (int8_t)q8_quantise(o[0], q8_inverse(e), e);
        if (n > 0 && (c & 31) == 0) p.ck.e[r * p.ck.lde + (c >> 5)] = (uint8_t)e;
      }
    }
  }
}

// Rows whose x is whole 16-byte pieces (and y's and q's rows aligned), up to
// 512 * NV * 8 values: as above, with the rows to come in a ring of slots that
// bulk copies fill, since one row ahead in registers is not enough in flight
// (3 blocks of 8 KB rows an SM: 24 KB, where the copy rate times the latency
// asks for 40).  The first of a row's two barriers frees its slot.
//
// THREADS bounds the block, and with it the registers so that 24 warps share
// an SM (32 with NV = 1, 16 with NV = 4).
template <typename TX, typename TY, int NV, int THREADS>
__global__ void __launch_bounds__(THREADS, NV == 1 ? 1024 / THREADS : NV == 2 && THREADS <= 256 ? 768 / THREADS : 1)
    ln_forward_ring_kernel(const LnForward p, const int stages, const uint32_t x_bytes, uint32_t *err,
                           const uint64_t wait_limit_ns) {
  constexpr bool kKeep = NV <= 2;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) float sm[2][16];
  __shared__ __align__(8) uint64_t bars[kMaxStages];
  __shared__ volatile uint32_t abort_flag;
  griddep_launch_dependents();
  const int T = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_addr(slots), bar0 = smem_addr(bars);
  RingPlace use, put;  // put: thread 0's
  const float inv_n = 1.0f / (float)p.cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 32) sm[threadIdx.x >> 4][threadIdx.x & 15] = 0.f;
  __syncthreads();
  griddep_wait();
  const int64_t mine = (p.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;  // rows of this block, at least one
  const auto row_of = [&](int64_t i) { return (int64_t)blockIdx.x + i * gridDim.x; };
  const auto fill = [&](int64_t i) {
    const uint32_t dst = ring + put.slot * x_bytes, bar = bar0 + 8u * put.slot;
    put.advance(stages);
    mbar_arrive_expect_tx(bar, x_bytes);
    bulk_load(dst, static_cast<const TX *>(p.x) + row_of(i) * p.ldx, x_bytes, bar);
  };
  int64_t filled = mine < stages ? mine : stages;
  if (threadIdx.x == 0)
    for (int64_t i = 0; i < filled; ++i) fill(i);
  const auto col = [&](int v) { return (v * T + (int)threadIdx.x) * 8; };
  const auto param = [&](const void *src, int c, float absent) {
    return make_float2(load_param(src, p.param_type, c, absent), load_param(src, p.param_type, c + 1, absent));
  };
  float2 gamma[kKeep ? NV * 4 : 1], beta[kKeep ? NV * 4 : 1];
  if constexpr (kKeep) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = col(v) < p.cols;
        gamma[v * 4 + j] = in ? param(p.gamma, col(v) + 2 * j, 1.f) : both(0.f);
        beta[v * 4 + j] = in ? param(p.beta, col(v) + 2 * j, 0.f) : both(0.f);
      }
  }
  bool ok = true;
  int64_t done = 0;
  for (int64_t i = 0; i < mine; done = ++i, use.advance(stages)) {
    const int64_t r = row_of(i);
    ok = mbar_wait(bar0 + 8u * use.slot, use.parity, &abort_flag, err, wait_limit_ns);
    float2 x[NV * 4], s2 = both(0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Chunk<TX, 8> raw;  // past the row's end: column 0, left out of the sums
      raw.load(slots + use.slot * x_bytes, col(v) < p.cols ? col(v) : 0);
      float2 t = both(0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[v * 4 + j] = raw.get2(j);
        t = add2(t, x[v * 4 + j]);
      }
      s2 = add2(s2, col(v) < p.cols ? t : both(0.f));
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
      float2 t = both(0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[v * 4 + j] = add2(x[v * 4 + j], both(-mean));
        t = fma2(x[v * 4 + j], x[v * 4 + j], t);
      }
      v2 = add2(v2, col(v) < p.cols ? t : both(0.f));
    }
    const float var = warp_sum(v2.x + v2.y);
    if (lane == 0) sm[1][warp] = var;
    __syncthreads();
    const float rstd = rsqrtf(sum_over_warps<THREADS / 32>(sm[1]) * inv_n + p.eps);
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[r] = mean;
      if (p.rstd) p.rstd[r] = rstd;
    }
    TY *y = static_cast<TY *>(p.y) + r * p.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = col(v);
      const bool in = c < p.cols;
      float2 o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 g = kKeep ? gamma[v * 4 + j] : in ? param(p.gamma, c + 2 * j, 1.f) : both(0.f);
        const float2 b = kKeep ? beta[v * 4 + j] : in ? param(p.beta, c + 2 * j, 0.f) : both(0.f);
        o[j] = fma2(mul2(x[v * 4 + j], both(rstd)), g, b);
      }
      store_eighth<TY>(y, p.ck, r, c, o, in ? 8 : 0);
    }
  }
  if (!ok && threadIdx.x == 0) ring_drain(bar0, stages, use, filled - done);
}

// Blocks of a kernel that an SM holds at once, asked once a kernel, block
// shape and shared memory size (the devices served are all the same).
template <typename K>
int blocks_per_sm(K kern, int threads, size_t smem, std::atomic<uint64_t> &known) {
  const uint64_t key = (uint64_t)smem << 16 | (uint64_t)threads << 8;
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

template <typename TX, typename TY, int NV, int V>
cudaError_t run_rows(const LnForward &p, int threads, const OpContext &c) {
  static std::atomic<uint64_t> known{0};
  const auto kern = ln_forward_kernel<TX, TY, NV, V>;
  return launch_ex(kern, dim3(persistent_grid(blocks_per_sm(kern, threads, 0, known), p.rows, c.sms)), dim3(threads), 0,
                   c.st, 1, p);
}

template <typename TX, typename TY, int NV, int THREADS>
cudaError_t run_ring(const LnForward &p, const OpContext &c) {
  static std::atomic<uint64_t> known{0};
  const auto kern = ln_forward_ring_kernel<TX, TY, NV, THREADS>;
  const int eights = (p.cols + 7) / 8, threads = ((eights + NV - 1) / NV + 31) / 32 * 32;
  const uint32_t x_bytes = (uint32_t)(p.cols * sizeof(TX));
  // the rings of the blocks that registers allow share the memory
  const int want = (NV == 1 ? 1024 : NV == 2 ? 768 : 512) / threads;
  int64_t stages = kRingBytes / (want < 8 ? want : 8) / x_bytes;
  stages = stages < 2 ? 2 : stages > kMaxStages ? kMaxStages : stages;
  const size_t smem = (size_t)stages * x_bytes;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(persistent_grid(blocks_per_sm(kern, threads, smem, known), p.rows, c.sms)), dim3(threads),
                   smem, c.st, 1, p, (int)stages, x_bytes, c.err, c.wait_limit_ns);
}

template <typename TX, typename TY>
cudaError_t run_types(const LnForward &p, const OpContext &c) {
  const int eights = (p.cols + 7) / 8;
  const bool vec = rows_on(p.x, p.ldx, sizeof(TX), 16) && rows_on(p.y, p.ldy, sizeof(TY), 16) &&
                   (!p.ck.q || rows_on(p.ck.q, p.ck.ldq, 1, 8));
  if (eights > 4 * kMaxThreads) {
    const int64_t most = (int64_t)c.sms * 8;
    return launch_ex(ln_forward_any_kernel<TX, TY>, dim3((unsigned)(p.rows < most ? p.rows : most)), dim3(kAnyThreads),
                     0, c.st, 1, p);
  }
  if (vec && p.cols % 8 == 0) {
    if (eights <= 128) return run_ring<TX, TY, 1, 128>(p, c);
    if (eights <= 512) return run_ring<TX, TY, 2, 256>(p, c);
    return eights <= 2 * kMaxThreads ? run_ring<TX, TY, 2, kMaxThreads>(p, c) : run_ring<TX, TY, 4, kMaxThreads>(p, c);
  }
  // values per thread: 8 for rows of up to 256 threads, else 16, else 32
  const int nv = eights <= 256 ? 1 : eights <= 2 * kMaxThreads ? 2 : 4;
  const int threads = ((eights + nv - 1) / nv + 31) / 32 * 32;
  if (nv == 1) return vec ? run_rows<TX, TY, 1, 8>(p, threads, c) : run_rows<TX, TY, 1, 1>(p, threads, c);
  if (nv == 2) return vec ? run_rows<TX, TY, 2, 8>(p, threads, c) : run_rows<TX, TY, 2, 1>(p, threads, c);
  return vec ? run_rows<TX, TY, 4, 8>(p, threads, c) : run_rows<TX, TY, 4, 1>(p, threads, c);
}

}  // namespace

cudaError_t launch_ln_forward(const LnForward &p, const OpContext &c) {
  const bool xb = p.x_type == GEMM_TYPE_BF16, yb = p.y_type == GEMM_TYPE_BF16;
  if (xb) return yb ? run_types<bf16, bf16>(p, c) : run_types<bf16, float>(p, c);
  return yb ? run_types<float, bf16>(p, c) : run_types<float, float>(p, c);
}

}  // namespace gb300
