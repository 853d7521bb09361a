// layer_ln_fwd.cu -- layer norm forward, optionally with the result's 8-bit
// checkpoint.
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
    const float rstd = 1.0f / sqrtf(block_sum2(v, 0.f, sm, 1).x * inv_n + p.eps);
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
__global__ void __launch_bounds__(kMaxThreads) ln_forward_kernel(const LnForward p) {
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
    const float rstd = 1.0f / sqrtf(block_sum(v, sm[1]) * inv_n + p.eps);
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
      store_chunk<TY, V>(y, c, o, n);
      if (p.ck.q) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          o[i] = i < n ? as_stored<TY>(o[i]) : 0.f;
          top = max(top, __float_as_uint(o[i]) & 0x7FFFFFFFu);
        }
        if constexpr (V == 1) {
          top = __reduce_max_sync(0xffffffffu, top);
        } else {
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        }
        const uint32_t e = q8_exponent(top);
        const float inverse = q8_inverse(e);
        int8_t *q = p.ck.q + r * p.ck.ldq + c;
        if constexpr (V == 8) {
          const uint32_t lo = q8_pack4(o, inverse, e), hi = q8_pack4(o + 4, inverse, e);
          if (n == V) {
            *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
          } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (i < n) q[i] = (int8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
          }
        } else if (n > 0) {
          q[0] = (int8_t)q8_quantise(o[0], inverse, e);
        }
        if (n > 0 && (c & 31) == 0) p.ck.e[r * p.ck.lde + (c >> 5)] = (uint8_t)e;
      }
    }
  }
}

// Whether rows of elements of `size` bytes at p, pitch ld, all start on a
// multiple of `align` bytes.
bool rows_on(const void *p, int64_t ld, int size, int align) {
  return (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0 && ld * size % align == 0;
}

// Blocks that fill the device once, no more than there are rows.
template <typename K>
unsigned persistent_grid(K kern, int threads, int64_t rows, int sms) {
  int per_sm = 0;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, 0) != cudaSuccess || per_sm < 1) per_sm = 1;
  const int64_t most = (int64_t)sms * per_sm;
  return (unsigned)(rows < most ? rows : most);
}

template <typename TX, typename TY, int NV, int V>
cudaError_t run_rows(const LnForward &p, int threads, int sms, cudaStream_t st) {
  const auto kern = ln_forward_kernel<TX, TY, NV, V>;
  return launch_ex(kern, dim3(persistent_grid(kern, threads, p.rows, sms)), dim3(threads), 0, st, 1, p);
}

template <typename TX, typename TY>
cudaError_t run_types(const LnForward &p, int sms, cudaStream_t st) {
  const int eights = (p.cols + 7) / 8;
  const bool vec = rows_on(p.x, p.ldx, sizeof(TX), 16) && rows_on(p.y, p.ldy, sizeof(TY), 16) &&
                   (!p.ck.q || rows_on(p.ck.q, p.ck.ldq, 1, 8));
  // values per thread: 8 for rows of up to 256 threads, else 16, else 32
  const int nv = eights <= 256 ? 1 : eights <= 2 * kMaxThreads ? 2 : 4;
  if (eights > nv * kMaxThreads) {
    const int64_t most = (int64_t)sms * 8;
    return launch_ex(ln_forward_any_kernel<TX, TY>, dim3((unsigned)(p.rows < most ? p.rows : most)), dim3(kAnyThreads),
                     0, st, 1, p);
  }
  const int threads = ((eights + nv - 1) / nv + 31) / 32 * 32;
  if (nv == 1) return vec ? run_rows<TX, TY, 1, 8>(p, threads, sms, st) : run_rows<TX, TY, 1, 1>(p, threads, sms, st);
  if (nv == 2) return vec ? run_rows<TX, TY, 2, 8>(p, threads, sms, st) : run_rows<TX, TY, 2, 1>(p, threads, sms, st);
  return vec ? run_rows<TX, TY, 4, 8>(p, threads, sms, st) : run_rows<TX, TY, 4, 1>(p, threads, sms, st);
}

}  // namespace

cudaError_t launch_ln_forward(const LnForward &p, int sms, cudaStream_t st) {
  const bool xb = p.x_type == GEMM_TYPE_BF16, yb = p.y_type == GEMM_TYPE_BF16;
  if (xb) return yb ? run_types<bf16, bf16>(p, sms, st) : run_types<bf16, float>(p, sms, st);
  return yb ? run_types<float, bf16>(p, sms, st) : run_types<float, float>(p, sms, st);
}

}  // namespace gb300
