// layer_rows.cu -- the layer operators that walk a matrix by rows: layer norm
// forward and backward, and the 8-bit checkpoint's save and restore.
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kRowThreads = 256;

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int grid_cap(int64_t want, int64_t cap) { return (int)(want < 1 ? 1 : (want > cap ? cap : want)); }

// ------------------------------------------------------- layer norm forward

// Any width, pitch and alignment: a block per row, the row read three times
// (mean, variance, result), the second and third time from L1 or L2.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kRowThreads) ln_forward_any_kernel(const LnForward p) {
  __shared__ float2 sm[2][32];
  griddep_launch_dependents();
  griddep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float inv_n = 1.0f / (float)p.cols;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const TX *x = static_cast<const TX *>(p.x) + r * p.ldx;
    float s = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kRowThreads) s += load_value<TX>(x, c);
    const float mean = block_sum2(s, 0.f, sm, 0).x * inv_n;
    float v = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kRowThreads) {
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
    for (int c0 = warp * 32; c0 < p.cols; c0 += kRowThreads) {
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

// ------------------------------------------------------ layer norm backward

// Value c of row r of the forward pass's input: of type TX, or (Q8) held in
// the checkpoint.
template <typename TX>
__device__ __forceinline__ float ln_input(const LnBackward &p, int64_t r, int c) {
  if constexpr (sizeof(TX) == 1)
    return (float)p.ck.q[r * p.ck.ldq + c] * q8_scale(p.ck.e[r * p.ck.lde + (c >> 5)]);
  else
    return load_value<TX>(p.x, r * p.ldx + c);
}

// Any width, pitch and alignment: dx, a block per row, the row's x and dy
// read twice (the two averages, then dx).
template <typename TX, typename TDY, typename TDX>
__global__ void __launch_bounds__(kRowThreads) ln_backward_any_kernel(const LnBackward p) {
  __shared__ float2 sm[2][32];
  griddep_launch_dependents();
  griddep_wait();
  const float inv_n = 1.0f / (float)p.cols;
  int buf = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float mean = p.mean[r], rstd = p.rstd[r];
    const TDY *dy = static_cast<const TDY *>(p.dy) + r * p.lddy;
    float a = 0.f, b = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kRowThreads) {
      const float xh = (ln_input<TX>(p, r, c) - mean) * rstd;
      const float g = load_value<TDY>(dy, c) * load_param(p.gamma, p.param_type, c, 1.f);
      a += g;
      b = fmaf(g, xh, b);
    }
    const float2 s = block_sum2(a, b, sm, buf);
    buf ^= 1;
    const float ga = s.x * inv_n, gx = s.y * inv_n;
    TDX *dx = static_cast<TDX *>(p.dx) + r * p.lddx;
    for (int c = threadIdx.x; c < p.cols; c += kRowThreads) {
      const float xh = (ln_input<TX>(p, r, c) - mean) * rstd;
      const float g = load_value<TDY>(dy, c) * load_param(p.gamma, p.param_type, c, 1.f);
      store_value<TDX>(dx, c, rstd * (g - ga - xh * gx));
    }
  }
}

// Partial dgamma and dbeta of a strip of 32 columns over every gridDim.y-th
// group of 8 rows: thread (i, j) walks column i of rows j, j + 8 gridDim.y,
// ...; the eight partial sums are added in order.  Partials: gridDim.y rows
// of dgamma, then as many of dbeta, cols floats each.
template <typename TX, typename TDY>
__global__ void __launch_bounds__(kRowThreads) ln_param_partials_kernel(const LnBackward p) {
  __shared__ float2 sm[8][32];
  griddep_launch_dependents();
  griddep_wait();
  const int i = threadIdx.x & 31, j = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + i;
  float dg = 0.f, db = 0.f;
  if (c < p.cols) {
    for (int64_t r = (int64_t)blockIdx.y * 8 + j; r < p.rows; r += (int64_t)gridDim.y * 8) {
      const float d = load_value<TDY>(p.dy, r * p.lddy + c);
      dg = fmaf(d, (ln_input<TX>(p, r, (int)c) - p.mean[r]) * p.rstd[r], dg);
      db += d;
    }
  }
  sm[j][i] = make_float2(dg, db);
  __syncthreads();
  if (j == 0 && c < p.cols) {
#pragma unroll
    for (int k = 1; k < 8; ++k) {
      dg += sm[k][i].x;
      db += sm[k][i].y;
    }
    p.partials[(int64_t)blockIdx.y * p.cols + c] = dg;
    p.partials[(int64_t)(gridDim.y + blockIdx.y) * p.cols + c] = db;
  }
}

// dgamma (blockIdx.y 0) or dbeta (1): `parts` rows of partials summed.  A
// block takes 32 columns; its 32 warps each add every 32nd row, and the 32
// sums are added in order.
__global__ void __launch_bounds__(1024) ln_param_sum_kernel(const float *partials, int parts, int cols, float *dgamma,
                                                            float *dbeta) {
  __shared__ float sm[32][33];
  griddep_launch_dependents();
  griddep_wait();
  float *out = blockIdx.y == 0 ? dgamma : dbeta;
  if (!out) return;
  const int i = threadIdx.x & 31, j = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + i;
  const float *src = partials + (int64_t)blockIdx.y * parts * cols + c;
  float s = 0.f;
  if (c < cols)
    for (int k = j; k < parts; k += 32) s += src[(int64_t)k * cols];
  sm[j][i] = s;
  __syncthreads();
  // warp j adds up column j: the 32 sums are added pairwise, in an order the
  // lane numbers fix
  const float t = warp_sum(sm[i][j]);
  const int64_t cj = (int64_t)blockIdx.x * 32 + j;
  if (i == 0 && cj < cols) out[cj] = t;
}

// ------------------------------------------------------------- checkpoints

// Any width, pitch and alignment: a warp per block of 32 values.
template <typename TX>
__global__ void __launch_bounds__(kRowThreads)
    q8_save_any_kernel(const void *x, int64_t ldx, int64_t rows, int64_t cols, Q8Ref ck) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t blocks = (cols + 31) / 32, items = rows * blocks;
  const int64_t step = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t t = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5); t < items; t += step) {
    const int64_t r = t / blocks, b = t - r * blocks, c = b * 32 + lane;
    const float v = c < cols ? load_value<TX>(x, r * ldx + c) : 0.f;
    const uint32_t e = q8_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7FFFFFFFu));
    if (c < cols) ck.q[r * ck.ldq + c] = (int8_t)q8_quantise(v, q8_inverse(e), e);
    if (lane == 0) ck.e[r * ck.lde + b] = (uint8_t)e;
  }
}

template <typename TX>
__global__ void __launch_bounds__(kRowThreads)
    q8_restore_any_kernel(Q8Ref ck, void *x, int64_t ldx, int64_t rows, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t blocks = (cols + 31) / 32, items = rows * blocks;
  const int64_t step = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t t = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5); t < items; t += step) {
    const int64_t r = t / blocks, b = t - r * blocks, c = b * 32 + lane;
    if (c < cols) store_value<TX>(x, r * ldx + c, (float)ck.q[r * ck.ldq + c] * q8_scale(ck.e[r * ck.lde + b]));
  }
}

template <typename TX, typename TDY, typename TDX>
cudaError_t ln_backward_any(const LnBackward &p, int sms, cudaStream_t st, int *launches) {
  cudaError_t e = cudaSuccess;
  if (p.rows > 0) {
    e = launch_ex(ln_backward_any_kernel<TX, TDY, TDX>, dim3(grid_cap(p.rows, (int64_t)sms * 8)), dim3(kRowThreads), 0,
                  st, 1, p);
    ++*launches;
    if (e != cudaSuccess) return e;
  }
  if (!p.dgamma && !p.dbeta) return e;
  const int strips = (int)ceil_div64(p.cols, 32);
  const int parts = (int)(ln_backward_partials(p, sms) / 2 / p.cols);
  e = launch_ex(ln_param_partials_kernel<TX, TDY>, dim3(strips, parts), dim3(kRowThreads), 0, st, 1, p);
  ++*launches;
  if (e != cudaSuccess) return e;
  e = launch_ex(ln_param_sum_kernel, dim3(strips, 2), dim3(1024), 0, st, 1, (const float *)p.partials, parts, p.cols,
                p.dgamma, p.dbeta);
  ++*launches;
  return e;
}

}  // namespace

cudaError_t launch_ln_forward(const LnForward &p, int sms, cudaStream_t st) {
  const dim3 grid(grid_cap(p.rows, (int64_t)sms * 8)), block(kRowThreads);
  const bool xb = p.x_type == GEMM_TYPE_BF16, yb = p.y_type == GEMM_TYPE_BF16;
  if (xb && yb) return launch_ex(ln_forward_any_kernel<bf16, bf16>, grid, block, 0, st, 1, p);
  if (xb) return launch_ex(ln_forward_any_kernel<bf16, float>, grid, block, 0, st, 1, p);
  if (yb) return launch_ex(ln_forward_any_kernel<float, bf16>, grid, block, 0, st, 1, p);
  return launch_ex(ln_forward_any_kernel<float, float>, grid, block, 0, st, 1, p);
}

// Rows of partial sums: enough blocks of 32 columns x 8 rows at a time to
// fill the device several times over, no more than there are groups of rows.
size_t ln_backward_partials(const LnBackward &p, int sms) {
  const int64_t strips = ceil_div64(p.cols, 32);
  const int64_t parts = grid_cap(ceil_div64((int64_t)sms * 16, strips), ceil_div64(p.rows < 1 ? 1 : p.rows, 8));
  return (size_t)(2 * parts * p.cols);
}

cudaError_t launch_ln_backward(const LnBackward &p, int sms, cudaStream_t st, int *launches) {
  const bool gb = p.dy_type == GEMM_TYPE_BF16, ob = p.dx_type == GEMM_TYPE_BF16;
  if (!p.x) {
    if (ob) return gb ? ln_backward_any<Q8, bf16, bf16>(p, sms, st, launches) : ln_backward_any<Q8, float, bf16>(p, sms, st, launches);
    return gb ? ln_backward_any<Q8, bf16, float>(p, sms, st, launches) : ln_backward_any<Q8, float, float>(p, sms, st, launches);
  }
  if (ob) return gb ? ln_backward_any<bf16, bf16, bf16>(p, sms, st, launches) : ln_backward_any<bf16, float, bf16>(p, sms, st, launches);
  return gb ? ln_backward_any<float, bf16, float>(p, sms, st, launches) : ln_backward_any<float, float, float>(p, sms, st, launches);
}

cudaError_t launch_q8_save(const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols, const Q8Ref &ck,
                           cudaStream_t st) {
  const int64_t items = rows * ceil_div64(cols, 32);
  const dim3 grid(grid_cap(ceil_div64(items, kRowThreads / 32), 1 << 20)), block(kRowThreads);
  return x_type == GEMM_TYPE_BF16 ? launch_ex(q8_save_any_kernel<bf16>, grid, block, 0, st, 1, x, ldx, rows, cols, ck)
                                  : launch_ex(q8_save_any_kernel<float>, grid, block, 0, st, 1, x, ldx, rows, cols, ck);
}

cudaError_t launch_q8_restore(const Q8Ref &ck, void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols,
                              cudaStream_t st) {
  const int64_t items = rows * ceil_div64(cols, 32);
  const dim3 grid(grid_cap(ceil_div64(items, kRowThreads / 32), 1 << 20)), block(kRowThreads);
  return x_type == GEMM_TYPE_BF16
             ? launch_ex(q8_restore_any_kernel<bf16>, grid, block, 0, st, 1, ck, x, ldx, rows, cols)
             : launch_ex(q8_restore_any_kernel<float>, grid, block, 0, st, 1, ck, x, ldx, rows, cols);
}

}  // namespace gb300
