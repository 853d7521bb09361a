// layer_ln_bwd.cu -- layer norm backward: dx, and the reduction of dgamma and
// dbeta over the rows.
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kRowThreads = 256;

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int grid_cap(int64_t want, int64_t cap) { return (int)(want < 1 ? 1 : (want > cap ? cap : want)); }

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

}  // namespace gb300
