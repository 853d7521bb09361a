// layer_ln_bwd.cu -- layer norm backward: dx, and the reduction of dgamma and
// dbeta over the rows.
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRingThreads = 512;     // most threads a block of the register-resident kernels has
// Threads of the ring kernel with NV eights of values each.
__host__ __device__ constexpr int ring_threads(int nv) { return nv == 1 ? 128 : kRingThreads; }

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

// Row r's mean and 1/std as the factors of xh = x * rstd - mean * rstd.
struct RowStats {
  float rstd, shift;
  __device__ __forceinline__ explicit RowStats(float2 mean_rstd)
      : rstd(mean_rstd.y), shift(-mean_rstd.x * mean_rstd.y) {}
};

// Rows whose x and dy are whole 16-byte pieces, up to 512 * NV * 8 values.
// A block walks rows gridDim.x apart.  Their x and dy come through a ring of
// row slots in shared memory, filled by bulk copies that run as far ahead as
// the ring is deep: dgamma and dbeta are summed in registers (16 values a
// thread and NV), which leaves none for rows in flight.  A row is read from
// its slot twice, for the two averages and for the results; the block-wide
// barrier between, passed by every thread once it has finished with the row
// before, also frees that row's slot, which thread 0 refills.  One partial
// row of dgamma and of dbeta a block goes to the workspace.
template <typename TX, typename TDY, typename TDX, int NV>
__global__ void __launch_bounds__(ring_threads(NV), NV == 1 ? 8 : 1)
    ln_backward_ring_kernel(const LnBackward p, const int stages, const uint32_t x_bytes, const uint32_t dy_bytes,
                            uint32_t *err, const uint64_t wait_limit_ns) {
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) float2 sm[2][16];
  __shared__ __align__(8) uint64_t bars[kMaxStages];
  __shared__ volatile uint32_t abort_flag;
  griddep_launch_dependents();
  const int T = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_addr(slots), bar0 = smem_addr(bars), slot_bytes = x_bytes + dy_bytes;
  RingPlace use, put;  // put: thread 0's
  const float inv_n = 1.0f / (float)p.cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 32) sm[threadIdx.x >> 4][threadIdx.x & 15] = make_float2(0.f, 0.f);
  __syncthreads();
  griddep_wait();
  const int64_t mine = (p.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;  // rows of this block, at least one
  const auto row_of = [&](int64_t i) { return (int64_t)blockIdx.x + i * gridDim.x; };
  const auto fill = [&](int64_t i) {
    const uint32_t dst = ring + put.slot * slot_bytes, bar = bar0 + 8u * put.slot;
    const int64_t r = row_of(i);
    put.advance(stages);
    mbar_arrive_expect_tx(bar, slot_bytes);
    if constexpr (sizeof(TX) == 1)
      bulk_load(dst, p.ck.q + r * p.ck.ldq, x_bytes, bar);
    else
      bulk_load(dst, static_cast<const TX *>(p.x) + r * p.ldx, x_bytes, bar);
    bulk_load(dst + x_bytes, static_cast<const TDY *>(p.dy) + r * p.lddy, dy_bytes, bar);
  };
  int64_t filled = mine < stages ? mine : stages;
  if (threadIdx.x == 0)
    for (int64_t i = 0; i < filled; ++i) fill(i);

  // the row's statistics and block exponents, fetched a row ahead
  float2 st_next;
  uint32_t ex[NV], ex_next[NV];
  const auto fetch = [&](int64_t i) {
    const int64_t r = row_of(i);
    st_next = make_float2(p.mean[r], p.rstd[r]);
    if constexpr (sizeof(TX) == 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * T + (int)threadIdx.x) * 8;
        ex_next[v] = c < p.cols ? p.ck.e[r * p.ck.lde + (c >> 5)] : 0;
      }
    }
  };
  fetch(0);
  float2 gamma[NV * 4], dg[NV * 4], db[NV * 4];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * T + (int)threadIdx.x) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      gamma[v * 4 + i] = c < p.cols ? make_float2(load_param(p.gamma, p.param_type, c + 2 * i, 1.f),
                                                  load_param(p.gamma, p.param_type, c + 2 * i + 1, 1.f))
                                    : both(0.f);
      dg[v * 4 + i] = db[v * 4 + i] = both(0.f);
    }
  }
  bool ok = true;
  int64_t done = 0;
  for (int64_t i = 0; i < mine; done = ++i, use.advance(stages)) {
    const uint8_t *slot = slots + use.slot * slot_bytes;
    const RowStats st(st_next);
#pragma unroll
    for (int v = 0; v < NV; ++v) ex[v] = ex_next[v];
    if (i + 1 < mine) fetch(i + 1);
    ok = mbar_wait(bar0 + 8u * use.slot, use.parity, &abort_flag, err, wait_limit_ns);
    const auto load = [&](int v, Chunk<TX, 8> &x, Chunk<TDY, 8> &y, float2 &scale) {
      const int c = (v * T + (int)threadIdx.x) * 8;
      x.load(slot, c);
      y.load(slot + x_bytes, c);
      if constexpr (sizeof(TX) == 1)
        scale = both(st.rstd * q8_scale(ex[v]));
      else
        scale = both(st.rstd);
    };
    const float2 shift = both(st.shift);
    float2 a2 = both(0.f), b2 = both(0.f);
    if (ok) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if ((v * T + (int)threadIdx.x) * 8 < p.cols) {
          Chunk<TX, 8> x;
          Chunk<TDY, 8> y;
          float2 scale;
          load(v, x, y, scale);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 g = mul2(y.get2(j), gamma[v * 4 + j]);
            a2 = add2(a2, g);
            b2 = fma2(g, fma2(x.get2(j), scale, shift), b2);
          }
        }
      }
    }
    const float a = warp_sum(a2.x + a2.y), b = warp_sum(b2.x + b2.y);
    if (lane == 0) sm[i & 1][warp] = make_float2(a, b);
    // every wait of the block succeeded, or the block gives up together
    if (!__syncthreads_and(ok)) {
      ok = false;
      break;
    }
    if (threadIdx.x == 0 && i > 0 && filled < mine) fill(filled++);  // the slot of row i - 1
    const float2 s = sum_over_warps<ring_threads(NV) / 32>(sm[i & 1]);
    const float2 ga = both(-s.x * inv_n * st.rstd), gx = both(-s.y * inv_n * st.rstd), rstd = both(st.rstd);
    TDX *dx = static_cast<TDX *>(p.dx) + row_of(i) * p.lddx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * T + (int)threadIdx.x) * 8;
      if (c < p.cols) {
        Chunk<TX, 8> x;
        Chunk<TDY, 8> y;
        float2 scale;
        load(v, x, y, scale);
        float o[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 d = y.get2(j), xh = fma2(x.get2(j), scale, shift);
          dg[v * 4 + j] = fma2(d, xh, dg[v * 4 + j]);
          db[v * 4 + j] = add2(db[v * 4 + j], d);
          const float2 r = fma2(mul2(d, gamma[v * 4 + j]), rstd, fma2(xh, gx, ga));
          o[2 * j] = r.x;
          o[2 * j + 1] = r.y;
        }
        store_chunk<TDX, 8>(dx, c, o, 8);
      }
    }
  }
  if (!ok) {
    if (threadIdx.x == 0) ring_drain(bar0, stages, use, filled - done);
    return;
  }
  if (!p.partials) return;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * T + (int)threadIdx.x) * 8;
    if (c < p.cols) {
      store_chunk<float, 8>(p.partials + (int64_t)blockIdx.x * p.cols, c, reinterpret_cast<const float *>(dg + v * 4), 8);
      store_chunk<float, 8>(p.partials + (int64_t)(gridDim.x + blockIdx.x) * p.cols, c,
                            reinterpret_cast<const float *>(db + v * 4), 8);
    }
  }
}

// Any alignment, up to 512 * NV * 8 values a row: x and dy are read straight
// into registers, in chunks of V values (V = 4 where the rows of every matrix
// start on a multiple of four values, else 1: neighbouring lanes still share
// sectors), and kept there between the two averages and the results.
template <typename TX, typename TDY, typename TDX, int NV, int V>
__global__ void __launch_bounds__(kRingThreads) ln_backward_regs_kernel(const LnBackward p) {
  constexpr int C = NV * 8 / V;
  __shared__ float2 sm[2][32];
  griddep_launch_dependents();
  griddep_wait();
  const int T = blockDim.x;
  const float inv_n = 1.0f / (float)p.cols;
  const auto col = [&](int k) { return (k * T + (int)threadIdx.x) * V; };
  const auto valid = [&](int k) { return max(0, min(V, p.cols - col(k))); };
  float gamma[C * V], dg[C * V], db[C * V];
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      gamma[k * V + i] = i < valid(k) ? load_param(p.gamma, p.param_type, col(k) + i, 1.f) : 0.f;
      dg[k * V + i] = db[k * V + i] = 0.f;
    }
  int buf = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const RowStats st(make_float2(p.mean[r], p.rstd[r]));
    Chunk<TX, V> x[C];
    Chunk<TDY, V> y[C];
    uint32_t ex[C];
    const void *xr;
    if constexpr (sizeof(TX) == 1)
      xr = p.ck.q + r * p.ck.ldq;
    else
      xr = static_cast<const TX *>(p.x) + r * p.ldx;
    const TDY *yr = static_cast<const TDY *>(p.dy) + r * p.lddy;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int n = valid(k), c = col(k);
      if (n == V) {
        x[k].load(xr, c);
        y[k].load(yr, c);
      } else {
        x[k].load_part(xr, c, n);
        y[k].load_part(yr, c, n);
      }
      if constexpr (sizeof(TX) == 1) ex[k] = n > 0 ? p.ck.e[r * p.ck.lde + (c >> 5)] : 0;
    }
    float a = 0.f, b = 0.f;
    const auto xhat = [&](int k, int i) {
      float scale = st.rstd;
      if constexpr (sizeof(TX) == 1) scale *= q8_scale(ex[k]);
      return fmaf(x[k].get(i), scale, st.shift);
    };
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (i < valid(k)) {
          const float g = y[k].get(i) * gamma[k * V + i];
          a += g;
          b = fmaf(g, xhat(k, i), b);
        }
      }
    const float2 s = block_sum2(a, b, sm, buf);
    buf ^= 1;
    const float ga = s.x * inv_n * st.rstd, gx = s.y * inv_n * st.rstd;
    TDX *dx = static_cast<TDX *>(p.dx) + r * p.lddx;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int n = valid(k);
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = y[k].get(i), xh = xhat(k, i);
        if (i < n) {
          dg[k * V + i] = fmaf(d, xh, dg[k * V + i]);
          db[k * V + i] += d;
        }
        o[i] = fmaf(d * gamma[k * V + i], st.rstd, -fmaf(xh, gx, ga));
      }
      store_chunk<TDX, V>(dx, col(k), o, n);
    }
  }
  if (!p.partials) return;
#pragma unroll
  for (int k = 0; k < C; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < valid(k)) {
        p.partials[(int64_t)blockIdx.x * p.cols + col(k) + i] = dg[k * V + i];
        p.partials[(int64_t)(gridDim.x + blockIdx.x) * p.cols + col(k) + i] = db[k * V + i];
      }
}

// How a backward pass runs.
enum LnPath { kLnAny, kLnRegs, kLnRing };
struct LnPlan {
  LnPath path;
  int nv, threads, grid;
  int chunk;                    // kLnRegs: V
  int stages;                   // kLnRing
  uint32_t x_bytes, dy_bytes;   // kLnRing: bytes of a row
  int parts;                    // partial rows of the parameter gradients
};

// Blocks that walk `rows` rows, `per_sm` at a time on an SM: every SM one
// while there are few rows, more only where each has at least eight rows to
// set against the partial row that it writes and another kernel reads.
int row_blocks(int64_t rows, int sms, int per_sm) {
  const int64_t few = rows < sms ? rows : sms, many = ceil_div64(rows, 8), most = (int64_t)sms * per_sm;
  const int64_t want = many > few ? many : few;
  return (int)(want < most ? want : most);
}

LnPlan plan_ln_backward(const LnBackward &p, int sms) {
  LnPlan l{};
  const int sx = !p.x ? 1 : p.x_type == GEMM_TYPE_BF16 ? 2 : 4, sg = p.dy_type == GEMM_TYPE_BF16 ? 2 : 4,
            so = p.dx_type == GEMM_TYPE_BF16 ? 2 : 4;
  const void *x = p.x ? p.x : (const void *)p.ck.q;
  const int64_t ldx = p.x ? p.ldx : p.ck.ldq;
  const int64_t eights = ceil_div64(p.cols, 8);
  // few threads with more values each: a row's fixed costs (its barrier, the
  // sums over lanes and warps) are paid by every warp
  const int ring_nv = eights <= ring_threads(1) ? 1 : eights <= 2 * kRingThreads ? 2 : (int)ceil_div64(eights, kRingThreads);
  const bool pieces = (int64_t)p.cols * sx % 16 == 0 && (int64_t)p.cols * sg % 16 == 0 && p.cols % 8 == 0;
  if (p.rows > 0 && ring_nv <= 4 && pieces && rows_on(x, ldx, sx, 16) && rows_on(p.dy, p.lddy, sg, 16) &&
      rows_on(p.dx, p.lddx, so, 16)) {
    l.x_bytes = (uint32_t)p.cols * sx;
    l.dy_bytes = (uint32_t)p.cols * sg;
    l.nv = ring_nv;
    l.threads = (int)ceil_div64(ceil_div64(eights, l.nv), 32) * 32;
    int per_sm = (l.nv == 1 ? 2 : 1) * (kRingThreads / l.threads);
    per_sm = per_sm > 8 ? 8 : per_sm;
    int64_t stages = kRingBytes / per_sm / (l.x_bytes + l.dy_bytes);
    if (stages < 2) {
      per_sm = 1;
      stages = kRingBytes / (l.x_bytes + l.dy_bytes);
    }
    if (stages >= 2) {
      l.path = kLnRing;
      l.stages = (int)(stages < kMaxStages ? stages : kMaxStages);
      l.grid = l.parts = row_blocks(p.rows, sms, per_sm);
      return l;
    }
  }
  if (p.rows > 0 && eights <= 2 * kRingThreads) {
    l.path = kLnRegs;
    l.nv = (int)ceil_div64(eights, kRingThreads);
    l.threads = (int)ceil_div64(ceil_div64(eights, l.nv), 32) * 32;
    l.chunk = rows_on(x, ldx, sx, 4 * sx) && rows_on(p.dy, p.lddy, sg, 4 * sg) && rows_on(p.dx, p.lddx, so, 4 * so) ? 4 : 1;
    const int per_sm = kRingThreads / l.threads;
    l.grid = l.parts = row_blocks(p.rows, sms, per_sm > 4 ? 4 : per_sm);
    return l;
  }
  // dx by one kernel, partials by another: enough blocks of 32 columns x 8
  // rows at a time to fill the device several times over, no more than there
  // are groups of rows
  l.path = kLnAny;
  l.grid = grid_cap(p.rows, (int64_t)sms * 8);
  l.parts = grid_cap(ceil_div64((int64_t)sms * 16, ceil_div64(p.cols, 32)), ceil_div64(p.rows < 1 ? 1 : p.rows, 8));
  return l;
}

template <typename TX, typename TDY, typename TDX, int NV>
cudaError_t run_ring(const LnBackward &p, const LnPlan &l, const OpContext &c) {
  const auto kern = ln_backward_ring_kernel<TX, TDY, TDX, NV>;
  const size_t smem = (size_t)l.stages * (l.x_bytes + l.dy_bytes);
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(l.grid), dim3(l.threads), smem, c.st, 1, p, l.stages, l.x_bytes, l.dy_bytes, c.err,
                   c.wait_limit_ns);
}

template <typename TX, typename TDY, typename TDX>
cudaError_t run_types(const LnBackward &p, const OpContext &c, int *launches) {
  const LnPlan l = plan_ln_backward(p, c.sms);
  const dim3 grid(l.grid), block(l.threads);
  cudaError_t e = cudaSuccess;
  if (p.rows > 0) {
    ++*launches;
    if (l.path == kLnRing)
      e = l.nv == 1   ? run_ring<TX, TDY, TDX, 1>(p, l, c)
          : l.nv == 2 ? run_ring<TX, TDY, TDX, 2>(p, l, c)
          : l.nv == 3 ? run_ring<TX, TDY, TDX, 3>(p, l, c)
                      : run_ring<TX, TDY, TDX, 4>(p, l, c);
    else if (l.path == kLnRegs && l.nv == 1)
      e = l.chunk == 4 ? launch_ex(ln_backward_regs_kernel<TX, TDY, TDX, 1, 4>, grid, block, 0, c.st, 1, p)
                       : launch_ex(ln_backward_regs_kernel<TX, TDY, TDX, 1, 1>, grid, block, 0, c.st, 1, p);
    else if (l.path == kLnRegs)
      e = l.chunk == 4 ? launch_ex(ln_backward_regs_kernel<TX, TDY, TDX, 2, 4>, grid, block, 0, c.st, 1, p)
                       : launch_ex(ln_backward_regs_kernel<TX, TDY, TDX, 2, 1>, grid, block, 0, c.st, 1, p);
    else
      e = launch_ex(ln_backward_any_kernel<TX, TDY, TDX>, grid, dim3(kRowThreads), 0, c.st, 1, p);
    if (e != cudaSuccess) return e;
  }
  if (!p.partials) return e;
  const int strips = (int)ceil_div64(p.cols, 32);
  if (l.path == kLnAny) {
    ++*launches;
    e = launch_ex(ln_param_partials_kernel<TX, TDY>, dim3(strips, l.parts), dim3(kRowThreads), 0, c.st, 1, p);
    if (e != cudaSuccess) return e;
  }
  ++*launches;
  return launch_ex(ln_param_sum_kernel, dim3(strips, 2), dim3(1024), 0, c.st, 1, (const float *)p.partials, l.parts,
                   p.cols, p.dgamma, p.dbeta);
}

}  // namespace

size_t ln_backward_partials(const LnBackward &p, int sms) {
  return p.dgamma || p.dbeta ? (size_t)2 * plan_ln_backward(p, sms).parts * p.cols : 0;
}

cudaError_t launch_ln_backward(const LnBackward &p, const OpContext &c, int *launches) {
  const bool gb = p.dy_type == GEMM_TYPE_BF16, ob = p.dx_type == GEMM_TYPE_BF16;
  if (!p.x) {
    if (ob) return gb ? run_types<Q8, bf16, bf16>(p, c, launches) : run_types<Q8, float, bf16>(p, c, launches);
    return gb ? run_types<Q8, bf16, float>(p, c, launches) : run_types<Q8, float, float>(p, c, launches);
  }
  if (ob) return gb ? run_types<bf16, bf16, bf16>(p, c, launches) : run_types<bf16, float, bf16>(p, c, launches);
  return gb ? run_types<float, bf16, float>(p, c, launches) : run_types<float, float, float>(p, c, launches);
}

}  // namespace gb300
