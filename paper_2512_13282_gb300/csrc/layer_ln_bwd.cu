// layer_ln_bwd.cu -- layer norm backward: with xh = (x - mean) * rstd and
// g = dy * gamma, by rows
//     dx = rstd * (g - avg(g) - xh * avg(g * xh)),
// and over the rows dgamma = sum(dy * xh), dbeta = sum(dy).  Sums are float32,
// in an order that the sizes fix: no atomics.  xh is the rounded difference
// x - mean times rstd, two roundings relative to xh itself (x * rstd - mean *
// rstd would carry one relative to mean * rstd, the same for a whole row); a
// checkpoint's byte is scaled and the mean subtracted in one operation, the
// product with a power of two being exact.
//
// HBM bounds it: x and dy read once and dx written once, 6 bytes a value in
// bf16.  Measured, back to back, bf16: 8192 x 12288 98 us (6.2 TB/s, 0.91 of
// the copy rate), 8192 x 4096 40 us (5.0 TB/s), 2048 x 4096 19 us (a row's
// latency times seven rows a block, and the second launch), 65536 x 512 47 us.
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRingThreads = 512;     // most threads a block of the register-resident kernels has
// Rows that the ring kernel takes at a time, between two barriers, where the
// ring has slots for twice as many: two where registers allow.
__host__ __device__ constexpr int most_rows(int nv, int v) { return v == 8 && nv <= 2 ? 2 : 1; }

// Floats from one partial row to the next: whole strips of 32 columns.
__host__ __device__ constexpr int partial_pitch(int cols) { return (cols + 31) / 32 * 32; }

// Blocks of the ring kernel that its registers are to leave room for: 1024
// threads an SM with 8 values each (768 at any alignment), else 512, or 384
// with 32 values each.
__host__ __device__ constexpr int ring_blocks(int nv, int v, int threads) {
  return (nv == 4 && threads <= 128 ? 384 : nv > 1 ? 512 : v == 8 ? 1024 : 768) / threads;
}

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
// read twice (the two averages, then dx).  For what the ring kernel does not
// take: rows above 16384 values, or above 12800 of float32 x and dy, of which
// two do not fit in its ring (4096 x 12800 146 us, 4096 x 16384 429), and
// unaligned ones below 64.  2048 x 4096 bf16 takes 37 us this way.
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
// of dgamma, then as many of dbeta, pitch partial_pitch(cols).
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
    const int64_t pitch = partial_pitch(p.cols);
    p.partials[blockIdx.y * pitch + c] = dg;
    p.partials[(gridDim.y + blockIdx.y) * pitch + c] = db;
  }
}

// dgamma (blockIdx.y 0) or dbeta (1): `parts` rows of partials (pitch
// partial_pitch) summed.  A block takes 32 columns; a warp reads four rows at a
// time, eight lanes a row in 16-byte pieces.  Many partial rows want the large
// blocks: launched while the kernel before is ending, small ones crowd on the
// SMs that it leaves first (8192 x 4096, 456 partial rows: 52 us a backward
// pass with blocks of 256, 38 of 1024); one partial row an SM wants the small
// ones (8192 x 12288: 95 and 98 us).  The sums are joined in an order that the
// lanes' and warps' numbers fix.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) ln_param_sum_kernel(const float *partials, int parts, int cols, int pitch,
                                                               float *dgamma, float *dbeta) {
  constexpr int kWarps = THREADS / 32;
  __shared__ float sm[32][33];  // [warp][column]
  griddep_launch_dependents();
  griddep_wait();
  float *out = blockIdx.y == 0 ? dgamma : dbeta;
  if (!out) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 7;
  const float *strip = partials + (int64_t)blockIdx.y * parts * pitch + (int64_t)blockIdx.x * 32;
  const float4 *src = reinterpret_cast<const float4 *>(strip) + piece;
  float2 lo = both(0.f), hi = lo;
#pragma unroll 4
  for (int k = warp * 4 + (lane >> 3); k < parts; k += THREADS / 8) {
    const float4 v = src[(int64_t)k * (pitch / 4)];
    lo = add2(lo, make_float2(v.x, v.y));
    hi = add2(hi, make_float2(v.z, v.w));
  }
#pragma unroll
  for (int o = 8; o <= 16; o <<= 1) {
    lo = add2(lo, make_float2(__shfl_xor_sync(0xffffffffu, lo.x, o), __shfl_xor_sync(0xffffffffu, lo.y, o)));
    hi = add2(hi, make_float2(__shfl_xor_sync(0xffffffffu, hi.x, o), __shfl_xor_sync(0xffffffffu, hi.y, o)));
  }
  if (lane < 8) {
    float *at = &sm[warp][piece * 4];
    at[0] = lo.x, at[1] = lo.y, at[2] = hi.x, at[3] = hi.y;
  }
  __syncthreads();
  // warp w adds up columns w, w + kWarps, ...
#pragma unroll
  for (int w = warp; w < 32; w += kWarps) {
    const float s = warp_sum(lane < kWarps ? sm[lane][w] : 0.f);
    const int64_t c = (int64_t)blockIdx.x * 32 + w;
    if (lane == 0 && c < cols) out[c] = s;
  }
}

// Rows of up to 512 * NV * 8 values of which two fit in the ring, at least 64
// where V = 1.  A block walks rows gridDim.x apart.  Their x and dy come through
// a ring of row slots in shared memory, filled by bulk copies that run as far
// ahead as the ring is deep (SlotRow): dgamma and dbeta are summed in registers
// (16 values a thread and NV), which leaves none for rows in flight.  A row is
// read from its slot twice, for the two averages and for the results; the
// block-wide barrier between, passed by every thread once it has finished with
// the row before, also frees that row's slot, which thread 0 refills.  `step`
// rows are taken between two barriers.  One partial row of dgamma and of dbeta a
// block goes to the workspace.
template <typename TX, typename TDY, typename TDX, int NV, int V, int THREADS>
__global__ void __launch_bounds__(THREADS, ring_blocks(NV, V, THREADS))
    ln_backward_ring_kernel(const LnBackward p, const int stages, const int step, const uint32_t x_bytes,
                            const uint32_t dy_bytes, uint32_t *err, const uint64_t wait_limit_ns) {
  constexpr bool kQ8 = sizeof(TX) == 1;
  constexpr int R = most_rows(NV, V);  // step is at most that
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) float2 sm[2][R][16];
  // block exponents of three steps' rows: being read, still being read by a
  // thread that is behind, and being written
  __shared__ uint8_t exps[kQ8 ? 3 : 1][R][kQ8 ? 512 : 1];
  __shared__ __align__(8) uint64_t bars[kMaxStages];
  __shared__ volatile uint32_t abort_flag;
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ring = smem_addr(slots), bar0 = smem_addr(bars), both_bytes = x_bytes + dy_bytes;
  RingPlace use, put;  // put: thread 0's
  const float inv_n = 1.0f / (float)p.cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) mbar_init(bar0 + 8 * s, 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  for (int i = threadIdx.x; i < 2 * R * 16; i += blockDim.x) (&sm[0][0][0])[i] = make_float2(0.f, 0.f);
  __syncthreads();
  griddep_wait();
  const int64_t mine = (p.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;  // rows of this block, at least one
  const auto row_of = [&](int64_t i) { return (int64_t)blockIdx.x + i * gridDim.x; };
  const auto x_row = [&](int64_t i) -> const void * {
    if constexpr (kQ8)
      return p.ck.q + row_of(i) * p.ck.ldq;
    else
      return static_cast<const TX *>(p.x) + row_of(i) * p.ldx;
  };
  const auto dy_row = [&](int64_t i) { return static_cast<const TDY *>(p.dy) + row_of(i) * p.lddy; };
  const auto fill = [&](int64_t i) {
    const uint32_t dst = ring + put.slot * both_bytes, bar = bar0 + 8u * put.slot;
    put.advance(stages);
    const uint32_t xb = SlotRow<TX, V, THREADS>::copy_bytes(x_row(i), p.cols);
    const uint32_t yb = SlotRow<TDY, V, THREADS>::copy_bytes(dy_row(i), p.cols);
    mbar_arrive_expect_tx(bar, xb + yb);
    SlotRow<TX, V, THREADS>::copy(dst, x_row(i), xb, bar);
    SlotRow<TDY, V, THREADS>::copy(dst + x_bytes, dy_row(i), yb, bar);
  };
  int64_t filled = mine < stages ? mine : stages;
  if (threadIdx.x == 0)
    for (int64_t i = 0; i < filled; ++i) fill(i);

  // fetched a step ahead: the statistics and the rows' ends; two steps ahead,
  // on their way through shared memory: the block exponents
  SlotRow<TX, V, THREADS> xr;
  SlotRow<TDY, V, THREADS> yr;
  xr.init(p.cols);
  yr.init(p.cols);
  float2 st_next[R];
  const auto fetch = [&](int64_t i) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < step && i + r < mine) st_next[r] = make_float2(p.mean[row_of(i + r)], p.rstd[row_of(i + r)]);
    if (V == 1 && i < mine) {  // one row a step
      xr.fetch_ends(x_row(i));
      yr.fetch_ends(dy_row(i));
    }
  };
  fetch(0);
  const int blocks = (p.cols + 31) / 32;  // at most one a thread
  const auto exp_at = [&](int64_t i) -> uint32_t {
    return kQ8 && i < mine && (int)threadIdx.x < blocks ? p.ck.e[row_of(i) * p.ck.lde + threadIdx.x] : 0u;
  };
  uint32_t exp_next[R] = {};
  int exp_use = 0;
  if constexpr (kQ8) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= step) break;
      if ((int)threadIdx.x < blocks) exps[0][r][threadIdx.x] = (uint8_t)exp_at(r);
      exp_next[r] = exp_at(step + r);
    }
    __syncthreads();
  }
  float2 gamma[NV * 4], dg[NV * 4], db[NV * 4];
  const auto gamma_at = [&](int c) { return c < p.cols ? load_param(p.gamma, p.param_type, c, 1.f) : 0.f; };
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = group_col<V, THREADS>(v, 2 * j), d = group_col<V, THREADS>(v, 2 * j + 1);
      gamma[v * 4 + j] = make_float2(gamma_at(c), gamma_at(d));
      dg[v * 4 + j] = db[v * 4 + j] = both(0.f);
    }
  }
  bool ok = true;
  int64_t done = 0;
  int buf = 0;
  for (int64_t i = 0; i < mine; i += step, done = i, buf ^= 1) {
    // rows i .. i + step - 1: their slots, statistics and what is past the end
    uint8_t *slot[R];
    uint32_t x_off[R], y_off[R];
    bool here[R];
    float2 st[R];
    RingPlace place = use;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      here[r] = r < step && i + r < mine;
      st[r] = st_next[r];
      slot[r] = slots + place.slot * both_bytes;
      x_off[r] = y_off[r] = 0;
      if (!here[r]) continue;
      ok = mbar_wait(bar0 + 8u * place.slot, place.parity, &abort_flag, err, wait_limit_ns) && ok;
      place.advance(stages);
      if constexpr (V == 1) {
        x_off[r] = xr.offset(x_row(i));
        y_off[r] = yr.offset(dy_row(i));
        if (ok) {
          xr.put_ends(slot[r], x_off[r]);
          yr.put_ends(slot[r] + x_bytes, y_off[r]);
        }
      }
    }
    fetch(i + step);
    const uint8_t(*exp_rows)[kQ8 ? 512 : 1] = exps[0];
    if constexpr (kQ8) {
      exp_rows = exps[exp_use];
      exp_use = exp_use == 2 ? 0 : exp_use + 1;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= step) break;
        if ((int)threadIdx.x < blocks) exps[exp_use][r][threadIdx.x] = (uint8_t)exp_next[r];
        exp_next[r] = exp_at(i + 2 * step + r);
      }
    }
    // x as xh and dy of group v of row r of the step
    const auto load = [&](int r, int v, float2(&xh)[4], float2(&d)[4]) {
      const float2 minus_mean = both(-st[r].x), rstd = both(st[r].y);
      xr.load(slot[r], x_off[r], v, p.cols, xh);
      yr.load(slot[r] + x_bytes, y_off[r], v, p.cols, d);
      float2 scale = both(1.f);
      if constexpr (kQ8 && V == 8) scale = both(q8_scale(exp_rows[r][group_col<V, THREADS>(v, 0) >> 5]));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kQ8 && V == 1) {
          const int c = group_col<V, THREADS>(v, 2 * j), e = group_col<V, THREADS>(v, 2 * j + 1);
          scale = make_float2(q8_scale(exp_rows[r][c < p.cols ? c >> 5 : 0]),
                              q8_scale(exp_rows[r][e < p.cols ? e >> 5 : 0]));
        }
        xh[j] = mul2(kQ8 ? fma2(xh[j], scale, minus_mean) : add2(xh[j], minus_mean), rstd);
      }
    };
    float a[R], b[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 a2 = both(0.f), b2 = both(0.f);
      if (here[r]) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          if (V == 8 && group_col<V, THREADS>(v, 0) >= p.cols) continue;
          float2 xh[4], d[4];
          load(r, v, xh, d);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 g = mul2(d[j], gamma[v * 4 + j]);
            a2 = add2(a2, g);
            b2 = fma2(g, xh[j], b2);
          }
        }
      }
      a[r] = a2.x + a2.y;
      b[r] = b2.x + b2.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        a[r] += __shfl_xor_sync(0xffffffffu, a[r], o);
        b[r] += __shfl_xor_sync(0xffffffffu, b[r], o);
      }
    if (lane == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) sm[buf][r][warp] = make_float2(a[r], b[r]);
    }
    // every wait of the block succeeded, or the block gives up together
    if (!__syncthreads_and(ok)) {
      ok = false;
      break;
    }
    if (threadIdx.x == 0 && i > 0)  // the slots of the step before
      for (int r = 0; r < step && filled < mine; ++r) fill(filled++);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!here[r]) continue;
      use.advance(stages);
      const float2 s = sum_over_warps<THREADS / 32>(sm[buf][r]);
      const float2 ga = both(-s.x * inv_n * st[r].y), gx = both(-s.y * inv_n * st[r].y), rstd = both(st[r].y);
      TDX *dx = static_cast<TDX *>(p.dx) + row_of(i + r) * p.lddx;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (V == 8 && group_col<V, THREADS>(v, 0) >= p.cols) continue;
        float2 xh[4], d[4];
        float o[8];
        load(r, v, xh, d);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dg[v * 4 + j] = fma2(d[j], xh[j], dg[v * 4 + j]);
          db[v * 4 + j] = add2(db[v * 4 + j], d[j]);
          const float2 w = fma2(mul2(d[j], gamma[v * 4 + j]), rstd, fma2(xh[j], gx, ga));
          o[2 * j] = w.x;
          o[2 * j + 1] = w.y;
        }
        if constexpr (V == 8) {
          store_chunk<TDX, 8>(dx, group_col<V, THREADS>(v, 0), o, 8);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int c = group_col<V, THREADS>(v, k);
            if (c < p.cols) store_value<TDX>(dx, c, o[k]);
          }
        }
      }
    }
  }
  if (!ok) {
    if (threadIdx.x == 0) ring_drain(bar0, stages, use, filled - done);
    return;
  }
  // the only block has the whole sums; else one partial row each of the block's
  const bool whole = gridDim.x == 1;
  if (!whole && !p.partials) return;
  float *dg_out = whole ? p.dgamma : p.partials + (int64_t)blockIdx.x * partial_pitch(p.cols);
  float *db_out = whole ? p.dbeta : p.partials + (int64_t)(gridDim.x + blockIdx.x) * partial_pitch(p.cols);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (V == 8 && !whole) {
      const int c = group_col<V, THREADS>(v, 0);
      if (c < p.cols) {
        store_chunk<float, 8>(dg_out, c, reinterpret_cast<const float *>(dg + v * 4), 8);
        store_chunk<float, 8>(db_out, c, reinterpret_cast<const float *>(db + v * 4), 8);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int c = group_col<V, THREADS>(v, k);
        if (c < p.cols) {
          if (dg_out) dg_out[c] = (k & 1) ? dg[v * 4 + (k >> 1)].y : dg[v * 4 + (k >> 1)].x;
          if (db_out) db_out[c] = (k & 1) ? db[v * 4 + (k >> 1)].y : db[v * 4 + (k >> 1)].x;
        }
      }
    }
  }
}

// How a backward pass runs.
enum LnPath { kLnAny, kLnRing };
struct LnPlan {
  LnPath path;
  int grid, parts;  // blocks; partial rows of the parameter gradients
  // kLnRing
  int nv, threads, stages, step;
  bool aligned;                // V = 8, else 1
  uint32_t x_bytes, dy_bytes;  // of a slot
};

// The ring kernel's only block writes dgamma and dbeta itself.
bool writes_whole_sums(const LnPlan &l) { return l.path == kLnRing && l.grid == 1; }

// Blocks that walk `rows` rows, `per_sm` at a time on an SM: every SM one
// while there are few rows, more where each still has two rows to set against
// the partial row that it writes and another kernel reads (1000 rows of 1500
// from a checkpoint: 36 us with 152 blocks, 17.5 with 500).
//
// Up to four rows go to one block, which then has the whole sums: a launch less
// is worth more than the rows' latencies side by side.
int row_blocks(int64_t rows, int sms, int per_sm) {
  if (rows <= 4) return 1;
  const int64_t few = rows < sms ? rows : sms, many = ceil_div64(rows, 2), most = (int64_t)sms * per_sm;
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
  l.aligned = (int64_t)p.cols * sx % 16 == 0 && (int64_t)p.cols * sg % 16 == 0 && p.cols % 8 == 0 &&
              rows_on(x, ldx, sx, 16) && rows_on(p.dy, p.lddy, sg, 16) && rows_on(p.dx, p.lddx, so, 16);
  // few threads with more values each: a row's fixed costs (its barrier, the
  // sums over lanes and warps) are paid by every warp.  32768 x 1024: 51 us
  // with 8 values a thread, 44 with 16; 8192 x 4096: 41.7 us with 16, 39.8 with
  // 32 (from a checkpoint 48.8 and 44.9), which take three blocks an SM where 16
  // take two, and so many rows that the third's partial sums do not matter (2048
  // x 4096: 18.9 and 19.9 us).  Four times as many rows lose a little: 32768 x
  // 4096 132 and 140 us.
  l.nv = eights <= (l.aligned ? 32 : 128) ? 1 : eights <= 2 * kRingThreads ? 2 : (int)ceil_div64(eights, kRingThreads);
  if (l.aligned && eights > 256 && eights <= 512 && p.rows >= (int64_t)32 * sms) l.nv = 4;
  // two blocks of up to 256 threads an SM instead of one of up to 384, where
  // both have four slots (8192 x 5120 bf16: 57.8 us with one, then 50.7 with two;
  // 3543 x 5690, unaligned: 49.9 and 39.8)
  if (eights > 512 && eights <= 768 &&
      kRingBytes / 2 / (slot_bytes(p.cols, sx, l.aligned) + slot_bytes(p.cols, sg, l.aligned)) >= 4)
    l.nv = 3;
  if (p.rows > 0 && l.nv <= 4 && (l.aligned || p.cols >= 64)) {
    l.x_bytes = slot_bytes(p.cols, sx, l.aligned);
    l.dy_bytes = slot_bytes(p.cols, sg, l.aligned);
    l.threads = (int)ceil_div64(ceil_div64(eights, l.nv), 32) * 32;
    if (!l.aligned) {  // one of the block sizes compiled
      l.threads = l.nv == 1              ? l.threads <= 32 ? 32 : l.threads <= 64 ? 64 : 128
                  : l.threads <= 128     ? 128
                  : l.threads <= 256 && l.nv <= 3 ? 256
                                         : 512;
    }
    int per_sm = ring_blocks(l.nv, l.aligned ? 8 : 1, l.threads);
    per_sm = per_sm > 16 ? 16 : per_sm;
    int64_t stages = kRingBytes / per_sm / (l.x_bytes + l.dy_bytes);
    if (stages < 2) {
      per_sm = 1;
      stages = kRingBytes / (l.x_bytes + l.dy_bytes);
    }
    if (stages >= 2) {
      l.path = kLnRing;
      l.stages = (int)(stages < kMaxStages ? stages : kMaxStages);
      l.step = l.stages >= 4 ? most_rows(l.nv, l.aligned ? 8 : 1) : 1;
      l.grid = l.parts = row_blocks(p.rows, sms, per_sm);
      return l;
    }
  }
  // dx by one kernel, partials by another: enough blocks of 32 columns x 8
  // rows at a time to fill the device several times over, no more than there
  // are groups of rows
  l.path = kLnAny;
  l.grid = grid_cap(p.rows, (int64_t)sms * 8);
  l.parts = grid_cap(ceil_div64((int64_t)sms * 16, ceil_div64(p.cols, 32)), ceil_div64(p.rows < 1 ? 1 : p.rows, 8));
  return l;
}

template <typename TX, typename TDY, typename TDX, int NV, int V, int THREADS>
cudaError_t run_ring(const LnBackward &p, const LnPlan &l, const OpContext &c) {
  const auto kern = ln_backward_ring_kernel<TX, TDY, TDX, NV, V, THREADS>;
  const size_t smem = (size_t)l.stages * (l.x_bytes + l.dy_bytes);
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared_memory((const void *)kern, kRingBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch_ex(kern, dim3(l.grid), dim3(l.threads), smem, c.st, 1, p, l.stages, l.step, l.x_bytes, l.dy_bytes,
                   c.err, c.wait_limit_ns);
}

template <typename TX, typename TDY, typename TDX>
cudaError_t run_width(const LnBackward &p, const LnPlan &l, const OpContext &c) {
  if (l.aligned)
    return l.nv == 1   ? run_ring<TX, TDY, TDX, 1, 8, 128>(p, l, c)
           : l.nv == 2 ? run_ring<TX, TDY, TDX, 2, 8, 512>(p, l, c)
           : l.nv == 3 ? l.threads <= 256 ? run_ring<TX, TDY, TDX, 3, 8, 256>(p, l, c)
                                          : run_ring<TX, TDY, TDX, 3, 8, 512>(p, l, c)
           : l.threads <= 128 ? run_ring<TX, TDY, TDX, 4, 8, 128>(p, l, c)
                              : run_ring<TX, TDY, TDX, 4, 8, 512>(p, l, c);
  if (l.nv == 1)
    return l.threads == 32   ? run_ring<TX, TDY, TDX, 1, 1, 32>(p, l, c)
           : l.threads == 64 ? run_ring<TX, TDY, TDX, 1, 1, 64>(p, l, c)
                             : run_ring<TX, TDY, TDX, 1, 1, 128>(p, l, c);
  if (l.nv == 3)
    return l.threads == 256 ? run_ring<TX, TDY, TDX, 3, 1, 256>(p, l, c) : run_ring<TX, TDY, TDX, 3, 1, 512>(p, l, c);
  if (l.nv == 4) return run_ring<TX, TDY, TDX, 4, 1, 512>(p, l, c);
  return l.threads == 128   ? run_ring<TX, TDY, TDX, 2, 1, 128>(p, l, c)
         : l.threads == 256 ? run_ring<TX, TDY, TDX, 2, 1, 256>(p, l, c)
                            : run_ring<TX, TDY, TDX, 2, 1, 512>(p, l, c);
}

template <typename TX, typename TDY, typename TDX>
cudaError_t run_types(const LnBackward &p, const OpContext &c, int *launches) {
  const LnPlan l = plan_ln_backward(p, c.sms);
  const dim3 grid(l.grid);
  cudaError_t e = cudaSuccess;
  if (p.rows > 0) {
    ++*launches;
    if (l.path == kLnRing)
      e = run_width<TX, TDY, TDX>(p, l, c);
    else
      e = launch_ex(ln_backward_any_kernel<TX, TDY, TDX>, grid, dim3(kRowThreads), 0, c.st, 1, p);
    if (e != cudaSuccess) return e;
  }
  if (!p.partials || writes_whole_sums(l)) return e;
  const int strips = (int)ceil_div64(p.cols, 32);
  if (l.path == kLnAny) {
    ++*launches;
    e = launch_ex(ln_param_partials_kernel<TX, TDY>, dim3(strips, l.parts), dim3(kRowThreads), 0, c.st, 1, p);
    if (e != cudaSuccess) return e;
  }
  ++*launches;
  const bool few = l.parts <= c.sms;
  return launch_ex(few ? ln_param_sum_kernel<256> : ln_param_sum_kernel<1024>, dim3(strips, 2),
                   dim3(few ? 256 : 1024), 0, c.st, 1, (const float *)p.partials, l.parts, p.cols,
                   partial_pitch(p.cols), p.dgamma, p.dbeta);
}

}  // namespace

size_t ln_backward_partials(const LnBackward &p, int sms) {
  if (!p.dgamma && !p.dbeta) return 0;
  const LnPlan l = plan_ln_backward(p, sms);
  return writes_whole_sums(l) ? 0 : (size_t)2 * l.parts * partial_pitch(p.cols);
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
