// layer_q8.cu -- the 8-bit checkpoint's save and restore.
//
// Both only move bytes: a saved value costs its own size read and 1 + 1/32
// bytes written, a restored one the reverse, so the HBM sets the time and the
// kernels' part is to keep enough loads in flight.  A thread takes half a
// block (16 values: 16-byte loads and stores on both sides), two neighbouring
// lanes one block, whose largest magnitude they exchange with one shuffle; the
// grid covers every half block once, which leaves the scheduling of loads to
// the many warps of an SM rather than to a loop.  Measured, 8192 x 12288 bf16:
// save 46 us (6.6 TB/s), restore 52 us (5.9 TB/s; it writes two bytes for each
// it reads, and writes are the slower half).
#include "layer_rows.cuh"

namespace gb300 {

namespace {

constexpr int kQ8Threads = 256;

// Half block h of the matrix -> its row and first column, `halves` of them a
// row (an even number).  With rows laid end to end the launcher makes the
// matrix one row, and 32-bit arithmetic serves any matrix below 2^32 halves.
__device__ __forceinline__ void half_block(int64_t h, int64_t halves, int64_t *r, int64_t *c) {
  int64_t row;
  if ((uint64_t)h <= 0xFFFFFFFFull && halves <= 0xFFFFFFFFll)
    row = (uint32_t)h / (uint32_t)halves;
  else
    row = h / halves;
  *r = row;
  *c = (h - row * halves) * 16;
}

// Rows of x and of q start on 16 bytes.
template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_save_kernel(const void *x, int64_t ldx, int64_t rows, int64_t cols, Q8Ref ck) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t halves = (cols + 31) / 32 * 2, items = rows * halves, step = (int64_t)gridDim.x * kQ8Threads;
  for (int64_t h0 = (int64_t)blockIdx.x * kQ8Threads; h0 < items; h0 += step) {
    // items is even, so both lanes of a block are in range or neither is
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    int64_t r, c;
    half_block(live ? h : items - 1, halves, &r, &c);
    const int n = !live || c >= cols ? 0 : (int)min((int64_t)16, cols - c);
    const TX *row = static_cast<const TX *>(x) + r * ldx;
    Chunk<TX, 16> raw;
    if (n == 16)
      raw.load(row, c);
    else
      raw.load_part(row, c, n);
    uint32_t top = 0;
    if constexpr (sizeof(TX) == 2) {
      top = max_magnitude_bf16<8>(raw.w);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, raw.w[i] & 0x7FFFFFFFu);
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t e = q8_exponent(top);
    float2 lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) lo[j] = raw.get2(j), hi[j] = raw.get2(4 + j);
    const uint2 wl = q8_pack8(lo, e), wh = q8_pack8(hi, e);
    const uint32_t w[4] = {wl.x, wl.y, wh.x, wh.y};
    int8_t *q = ck.q + r * ck.ldq + c;
    if (n == 16) {
      *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) q[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
    }
    if (live && (h & 1) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)e;
  }
}

template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_restore_kernel(Q8Ref ck, void *x, int64_t ldx, int64_t rows, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t halves = (cols + 31) / 32 * 2, items = rows * halves, step = (int64_t)gridDim.x * kQ8Threads;
  for (int64_t h = (int64_t)blockIdx.x * kQ8Threads + threadIdx.x; h < items; h += step) {
    int64_t r, c;
    half_block(h, halves, &r, &c);
    if (c >= cols) continue;
    const int n = (int)min((int64_t)16, cols - c);
    const int8_t *q = ck.q + r * ck.ldq;
    const float scale = q8_scale(ck.e[r * ck.lde + (c >> 5)]);
    Chunk<Q8, 16> raw;
    if (n == 16)
      raw.load(q, c);
    else
      raw.load_part(q, c, n);
    TX *row = static_cast<TX *>(x) + r * ldx;
    if constexpr (sizeof(TX) == 2) {
      if (n == 16) {
        const __nv_bfloat162 s = __float2bfloat162_rn(scale);
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s8x4_to_bf16x4(raw.w[i], o[2 * i], o[2 * i + 1]);
          o[2 * i] = scale_bf16x2(o[2 * i], s);
          o[2 * i + 1] = scale_bf16x2(o[2 * i + 1], s);
        }
        store_32_bytes(row + c, o);
        continue;
      }
    }
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = raw.get(i) * scale;
    store_chunk<TX, 16>(row, c, v, n);
  }
}

// Any alignment: a warp takes kRun blocks of a row, a lane one value of each,
// so that neighbouring lanes are neighbours in memory and kRun loads are in
// flight a lane; a block's largest magnitude is one reduction over the warp.
// Save and restore of 512 x 10216 float32 with a pitch of 10221: 20 us, which
// a thread per half block with element accesses took 43 for.
constexpr int kRun = 8;

template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_save_any_kernel(const void *x, int64_t ldx, int64_t rows, int64_t cols, Q8Ref ck) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t runs = (cols + 32 * kRun - 1) / (32 * kRun), items = rows * runs;
  const int64_t step = (int64_t)gridDim.x * (kQ8Threads / 32);
  for (int64_t t = (int64_t)blockIdx.x * (kQ8Threads / 32) + (threadIdx.x >> 5); t < items; t += step) {
    const int64_t r = t / runs, c0 = (t - r * runs) * (32 * kRun) + lane;
    float v[kRun];
#pragma unroll
    for (int k = 0; k < kRun; ++k) v[k] = c0 + 32 * k < cols ? load_value<TX>(x, r * ldx + c0 + 32 * k) : 0.f;
    int8_t *q = ck.q + r * ck.ldq;
    uint8_t *ex = ck.e + r * ck.lde;
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const int64_t c = c0 + 32 * k;
      const uint32_t e = q8_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(v[k]) & 0x7FFFFFFFu));
      if (c < cols) q[c] = (int8_t)q8_byte(v[k], q8_inverse(e), e);
      if (lane == 0 && c < cols) ex[c >> 5] = (uint8_t)e;
    }
  }
}

template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_restore_any_kernel(Q8Ref ck, void *x, int64_t ldx, int64_t rows, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t runs = (cols + 32 * kRun - 1) / (32 * kRun), items = rows * runs;
  const int64_t step = (int64_t)gridDim.x * (kQ8Threads / 32);
  for (int64_t t = (int64_t)blockIdx.x * (kQ8Threads / 32) + (threadIdx.x >> 5); t < items; t += step) {
    const int64_t r = t / runs, c0 = (t - r * runs) * (32 * kRun) + lane;
    const int8_t *q = ck.q + r * ck.ldq;
    const uint8_t *ex = ck.e + r * ck.lde;
    float v[kRun];
    uint32_t e[kRun];
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const int64_t c = c0 + 32 * k;
      v[k] = c < cols ? (float)q[c] : 0.f;
      e[k] = c < cols ? ex[c >> 5] : 0u;
    }
#pragma unroll
    for (int k = 0; k < kRun; ++k)
      if (c0 + 32 * k < cols) store_value<TX>(x, r * ldx + c0 + 32 * k, v[k] * q8_scale(e[k]));
  }
}

struct Q8Launch {
  int64_t rows, cols;
  bool vec;
  dim3 grid;
};
Q8Launch plan_q8(const Q8Ref &ck, const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols) {
  const int size = x_type == GEMM_TYPE_BF16 ? 2 : 4;
  Q8Launch l{rows, cols, rows_on(x, ldx, size, 16) && rows_on(ck.q, ck.ldq, 1, 16), dim3(1)};
  // rows that follow one another without a gap, in whole blocks: one long row
  if (cols % kQ8Block == 0 && ldx == cols && ck.ldq == cols && ck.lde == cols / kQ8Block) {
    l.cols = rows * cols;
    l.rows = 1;
  }
  const int64_t items = l.vec ? l.rows * ((l.cols + 31) / 32 * 2)
                              : l.rows * ((l.cols + 32 * kRun - 1) / (32 * kRun)) * 32;
  const int64_t blocks = (items + kQ8Threads - 1) / kQ8Threads;
  l.grid.x = (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30));
  return l;
}

}  // namespace

cudaError_t launch_q8_save(const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols, const Q8Ref &ck,
                           cudaStream_t st) {
  const Q8Launch l = plan_q8(ck, x, ldx, x_type, rows, cols);
  const bool bf = x_type == GEMM_TYPE_BF16;
  const auto kern = l.vec ? bf ? q8_save_kernel<bf16> : q8_save_kernel<float>
                          : bf ? q8_save_any_kernel<bf16> : q8_save_any_kernel<float>;
  return launch_ex(kern, l.grid, dim3(kQ8Threads), 0, st, 1, x, ldx, l.rows, l.cols, ck);
}

cudaError_t launch_q8_restore(const Q8Ref &ck, void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols,
                              cudaStream_t st) {
  const Q8Launch l = plan_q8(ck, x, ldx, x_type, rows, cols);
  const bool bf = x_type == GEMM_TYPE_BF16;
  const auto kern = l.vec ? bf ? q8_restore_kernel<bf16> : q8_restore_kernel<float>
                          : bf ? q8_restore_any_kernel<bf16> : q8_restore_any_kernel<float>;
  return launch_ex(kern, l.grid, dim3(kQ8Threads), 0, st, 1, ck, x, ldx, l.rows, l.cols);
}

}  // namespace gb300
