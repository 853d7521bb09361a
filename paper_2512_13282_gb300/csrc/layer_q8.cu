// layer_q8.cu -- the 8-bit checkpoint's save and restore.
//
// Both only move bytes: a saved value costs its own size read and 1 + 1/32
// bytes written, a restored one the reverse, so the HBM sets the time and the
// kernels' part is to keep enough loads in flight.  A thread takes half a
// block (16 values: 16-byte loads and stores on both sides), two neighbouring
// lanes one block, whose largest magnitude they exchange with one shuffle; the
// grid covers every half block once, which leaves the scheduling of loads to
// the many warps of an SM rather than to a loop.
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

// VEC: rows of x start on 16 bytes and rows of q on 16; else any alignment.
template <typename TX, bool VEC>
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
    if (VEC && n == 16)
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
    if (VEC && n == 16) {
      *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) q[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
    }
    if (live && (h & 1) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)e;
  }
}

template <typename TX, bool VEC>
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
    if (VEC && n == 16)
      raw.load(q, c);
    else
      raw.load_part(q, c, n);
    TX *row = static_cast<TX *>(x) + r * ldx;
    if constexpr (sizeof(TX) == 2) {
      if (VEC && n == 16) {
        const __nv_bfloat162 s = __float2bfloat162_rn(scale);
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s8x4_to_bf16x4(raw.w[i], o[2 * i], o[2 * i + 1]);
          o[2 * i] = scale_bf16x2(o[2 * i], s);
          o[2 * i + 1] = scale_bf16x2(o[2 * i + 1], s);
        }
        uint4 *d = reinterpret_cast<uint4 *>(row + c);
        d[0] = make_uint4(o[0], o[1], o[2], o[3]);
        d[1] = make_uint4(o[4], o[5], o[6], o[7]);
        continue;
      }
    }
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = raw.get(i) * scale;
    if constexpr (VEC)
      store_chunk<TX, 16>(row, c, v, n);
    else
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) store_value<TX>(row, c + i, v[i]);
  }
}

// Whether a matrix's rows, and with it a vector access per 16 elements, start
// on 16-byte boundaries.
bool rows16(const void *p, int64_t ld, int size) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0;
}

struct Q8Launch {
  int64_t rows, cols;
  bool vec;
  dim3 grid;
};
Q8Launch plan_q8(const Q8Ref &ck, const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols) {
  Q8Launch l{rows, cols, rows16(x, ldx, x_type == GEMM_TYPE_BF16 ? 2 : 4) && rows16(ck.q, ck.ldq, 1), dim3(1)};
  // rows that follow one another without a gap, in whole blocks: one long row
  if (cols % kQ8Block == 0 && ldx == cols && ck.ldq == cols && ck.lde == cols / kQ8Block) {
    l.cols = rows * cols;
    l.rows = 1;
  }
  const int64_t items = l.rows * ((l.cols + 31) / 32 * 2), blocks = (items + kQ8Threads - 1) / kQ8Threads;
  l.grid.x = (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30));
  return l;
}

}  // namespace

cudaError_t launch_q8_save(const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols, const Q8Ref &ck,
                           cudaStream_t st) {
  const Q8Launch l = plan_q8(ck, x, ldx, x_type, rows, cols);
  const dim3 block(kQ8Threads);
  if (x_type == GEMM_TYPE_BF16)
    return l.vec ? launch_ex(q8_save_kernel<bf16, true>, l.grid, block, 0, st, 1, x, ldx, l.rows, l.cols, ck)
                 : launch_ex(q8_save_kernel<bf16, false>, l.grid, block, 0, st, 1, x, ldx, l.rows, l.cols, ck);
  return l.vec ? launch_ex(q8_save_kernel<float, true>, l.grid, block, 0, st, 1, x, ldx, l.rows, l.cols, ck)
               : launch_ex(q8_save_kernel<float, false>, l.grid, block, 0, st, 1, x, ldx, l.rows, l.cols, ck);
}

cudaError_t launch_q8_restore(const Q8Ref &ck, void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols,
                              cudaStream_t st) {
  const Q8Launch l = plan_q8(ck, x, ldx, x_type, rows, cols);
  const dim3 block(kQ8Threads);
  if (x_type == GEMM_TYPE_BF16)
    return l.vec ? launch_ex(q8_restore_kernel<bf16, true>, l.grid, block, 0, st, 1, ck, x, ldx, l.rows, l.cols)
                 : launch_ex(q8_restore_kernel<bf16, false>, l.grid, block, 0, st, 1, ck, x, ldx, l.rows, l.cols);
  return l.vec ? launch_ex(q8_restore_kernel<float, true>, l.grid, block, 0, st, 1, ck, x, ldx, l.rows, l.cols)
               : launch_ex(q8_restore_kernel<float, false>, l.grid, block, 0, st, 1, ck, x, ldx, l.rows, l.cols);
}

}  // namespace gb300
