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

// A half block's bytes and its block's exponent (the other half is the
// neighbouring lane's).
struct Q8Half {
  uint32_t w[4], e;
};
template <typename TX>
__device__ __forceinline__ Q8Half q8_half(const Chunk<TX, 16> &raw) {
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
  return Q8Half{{wl.x, wl.y, wh.x, wh.y}, e};
}
// A half block's values in bf16.
__device__ __forceinline__ void q8_restored(const Chunk<Q8, 16> &raw, float scale, uint32_t (&o)[8]) {
  const __nv_bfloat162 s = __float2bfloat162_rn(scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s8x4_to_bf16x4(raw.w[i], o[2 * i], o[2 * i + 1]);
    o[2 * i] = scale_bf16x2(o[2 * i], s);
    o[2 * i + 1] = scale_bf16x2(o[2 * i + 1], s);
  }
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
    const Q8Half b = q8_half(raw);
    int8_t *q = ck.q + r * ck.ldq + c;
    if (n == 16)
      *reinterpret_cast<uint4 *>(q) = make_uint4(b.w[0], b.w[1], b.w[2], b.w[3]);
    else
      store_bytes(q, b.w, n);
    if (live && (h & 1) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)b.e;
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
        uint32_t o[8];
        q8_restored(raw, scale, o);
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

// Rows at any alignment: the same half blocks, shifted between registers and
// the 16-byte pieces of memory that they lie in (load_half, store_shifted).
// 1792 x 10471 bf16: save 16.5 us, restore 15.3; a warp per 256 values of a
// row, a lane one value of each 32, took 36.4 and 23.6.

template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_save_any_kernel(const void *x, int64_t ldx, int64_t rows, int64_t cols, Q8Ref ck) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t halves = (cols + 31) / 32 * 2, items = rows * halves, step = (int64_t)gridDim.x * kQ8Threads;
  const int lane = threadIdx.x & 31;
  for (int64_t h0 = (int64_t)blockIdx.x * kQ8Threads; h0 < items; h0 += step) {
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    int64_t r, c;
    half_block(live ? h : items - 1, halves, &r, &c);
    const int n = !live || c >= cols ? 0 : (int)min((int64_t)16, cols - c);
    const TX *row = static_cast<const TX *>(x) + r * ldx;
    Chunk<TX, 16> raw;
    if (n == 16)
      load_half(row + c, c == 0, (cols - c - 16) * (int64_t)sizeof(TX), raw.w);
    else
      raw.load_part(row, c, n);
    const Q8Half b = q8_half(raw);
    int8_t *q = ck.q + r * ck.ldq + c;
    store_shifted<4>(q, n == 16, lane > 0 && c > 0, lane < 31 && c + 32 <= cols, b.w);
    if (n < 16) store_bytes(q, b.w, n);
    if (live && (h & 1) == 0) ck.e[r * ck.lde + (c >> 5)] = (uint8_t)b.e;
  }
}

template <typename TX>
__global__ void __launch_bounds__(kQ8Threads)
    q8_restore_any_kernel(Q8Ref ck, void *x, int64_t ldx, int64_t rows, int64_t cols) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t halves = (cols + 31) / 32 * 2, items = rows * halves, step = (int64_t)gridDim.x * kQ8Threads;
  const int lane = threadIdx.x & 31;
  for (int64_t h0 = (int64_t)blockIdx.x * kQ8Threads; h0 < items; h0 += step) {
    const int64_t h = h0 + threadIdx.x;
    const bool live = h < items;
    int64_t r, c;
    half_block(live ? h : items - 1, halves, &r, &c);
    const int n = !live || c >= cols ? 0 : (int)min((int64_t)16, cols - c);
    const int8_t *q = ck.q + r * ck.ldq;
    const float scale = n > 0 ? q8_scale(ck.e[r * ck.lde + (c >> 5)]) : 0.f;
    Chunk<Q8, 16> raw;
    if (n == 16)
      load_half(q + c, c == 0, cols - c - 16, raw.w);
    else
      raw.load_part(q, c, n);
    TX *row = static_cast<TX *>(x) + r * ldx;
    uint32_t o[4 * sizeof(TX)];
    if constexpr (sizeof(TX) == 2) {
      q8_restored(raw, scale, o);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(raw.get(i) * scale);
    }
    store_shifted<4>(row + c, n == 16, lane > 0 && c > 0, lane < 31 && c + 32 <= cols, o);
    if (n < 16) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) {
          if constexpr (sizeof(TX) == 2)
            reinterpret_cast<uint16_t *>(row)[c + i] = (uint16_t)(o[i / 2] >> (16 * (i & 1)));
          else
            reinterpret_cast<uint32_t *>(row)[c + i] = o[i];
        }
    }
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
  const int64_t items = l.rows * ((l.cols + 31) / 32 * 2);
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
