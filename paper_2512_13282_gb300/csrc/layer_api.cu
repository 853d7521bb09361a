// layer_api.cu -- the C ABI of include/gb300_layer.h: argument checks,
// scratch and launches of the layer operators.
#include <cmath>

#include "gb300_layer.h"
#include "layer_internal.h"

using namespace gb300;

namespace {

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t type_size(int type) { return type == GEMM_TYPE_BF16 ? 2 : 4; }
inline bool known_type(int type) { return type == GEMM_TYPE_F32 || type == GEMM_TYPE_BF16; }
inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Row widths and extents the kernels count in 32 bits.
constexpr int64_t kMaxExtent = int64_t(1) << 30;

// A rows x cols matrix of `type` with rows and cols above zero.
bool matrix_ok(const void *p, int type, int64_t ld, int64_t cols) {
  return p && known_type(type) && ld >= cols && aligned_to(p, type_size(type));
}
bool checkpoint_ok(const void *q, int64_t ldq, const void *e, int64_t lde, int64_t cols) {
  return q && e && ldq >= cols && lde >= ceil_div64(cols, kQ8Block);
}
// A vector of `type`, or absent.
bool vector_ok(const void *p, int type) { return !p || (known_type(type) && aligned_to(p, type_size(type))); }

gemm_status_t launched(cudaError_t e) { return e == cudaSuccess ? GEMM_OK : GEMM_ERR_CUDA; }

gemm_status_t extents(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return GEMM_ERR_INVALID_ARG;
  return rows > INT32_MAX || cols > kMaxExtent ? GEMM_ERR_UNSUPPORTED : GEMM_OK;
}

bool bf16_ok(const void *p, int64_t ld, int64_t cols) { return matrix_ok(p, GEMM_TYPE_BF16, ld, cols); }

// A gate's gradient: everything but where dH comes from.
bool gate_backward_ok(const GatedBackward &p, int64_t F) {
  return bf16_ok(p.g, p.ldg, F) && bf16_ok(p.u, p.ldu, F) && bf16_ok(p.dg, p.lddg, F) && bf16_ok(p.du, p.lddu, F) &&
         !p.ck.q == !p.ck.e && (!p.ck.q || checkpoint_ok(p.ck.q, p.ck.ldq, p.ck.e, p.ck.lde, F));
}
inline bool known_layout(int l) { return l == GEMM_B_ROW_MAJOR_KxN || l == GEMM_B_COL_MAJOR_NxK; }
inline bool known_activation(int a) { return a >= GEMM_ACT_SILU && a <= GEMM_ACT_RELU; }

gemm_status_t dropout(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type, const void *residual,
                      int64_t ldr, void *y, int64_t ldy, int y_type, float p, uint64_t seed, uint64_t step,
                      const uint64_t *step_device, gemm_stream_t stream) {
  gemm_status_t s = extents(rows, cols);
  if (s == GEMM_ERR_INVALID_ARG || !known_type(x_type) || !known_type(y_type) || !(p >= 0.f && p <= 1.f))
    return GEMM_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return GEMM_OK;
  if (!matrix_ok(x, x_type, ldx, cols) || !matrix_ok(y, y_type, ldy, cols) ||
      (residual && !matrix_ok(residual, y_type, ldr, cols)) || !aligned_to(step_device, 8))
    return GEMM_ERR_INVALID_ARG;
  if (s != GEMM_OK) return s;
  OpContext c;
  if ((s = op_context(reinterpret_cast<cudaStream_t>(stream), &c)) != GEMM_OK) return s;
  count_launches(1);
  return launched(launch_dropout(Dropout{rows, cols, x, ldx, x_type, residual, ldr, y, ldy, y_type,
                                         (uint32_t)std::lrintf(p * 65536.f), seed, step, step_device},
                                 c.st));
}

}  // namespace

extern "C" {

gemm_status_t gemm_layernorm_forward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                     const void *gamma, const void *beta, int param_type, float eps,
                                     void *y, int64_t ldy, int y_type, float *mean, float *rstd,
                                     int8_t *q, int64_t ldq, uint8_t *e, int64_t lde, gemm_stream_t stream) {
  gemm_status_t s = extents(rows, cols);
  if (s == GEMM_ERR_INVALID_ARG || !known_type(x_type) || !known_type(y_type) || !known_type(param_type) ||
      !(eps >= 0.0f))
    return GEMM_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return GEMM_OK;
  if (!matrix_ok(x, x_type, ldx, cols) || !matrix_ok(y, y_type, ldy, cols) || !vector_ok(gamma, param_type) ||
      !vector_ok(beta, param_type) || !vector_ok(mean, GEMM_TYPE_F32) || !vector_ok(rstd, GEMM_TYPE_F32) || !q != !e)
    return GEMM_ERR_INVALID_ARG;
  if (q && !checkpoint_ok(q, ldq, e, lde, cols)) return GEMM_ERR_INVALID_ARG;
  if (s != GEMM_OK) return s;
  OpContext c;
  if ((s = op_context(reinterpret_cast<cudaStream_t>(stream), &c)) != GEMM_OK) return s;
  const LnForward p{rows, (int)cols, x, ldx, x_type, gamma, beta, param_type, eps, y, ldy, y_type, mean, rstd,
                    Q8Ref{q, ldq, e, lde}};
  count_launches(1);
  return launched(launch_ln_forward(p, c));
}

gemm_status_t gemm_layernorm_backward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                      const int8_t *q, int64_t ldq, const uint8_t *e, int64_t lde,
                                      const void *gamma, int param_type, const float *mean, const float *rstd,
                                      const void *dy, int64_t lddy, int dy_type, void *dx, int64_t lddx,
                                      int dx_type, float *dgamma, float *dbeta, gemm_stream_t stream) {
  gemm_status_t s = extents(rows, cols);
  if (s == GEMM_ERR_INVALID_ARG || !known_type(dy_type) || !known_type(dx_type) || !known_type(param_type))
    return GEMM_ERR_INVALID_ARG;
  if (cols == 0) return GEMM_OK;
  if (!vector_ok(gamma, param_type) || !vector_ok(dgamma, GEMM_TYPE_F32) || !vector_ok(dbeta, GEMM_TYPE_F32))
    return GEMM_ERR_INVALID_ARG;
  if (rows > 0) {
    if (x ? (q || e || x_type != dx_type || !matrix_ok(x, x_type, ldx, cols)) : !checkpoint_ok(q, ldq, e, lde, cols))
      return GEMM_ERR_INVALID_ARG;
    if (!matrix_ok(dy, dy_type, lddy, cols) || !matrix_ok(dx, dx_type, lddx, cols) || !mean || !rstd ||
        !vector_ok(mean, GEMM_TYPE_F32) || !vector_ok(rstd, GEMM_TYPE_F32))
      return GEMM_ERR_INVALID_ARG;
  }
  if (s != GEMM_OK) return s;
  if (rows == 0 && !dgamma && !dbeta) return GEMM_OK;
  LnBackward p{rows, (int)cols, x, ldx, x_type,
               Q8Ref{const_cast<int8_t *>(q), ldq, const_cast<uint8_t *>(e), lde}, gamma, param_type, mean, rstd, dy,
               lddy, dy_type, dx, lddx, dx_type, dgamma, dbeta, nullptr};
  return with_scratch(reinterpret_cast<cudaStream_t>(stream), [&](const OpContext &c) -> gemm_status_t {
    if (const size_t partials = ln_backward_partials(p, c.sms)) {
      void *ws = nullptr;
      const gemm_status_t w = op_workspace(partials * sizeof(float), c.st, &ws);
      if (w != GEMM_OK) return w;
      p.partials = static_cast<float *>(ws);
    }
    int launches = 0;
    const cudaError_t err = launch_ln_backward(p, c, &launches);
    count_launches(launches);
    return launched(err);
  });
}

gemm_status_t gemm_q8_save(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                           int8_t *q, int64_t ldq, uint8_t *e, int64_t lde, gemm_stream_t stream) {
  gemm_status_t s = extents(rows, cols);
  if (s == GEMM_ERR_INVALID_ARG || !known_type(x_type)) return GEMM_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return GEMM_OK;
  if (!matrix_ok(x, x_type, ldx, cols) || !checkpoint_ok(q, ldq, e, lde, cols)) return GEMM_ERR_INVALID_ARG;
  if (s != GEMM_OK) return s;
  OpContext c;
  if ((s = op_context(reinterpret_cast<cudaStream_t>(stream), &c)) != GEMM_OK) return s;
  count_launches(1);
  return launched(launch_q8_save(x, ldx, x_type, rows, cols, Q8Ref{q, ldq, e, lde}, c.st));
}

gemm_status_t gemm_q8_restore(int64_t rows, int64_t cols, const int8_t *q, int64_t ldq, const uint8_t *e,
                              int64_t lde, void *x, int64_t ldx, int x_type, gemm_stream_t stream) {
  gemm_status_t s = extents(rows, cols);
  if (s == GEMM_ERR_INVALID_ARG || !known_type(x_type)) return GEMM_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return GEMM_OK;
  if (!matrix_ok(x, x_type, ldx, cols) || !checkpoint_ok(q, ldq, e, lde, cols)) return GEMM_ERR_INVALID_ARG;
  if (s != GEMM_OK) return s;
  OpContext c;
  if ((s = op_context(reinterpret_cast<cudaStream_t>(stream), &c)) != GEMM_OK) return s;
  count_launches(1);
  return launched(launch_q8_restore(Q8Ref{const_cast<int8_t *>(q), ldq, const_cast<uint8_t *>(e), lde}, x, ldx, x_type,
                                    rows, cols, c.st));
}

gemm_status_t gemm_q8_weight_grad(int64_t T, int64_t K, int64_t N, const int8_t *q, int64_t ldq,
                                  const uint8_t *e, int64_t lde, const uint16_t *dY, int64_t lddy,
                                  const void *base, int64_t ldbase, void *dW, int64_t ldw, int w_layout,
                                  int w_type, gemm_stream_t stream) {
  if (T < 0 || K < 0 || N < 0 || !known_type(w_type)) return GEMM_ERR_INVALID_ARG;
  if (w_layout != GEMM_B_ROW_MAJOR_KxN && w_layout != GEMM_B_COL_MAJOR_NxK) return GEMM_ERR_INVALID_ARG;
  if (K == 0 || N == 0) return GEMM_OK;
  const bool kn = w_layout == GEMM_B_ROW_MAJOR_KxN;
  const int64_t M = kn ? K : N, cols = kn ? N : K;  // dW as stored
  if (!matrix_ok(dW, w_type, ldw, cols) || (base && !matrix_ok(base, w_type, ldbase, cols)))
    return GEMM_ERR_INVALID_ARG;
  if (T > 0 && (!checkpoint_ok(q, ldq, e, lde, K) || !matrix_ok(dY, GEMM_TYPE_BF16, lddy, N)))
    return GEMM_ERR_INVALID_ARG;
  if (T > kMaxExtent || K > kMaxExtent || N > kMaxExtent ||
      ceil_div64(M, kBM) * ceil_div64(cols, 64) > kMaxExtent)
    return GEMM_ERR_UNSUPPORTED;
  const bool bf = w_type == GEMM_TYPE_BF16;
  return with_scratch(reinterpret_cast<cudaStream_t>(stream), [&](const OpContext &c) -> gemm_status_t {
    WgradParams p{};
    p.tc.M = (int)M;
    p.tc.N = (int)cols;
    p.tc.K = (int)T;
    p.tc.C = dW;
    p.tc.ldc = ldw;
    p.base = base;
    p.ldbase = ldbase;
    p.out_bf16 = bf ? 1 : 0;
    if (T == 0) {
      if (base == dW && ldbase == ldw) return GEMM_OK;
      count_launches(1);
      return launched(launch_wgrad_base(p, c.sms, c.st));
    }
    const WgradPlan pl = plan_wgrad(M, cols, T, bf ? 2 : 4, base != nullptr, c.sms, pair_slots());
    if (pl.grid <= 0) return GEMM_ERR_CUDA;
    // scratch: X restored to bf16 with 16-byte aligned rows, dY re-pitched
    // where TMA cannot read it, the split tail's partials
    const int64_t ldk = (K + 7) / 8 * 8, ldn = (N + 7) / 8 * 8;
    const bool pack = !aligned_to(dY, 16) || lddy % 8 != 0;
    const size_t x_bytes = align256((size_t)T * ldk * 2);
    const size_t g_bytes = pack ? align256((size_t)T * ldn * 2) : 0;
    void *ws = nullptr;
    const gemm_status_t s = op_workspace(x_bytes + g_bytes + wgrad_partial_bytes(pl), c.st, &ws);
    if (s != GEMM_OK) return s;
    uint8_t *xs = static_cast<uint8_t *>(ws), *gs = xs + x_bytes, *parts = gs + g_bytes;
    const Q8Ref ck{const_cast<int8_t *>(q), ldq, const_cast<uint8_t *>(e), lde};
    const bool x16 = aligned_to(q, 16) && ldq % 16 == 0;
    count_launches(1);
    uint16_t *x16s = reinterpret_cast<uint16_t *>(xs), *g16s = reinterpret_cast<uint16_t *>(gs);
    const cudaError_t staged =
        x16 && !pack ? launch_q8_restore(ck, xs, ldk, GEMM_TYPE_BF16, T, K, c.st)
                     : launch_wgrad_stage(ck, T, K, x16s, ldk, pack ? dY : nullptr, lddy, N, g16s, ldn, c.st);
    if (staged != cudaSuccess) return GEMM_ERR_CUDA;
    const void *g = pack ? (const void *)gs : dY;
    const int64_t ldg = pack ? ldn : lddy;
    WgradMaps m;
    CUtensorMap &tx = kn ? m.a : m.b, &tg = kn ? m.b : m.a;
    if (!bf16_box_map(&tx, xs, (uint64_t)K, (uint64_t)T, (uint64_t)ldk, 64, kBK) ||
        !bf16_box_map(&tg, g, (uint64_t)N, (uint64_t)T, (uint64_t)ldg, 64, kBK))
      return GEMM_ERR_CUDA;
    m.out = m.partials = m.base = tx;
    // C through TMA where its base, pitch and row ends are multiples of 16
    // bytes (a clipped TMA store would write into the row's padding), and the
    // base, read in 16-byte pieces then, likewise
    const int64_t es = bf ? 2 : 4;
    p.tc.out_tma = kOutDirect;
    if (tma_store_enabled() && aligned_to(dW, 16) && ldw * es % 16 == 0 && cols * es % 16 == 0 &&
        (!base || (aligned_to(base, 16) && ldbase * es % 16 == 0))) {
      if (!float_out_map(&m.out, bf, dW, (uint64_t)cols, (uint64_t)M, (uint64_t)ldw, 1) ||
          (base && !float_out_map(&m.base, bf, base, (uint64_t)cols, (uint64_t)M, (uint64_t)ldbase, 1)))
        return GEMM_ERR_CUDA;
      p.tc.out_tma = kOutTmaC;
    }
    p.tc.tiles_m = pl.tiles_m;
    p.tc.tiles_n = pl.tiles_n;
    p.tc.num_kb = pl.num_kb;
    p.tc.splits = 1;
    p.tc.kb_per_split = pl.num_kb;
    p.tc.group_m = 8;
    p.tc.tail_first = pl.tail_first;
    p.tc.tail_splits = pl.tail_splits;
    p.tc.tail_kb_per = pl.tail_kb_per;
    p.tc.err = c.err;
    p.tc.wait_limit_ns = c.wait_limit_ns;
    if (pl.tail_splits > 0) {
      p.tc.ws = parts;
      const int tile_m = pl.tile.pair ? 2 * kBM : kBM;
      const int64_t tail_rows = ((int64_t)pl.tiles_m * pl.tiles_n - pl.tail_first) * tile_m;
      if (!float_out_map(&m.partials, false, parts, (uint64_t)pl.tile.bn, (uint64_t)tail_rows, (uint64_t)pl.tile.bn,
                         (uint64_t)pl.tail_splits))
        return GEMM_ERR_CUDA;
    }
    count_launches(1);
    if (launch_wgrad(pl.tile, m, p, pl.grid, c.st) != cudaSuccess) return GEMM_ERR_CUDA;
    if (pl.tail_splits > 0) {
      count_launches(1);
      return launched(launch_wgrad_reduce(pl.tile, p, c.st));
    }
    return GEMM_OK;
  });
}

gemm_status_t gemm_gated_forward(int64_t T, int64_t K, int64_t F, const uint16_t *X, int64_t ldx,
                                 const uint16_t *Wg, int64_t ldwg, const uint16_t *Wu, int64_t ldwu, int w_layout,
                                 int activation, uint16_t *H, int64_t ldh, uint16_t *G, int64_t ldg, uint16_t *U,
                                 int64_t ldu, gemm_stream_t stream) {
  if (T < 0 || K < 0 || F < 0 || !known_layout(w_layout) || !known_activation(activation))
    return GEMM_ERR_INVALID_ARG;
  if (T == 0 || F == 0) return GEMM_OK;
  const bool kn = w_layout == GEMM_B_ROW_MAJOR_KxN;
  const int64_t w_cols = kn ? F : K;
  if (!bf16_ok(H, ldh, F) || !G != !U || (G && (!bf16_ok(G, ldg, F) || !bf16_ok(U, ldu, F))))
    return GEMM_ERR_INVALID_ARG;
  if (K > 0 && (!bf16_ok(X, ldx, K) || !bf16_ok(Wg, ldwg, w_cols) || !bf16_ok(Wu, ldwu, w_cols)))
    return GEMM_ERR_INVALID_ARG;
  if (T > kMaxExtent || K > kMaxExtent || F > kMaxExtent || ceil_div64(T, kBM) * ceil_div64(F, 32) > kMaxExtent)
    return GEMM_ERR_UNSUPPORTED;
  return with_scratch(reinterpret_cast<cudaStream_t>(stream), [&](const OpContext &c) -> gemm_status_t {
    const GatedForward p{T, (int)K, (int)F, X, ldx, Wg, Wu, ldwg, ldwu, !kn, activation, H, ldh, G, U, ldg, ldu};
    return gated_forward(p, c);
  });
}

gemm_status_t gemm_gated_backward(int64_t T, int64_t F, const uint16_t *dH, int64_t lddh, const uint16_t *G,
                                  int64_t ldg, const uint16_t *U, int64_t ldu, int activation, uint16_t *dG,
                                  int64_t lddg, uint16_t *dU, int64_t lddu, int8_t *q, int64_t ldq, uint8_t *e,
                                  int64_t lde, gemm_stream_t stream) {
  gemm_status_t s = extents(T, F);
  if (s == GEMM_ERR_INVALID_ARG || !known_activation(activation)) return GEMM_ERR_INVALID_ARG;
  if (T == 0 || F == 0) return GEMM_OK;
  const GatedBackward p{T, (int)F, dH, lddh, G, U, ldg, ldu, activation, dG, dU, lddg, lddu, Q8Ref{q, ldq, e, lde}};
  if (!bf16_ok(dH, lddh, F) || !gate_backward_ok(p, F)) return GEMM_ERR_INVALID_ARG;
  if (s != GEMM_OK) return s;
  OpContext c;
  if ((s = op_context(reinterpret_cast<cudaStream_t>(stream), &c)) != GEMM_OK) return s;
  count_launches(1);
  return launched(launch_gated_backward(p, c));
}

gemm_status_t gemm_gated_down_backward(int64_t T, int64_t N, int64_t F, const uint16_t *dO, int64_t lddo,
                                       const uint16_t *Wd, int64_t ldwd, int w_layout, const uint16_t *G, int64_t ldg,
                                       const uint16_t *U, int64_t ldu, int activation, uint16_t *dG, int64_t lddg,
                                       uint16_t *dU, int64_t lddu, int8_t *q, int64_t ldq, uint8_t *e, int64_t lde,
                                       gemm_stream_t stream) {
  if (T < 0 || N < 0 || F < 0 || !known_layout(w_layout) || !known_activation(activation))
    return GEMM_ERR_INVALID_ARG;
  if (T == 0 || F == 0) return GEMM_OK;
  const bool kn = w_layout == GEMM_B_ROW_MAJOR_KxN;
  const GatedBackward b{T, (int)F, nullptr, 0, G, U, ldg, ldu, activation, dG, dU, lddg, lddu, Q8Ref{q, ldq, e, lde}};
  if (!gate_backward_ok(b, F) || (N > 0 && (!bf16_ok(dO, lddo, N) || !bf16_ok(Wd, ldwd, kn ? N : F))))
    return GEMM_ERR_INVALID_ARG;
  if (T > kMaxExtent || N > kMaxExtent || F > kMaxExtent || ceil_div64(T, kBM) * ceil_div64(F, 32) > kMaxExtent)
    return GEMM_ERR_UNSUPPORTED;
  return with_scratch(reinterpret_cast<cudaStream_t>(stream), [&](const OpContext &c) -> gemm_status_t {
    if (N == 0) {
      count_launches(1);
      return launched(launch_gated_backward(b, c));
    }
    return gated_down_backward(GatedDownBackward{b, (int)N, dO, lddo, Wd, ldwd, kn}, c);
  });
}

gemm_status_t gemm_dropout_forward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                   const void *residual, int64_t ldr, void *y, int64_t ldy, int y_type, float p,
                                   uint64_t seed, uint64_t step, const uint64_t *step_device, gemm_stream_t stream) {
  return dropout(rows, cols, x, ldx, x_type, residual, ldr, y, ldy, y_type, p, seed, step, step_device, stream);
}

gemm_status_t gemm_dropout_backward(int64_t rows, int64_t cols, const void *dy, int64_t lddy, int dy_type, void *dx,
                                    int64_t lddx, int dx_type, float p, uint64_t seed, uint64_t step,
                                    const uint64_t *step_device, gemm_stream_t stream) {
  return dropout(rows, cols, dy, lddy, dy_type, nullptr, 0, dx, lddx, dx_type, p, seed, step, step_device, stream);
}

}  // extern "C"
