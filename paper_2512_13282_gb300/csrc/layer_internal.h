// layer_internal.h -- host-side declarations of the layer operators
// (layer_api.cu, layer_ln_fwd.cu, layer_ln_bwd.cu, layer_q8.cu,
// wgrad.cu); not part of the public ABI.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "gb300_layer.h"
#include "gemm_internal.h"

namespace gb300 {

constexpr int kQ8Block = GEMM_Q8_BLOCK;

// A checkpoint: signed bytes q (pitch ldq) and block exponents e (pitch lde).
struct Q8Ref {
  int8_t *q;
  int64_t ldq;
  uint8_t *e;
  int64_t lde;
};

struct LnForward {
  int64_t rows;
  int cols;
  const void *x;
  int64_t ldx;
  int x_type;
  const void *gamma, *beta;  // either may be null: ones, zeros
  int param_type;
  float eps;
  void *y;
  int64_t ldy;
  int y_type;
  float *mean, *rstd;  // either may be null
  Q8Ref ck;            // checkpoint of y, or ck.q null
};
cudaError_t launch_ln_forward(const LnForward &p, const OpContext &c);

struct LnBackward {
  int64_t rows;
  int cols;
  const void *x;  // null: x is read from ck
  int64_t ldx;
  int x_type;     // of x; where x is null, of nothing
  Q8Ref ck;
  const void *gamma;  // null: ones
  int param_type;
  const float *mean, *rstd;
  const void *dy;
  int64_t lddy;
  int dy_type;
  void *dx;
  int64_t lddx;
  int dx_type;
  float *dgamma, *dbeta;  // either may be null
  float *partials;        // ln_backward_partials() floats, or null
};
// Floats of workspace a backward pass wants for its partial parameter
// gradients (0: it computes none, or has no partial ones).
size_t ln_backward_partials(const LnBackward &p, int sms);
// *launches is increased by the kernels launched.
cudaError_t launch_ln_backward(const LnBackward &p, const OpContext &c, int *launches);

cudaError_t launch_q8_save(const void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols, const Q8Ref &ck,
                           cudaStream_t st);
cudaError_t launch_q8_restore(const Q8Ref &ck, void *x, int64_t ldx, int x_type, int64_t rows, int64_t cols,
                              cudaStream_t st);

// Operands of the weight gradient that TMA cannot read as they are, in one
// launch: the checkpoint restored to bf16 (T x K at x, pitch ldx) and, where g
// is not null, the T x N bf16 matrix g copied to gx (pitch ldgx); x and gx have
// 16-byte aligned rows, the sources any alignment (wgrad.cu).
cudaError_t launch_wgrad_stage(const Q8Ref &ck, int64_t T, int64_t K, uint16_t *x, int64_t ldx, const uint16_t *g,
                               int64_t ldg, int64_t N, uint16_t *gx, int64_t ldgx, cudaStream_t st);

// C[m][n] = base[m][n] + sum_t A[t][m] * B[t][n] with bf16 A (T x M) and B
// (T x N), both read with their rows (t) outermost (wgrad.cu).
struct WgradParams {
  TcParams tc;  // M, N, K = T; tiling, split tail, C, ldc, partials, error word
  const void *base;  // null: none
  int64_t ldbase;
  int out_bf16;      // type of C and base
};
// A compiled tile shape of the kernel.
struct WgradTile {
  bool pair;  // a CTA pair per 256-row tile (256 wide), or one CTA per 128-row tile
  int bn;     // tile width: 256, or 128 or 64
};
// Tile shape, split tail and grid for an M x N result of out_bytes each summed
// over T rows, with or without a base to read: the least modelled time.
struct WgradPlan {
  WgradTile tile;
  int tiles_m, tiles_n, num_kb;
  int tail_first, tail_splits, tail_kb_per;
  int grid;
};
WgradPlan plan_wgrad(int64_t M, int64_t N, int64_t T, int out_bytes, bool base, int sms, int pairs);
// Bytes of partial sums a plan's split tail writes (0: none).
size_t wgrad_partial_bytes(const WgradPlan &pl);
// Tensor maps of its operands; out and base where C goes through TMA, partials
// with a split tail (any valid map else).
struct WgradMaps {
  CUtensorMap a, b, out, partials, base;
};
cudaError_t launch_wgrad(const WgradTile &tile, const WgradMaps &m, const WgradParams &p, int grid, cudaStream_t st);
// T == 0: C = base, or zero.
cudaError_t launch_wgrad_base(const WgradParams &p, int sms, cudaStream_t st);
// The split tail's tiles: partials summed in split order, base added, rounded
// and stored.
cudaError_t launch_wgrad_reduce(const WgradTile &tile, const WgradParams &p, cudaStream_t st);

}  // namespace gb300
