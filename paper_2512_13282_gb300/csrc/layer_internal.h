// layer_internal.h -- host-side declarations of the layer operators
// (layer_api.cu, layer_ln_fwd.cu, layer_ln_bwd.cu, layer_q8.cu, wgrad.cu,
// layer_gate.cu, gated_*.cu, layer_dropout.cu); not part of the public ABI.
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

// Gated feed-forward block (layer_gate.cu).  T x F matrices of bf16.
struct GatedForward {
  int64_t T;
  int K, F;
  const uint16_t *x;
  int64_t ldx;
  const uint16_t *wg, *wu;
  int64_t ldwg, ldwu;
  bool w_kmajor;  // W's k index contiguous
  int act;
  uint16_t *h;
  int64_t ldh;
  uint16_t *g, *u;  // both null: not kept
  int64_t ldg, ldu;
};
// Within with_scratch().
gemm_status_t gated_forward(const GatedForward &p, const OpContext &c);

struct GatedBackward {
  int64_t T;
  int F;
  const uint16_t *dh;  // null: zero
  int64_t lddh;
  const uint16_t *g, *u;
  int64_t ldg, ldu;
  int act;
  uint16_t *dg, *du;  // may be g, u
  int64_t lddg, lddu;
  Q8Ref ck;  // checkpoint of act(g) * u, or ck.q null
};
cudaError_t launch_gated_backward(const GatedBackward &p, const OpContext &c);
// dh = dO . Wd^T over N columns; b.dh is not used.
struct GatedDownBackward {
  GatedBackward b;
  int N;
  const uint16_t *d;
  int64_t ldd;
  const uint16_t *w;
  int64_t ldw;
  bool w_kmajor;  // Wd's n index contiguous
};
gemm_status_t gated_down_backward(const GatedDownBackward &p, const OpContext &c);

// The tensor-core kernel of both (gated_tc.cuh).
struct GatedTcParams {
  int T, F;  // rows, features
  int tiles_m, tiles_n, num_kb, group_m;
  // split tail, as in TcParams: the tiles from raster position tail_first on are
  // split into tail_splits (0: none) ranges of tail_kb_per k-blocks, whose sums
  // go to ws (float32): plane s has tile i's block of tile rows x bn words at row
  // i * tile rows, pitch bn
  int tail_first, tail_splits, tail_kb_per;
  float *ws;
  int act;
  // forward: out[0] = H, out[1], out[2] = G, U or null; backward: out[0], out[1]
  // = dG, dU.  vec: their rows, and gate's and up's, start on 16 bytes and are
  // whole 16-byte pieces.
  uint16_t *out[3];
  int64_t ldout[3];
  int vec;
  const uint16_t *gate, *up;  // backward: G, U
  int64_t ldgate, ldup;
  Q8Ref ck;     // backward: or ck.q null
  int q_align;  // its rows start on 16 or 8 bytes, or (1) anywhere
  uint32_t *err;
  uint64_t wait_limit_ns;
};
// A compiled tile shape: bn columns of the accumulator (forward: bn / 2
// features, each with its gate and up value).
struct GatedTile {
  bool pair;  // a CTA pair per 256-row tile, or one CTA per 128-row tile
  int bn;     // 256 (pair), 128, or 64 (backward)
};
// Tensor maps: X or dO; Wg and Wu, or Wd twice.
struct GatedMaps {
  CUtensorMap a, b[2];
};
cudaError_t launch_gated_tc_fwd(const GatedTile &tile, bool km, const GatedMaps &m, const GatedTcParams &p, int grid,
                                cudaStream_t st);
// The kernel of at most kFewTokens tokens (gated_few.cu): X or dO in boxes of 64
// x gated_few_columns(T), each weight in boxes of 64 x 64.
constexpr int kFewTokens = 64;
int gated_few_columns(int64_t T);
cudaError_t launch_gated_few(bool forward, bool km, const GatedMaps &m, const GatedTcParams &p, int sms,
                             cudaStream_t st);
cudaError_t launch_gated_tc_bwd(const GatedTile &tile, bool km, const GatedMaps &m, const GatedTcParams &p, int grid,
                                cudaStream_t st);
// The split tail's tiles: partial sums added in split order, then as the kernel
// does (gated_tail.cu).
cudaError_t launch_gated_tail(const GatedTile &tile, bool forward, const GatedTcParams &p, cudaStream_t st);

// Dropout (layer_dropout.cu), forward or backward (without a residual).
struct Dropout {
  int64_t rows, cols;
  const void *x;
  int64_t ldx;
  int x_type;
  const void *residual;  // null: none
  int64_t ldr;
  void *y;
  int64_t ldy;
  int y_type;
  uint32_t threshold;  // numbers below it are dropped, 0 .. 65536
  uint64_t seed, step;
  const uint64_t *step_device;  // null: none
};
cudaError_t launch_dropout(const Dropout &p, cudaStream_t st);

}  // namespace gb300
