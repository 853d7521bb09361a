"""A pre-norm projection block in training, on the library's calls only:

    y = layer_norm(x) * gamma + beta,    o = y . W        (forward)
    dy = do . W^T,  dW += y^T . do,  dx, dgamma, dbeta    (backward)

Between the two passes the block holds no activation in full: x and y stay as
8-bit checkpoints (1.03 bytes a value instead of 2 or 4), which the backward
pass reads directly -- the weight gradient multiplies y's, the layer norm's
gradient takes x's.

    python -m paper_2512_13282_gb300.projection_block [--tokens T --width K --out N --steps S]

trains a block towards a fixed random one of the same shape and prints the
loss, the time of a step and the bytes held between the passes.
"""
from __future__ import annotations

import argparse

import torch

from . import gemm as G
from . import layer as L

_TYPE = {torch.float32: L.GEMM_TYPE_F32, torch.bfloat16: L.GEMM_TYPE_BF16}


def _pitch(x, rows, cols, device, types=tuple(_TYPE)):
    """Elements from one row of x to the next, for the library, which takes
    addresses and sizes on trust: ValueError unless x is rows x cols of one of
    the types on the device, with contiguous rows that do not overlap."""
    if tuple(x.shape) != (rows, cols) or x.dtype not in types or x.device != device:
        raise ValueError(f"expected {rows} x {cols} of {' or '.join(map(str, types))} on {device}, "
                         f"got {tuple(x.shape)} of {x.dtype} on {x.device}")
    if (cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols):
        raise ValueError(f"expected contiguous rows, got strides {x.stride()} of {tuple(x.shape)}")
    return x.stride(0) if rows > 1 else cols


class Checkpoint:
    """An activation held in 8 bits on the device (see gb300_layer.h)."""

    def __init__(self, rows, cols, device="cuda"):
        self.rows, self.cols = rows, cols
        self.q = torch.empty((rows, cols), dtype=torch.int8, device=device)
        self.e = torch.empty((rows, -(-cols // L.GEMM_Q8_BLOCK)), dtype=torch.uint8, device=device)

    @property
    def args(self):
        return self.q, self.q.stride(0), self.e, self.e.stride(0)

    @property
    def nbytes(self):
        return self.q.numel() + self.e.numel()

    def save(self, x):
        ld = _pitch(x, self.rows, self.cols, self.q.device)
        L.check(L.gemm_q8_save(self.rows, self.cols, x, ld, _TYPE[x.dtype], *self.args))
        return self

    def restore(self, dtype=torch.bfloat16):
        if dtype not in _TYPE:
            raise ValueError(f"restores to {' or '.join(map(str, _TYPE))}, not {dtype}")
        x = torch.empty((self.rows, self.cols), dtype=dtype, device=self.q.device)
        L.check(L.gemm_q8_restore(self.rows, self.cols, *self.args, x, self.cols, _TYPE[dtype]))
        return x


class ProjectionBlock:
    """Parameters, float32 gradients (accumulated until ``zero_grad``) and the
    two passes.  x may be bf16 or float32 (a residual stream); W is bf16,
    K x N row-major.  A pass raises ValueError for a tensor of another shape,
    type or device, or without contiguous rows."""

    def __init__(self, width, out, generator=None, eps=1e-5):
        dev = dict(device="cuda", generator=generator)
        self.width, self.out, self.eps = width, out, eps
        self.gamma = torch.ones(width, device="cuda")
        self.beta = torch.zeros(width, device="cuda")
        self.weight = (torch.randn((width, out), **dev) / width ** 0.5).to(torch.bfloat16)
        self.dgamma, self.dbeta = torch.zeros_like(self.gamma), torch.zeros_like(self.beta)
        self.dweight = torch.zeros((width, out), device="cuda")
        self._held = None

    def zero_grad(self):
        for g in (self.dgamma, self.dbeta, self.dweight):
            g.zero_()

    def forward(self, x):
        T, K, N, dev = x.shape[0], self.width, self.out, self.weight.device
        ldx = _pitch(x, T, K, dev)
        y = torch.empty((T, K), dtype=torch.bfloat16, device=dev)
        mean, rstd = (torch.empty(T, device=dev) for _ in range(2))
        cx, cy = Checkpoint(T, K, dev).save(x), Checkpoint(T, K, dev)
        L.check(L.gemm_layernorm_forward(T, K, x, ldx, _TYPE[x.dtype], self.gamma, self.beta,
                                         L.GEMM_TYPE_F32, self.eps, y, K, L.GEMM_TYPE_BF16, mean, rstd, *cy.args))
        o = torch.empty((T, N), dtype=torch.bfloat16, device=dev)
        G.check(G.gemm_bf16_f32acc_bf16(T, N, K, y, K, self.weight, N, G.GEMM_B_ROW_MAJOR_KxN, o, N))
        self._held = (cx, cy, mean, rstd, x.dtype)
        return o

    @property
    def held_bytes(self):
        """Bytes kept for the backward pass."""
        cx, cy, mean, rstd, _ = self._held
        return cx.nbytes + cy.nbytes + 4 * (mean.numel() + rstd.numel())

    def backward(self, do):
        """dx of the last forward pass (of x's type) from do, a row for each of
        its rows, bf16; adds to the gradients."""
        if self._held is None:
            raise RuntimeError("backward takes what a forward pass holds, once")
        cx, cy, mean, rstd, dtype = self._held
        T, K, N, dev = cx.rows, self.width, self.out, self.weight.device
        lddo = _pitch(do, T, N, dev, (torch.bfloat16,))
        # do . W^T: W as stored (K x N) is the transposed factor N x K, column-major
        dy = torch.empty((T, K), dtype=torch.bfloat16, device=dev)
        G.check(G.gemm_bf16_f32acc_bf16(T, K, N, do, lddo, self.weight, N, G.GEMM_B_COL_MAJOR_NxK, dy, K))
        L.check(L.gemm_q8_weight_grad(T, K, N, *cy.args, do, lddo, self.dweight, N, self.dweight, N,
                                      L.GEMM_B_ROW_MAJOR_KxN, L.GEMM_TYPE_F32))
        dx = torch.empty((T, K), dtype=dtype, device=dev)
        dgamma, dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        L.check(L.gemm_layernorm_backward(T, K, None, 0, L.GEMM_TYPE_F32, *cx.args, self.gamma, L.GEMM_TYPE_F32, mean,
                                          rstd, dy, K, L.GEMM_TYPE_BF16, dx, K, _TYPE[dtype], dgamma, dbeta))
        self.dgamma += dgamma
        self.dbeta += dbeta
        self._held = None
        return dx


def train(tokens, width, out, steps, report=print):
    """Losses of `steps` steps of plain gradient descent towards a fixed block."""
    # X^T X / tokens of normalised rows has eigenvalues up to about
    # (1 + sqrt(width / tokens))^2; the step stays below their inverse
    lr = 0.8 / (1 + (width / tokens) ** 0.5) ** 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    teacher, block = ProjectionBlock(width, out, gen), ProjectionBlock(width, out, gen)
    master = block.weight.float()
    losses = []
    for step in range(steps):
        x = torch.randn((tokens, width), device="cuda", generator=gen).to(torch.bfloat16)
        target = teacher.forward(x)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        block.zero_grad()
        o = block.forward(x)
        held = block.held_bytes
        diff = o.float() - target.float()
        block.backward((diff * (2 / (tokens * out))).to(torch.bfloat16))
        # the loss averages over N outputs, its gradients scale with 1 / N
        master -= lr * out * block.dweight
        block.gamma -= lr * block.dgamma
        block.beta -= lr * block.dbeta
        block.weight.copy_(master)
        end.record()
        losses.append(float(diff.square().mean()))
        report(f"step {step:3d}  loss {losses[-1]:.5f}  {start.elapsed_time(end):7.3f} ms  held between the passes "
               f"{held / 2**20:.1f} MiB (in full: {(2 * 2 * tokens * width) / 2**20:.1f} MiB)")
    G.check(G.gemm_device_status())
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--out", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    train(a.tokens, a.width, a.out, a.steps)


if __name__ == "__main__":
    main()
