"""A pre-norm gated feed-forward block in training, on the library's calls:

    n = layer_norm(x) * gamma + beta,   G = n . Wg,  U = n . Wu,
    H = act(G) * U,   y = x + dropout(H . Wd)                       (forward)
    do = dropout'(dy),  dH = do . Wd^T,  dG = dH * U * act'(G),  dU = dH * act(G),
    dWd += H^T . do,  dW += n^T . [dG dU],  dn = [dG dU] . W^T,
    dx = dy + layer_norm'(dn)                                       (backward)

with W = [Wg Wu].  Between the two passes the block holds G and U in bf16 and
x and n as 8-bit checkpoints; H comes back from G and U as a checkpoint, which
Wd's gradient multiplies, dH never leaves the kernel that takes it, dG and dU
are written over G and U, and dropout's mask is drawn again instead of stored.

    python -m paper_2512_13282_gb300.feed_forward_block [--tokens T --width K --hidden F --act silu --drop P --steps S]

trains a block towards a fixed random one of the same shape and prints the
loss, the time of a step and the bytes held between the passes.
"""
from __future__ import annotations

import argparse

import torch

from . import gemm as G
from . import layer as L
from .projection_block import _TYPE, Checkpoint, _pitch, _read_here

ACTIVATIONS = {"silu": L.GEMM_ACT_SILU, "gelu": L.GEMM_ACT_GELU, "gelu_tanh": L.GEMM_ACT_GELU_TANH,
               "relu": L.GEMM_ACT_RELU}
_BF16 = torch.bfloat16


def _drawn(step):
    """Dropout's step arguments: a number, and what is added to it on the device."""
    return step if isinstance(step, tuple) else (step, None)


class FeedForwardBlock:
    """Parameters, float32 gradients (accumulated until ``zero_grad``) and the
    two passes.  x and y are bf16 or float32 (a residual stream); the weights
    are bf16, row-major: W is width x 2 hidden (Wg, then Wu), Wd hidden x width.
    ``drop`` is dropout's share, ``seed`` its key: one drawn after the weights
    if none is given, so that blocks drop apart from one another (processes
    whose generators are alike, as those of one set of weights are, need seeds).
    Each forward pass draws with the next ``step``, each replay of a captured one
    too.  A pass raises ValueError for a tensor of another shape, type or device,
    or without contiguous rows.  The backward pass may run on another stream, one
    that waits for the forward pass."""

    # The next step is _start, which passes count up on the host; from the first
    # captured pass on it is _start + _word, and all passes count the word up on
    # the device, as replays do.  (That takes two launches: 30 us of an eager
    # forward pass of few tokens, 73 without.)
    _start, _word, _counted = 0, None, False
    _home = None  # the last forward pass's stream

    def __init__(self, width, hidden, act="silu", drop=0.0, generator=None, eps=1e-5, seed=None):
        if act not in ACTIVATIONS or not 0 <= drop < 1:
            raise ValueError(f"an activation of {', '.join(ACTIVATIONS)} and a share in [0, 1), not {act} and {drop}")
        dev = dict(device="cuda", generator=generator)
        self.width, self.hidden, self.act, self.drop, self.eps = width, hidden, act, drop, eps
        self.gamma = torch.ones(width, device="cuda")
        self.beta = torch.zeros(width, device="cuda")
        self.weight = (torch.randn((width, 2 * hidden), **dev) / width ** 0.5).to(_BF16)
        self.down = (torch.randn((hidden, width), **dev) / hidden ** 0.5).to(_BF16)
        self.seed = int(torch.randint(2 ** 63 - 1, (), **dev)) if seed is None else seed
        self.dgamma, self.dbeta = torch.zeros_like(self.gamma), torch.zeros_like(self.beta)
        self.dweight = torch.zeros((width, 2 * hidden), device="cuda")
        self.ddown = torch.zeros((hidden, width), device="cuda")
        self._word = torch.zeros((), dtype=torch.int64, device="cuda")
        self._held = None

    def _on_device(self):
        """Whether steps are counted on the device."""
        if self._word is not None and not self._counted:
            self._counted = torch.cuda.is_current_stream_capturing()
        return self._counted

    @property
    def step(self):
        """The step of the next forward pass, modulo 2^64.  Reading it waits for
        the device once a pass has been captured; set within a capture, it is set
        by every replay."""
        return (self._start + (int(self._word) if self._counted else 0)) % 2 ** 64

    @step.setter
    def step(self, value):
        if self._on_device():
            self._word.fill_((value - self._start + 2 ** 63) % 2 ** 64 - 2 ** 63)
        else:
            self._start = value % 2 ** 64

    def zero_grad(self):
        for g in (self.dgamma, self.dbeta, self.dweight, self.ddown):
            g.zero_()

    def forward(self, x):
        T, K, F, dev = x.shape[0], self.width, self.hidden, self.weight.device
        ldx = _pitch(x, T, K, dev)
        n = torch.empty((T, K), dtype=_BF16, device=dev)
        mean, rstd = (torch.empty(T, device=dev) for _ in range(2))
        cx, cn = Checkpoint(T, K, dev).save(x), Checkpoint(T, K, dev)
        L.check(L.gemm_layernorm_forward(T, K, x, ldx, _TYPE[x.dtype], self.gamma, self.beta, L.GEMM_TYPE_F32,
                                         self.eps, n, K, L.GEMM_TYPE_BF16, mean, rstd, *cn.args))
        gu, h = torch.empty((T, 2 * F), dtype=_BF16, device=dev), torch.empty((T, F), dtype=_BF16, device=dev)
        L.check(L.gemm_gated_forward(T, K, F, n, K, self.weight, 2 * F, self.weight[:, F:], 2 * F,
                                     L.GEMM_B_ROW_MAJOR_KxN, ACTIVATIONS[self.act], h, F, gu, 2 * F, gu[:, F:], 2 * F))
        o, y = torch.empty((T, K), dtype=_BF16, device=dev), torch.empty((T, K), dtype=x.dtype, device=dev)
        G.check(G.gemm_bf16_f32acc_bf16(T, K, F, h, F, self.down, K, G.GEMM_B_ROW_MAJOR_KxN, o, K))
        # this pass's step, and its backward pass's
        step = (self._start, self._word.clone()) if self._on_device() else self._start
        L.check(L.gemm_dropout_forward(T, K, o, K, L.GEMM_TYPE_BF16, x, ldx, y, K, _TYPE[x.dtype], self.drop, self.seed,
                                       *_drawn(step)))
        self._held, self._home = (cx, cn, mean, rstd, gu, x.dtype, step), G._stream(None)
        if self._counted:
            self._word += 1
        else:
            self._start += 1
        return y

    @property
    def held_bytes(self):
        """Bytes kept for the backward pass."""
        cx, cn, mean, rstd, gu, _, _ = self._held
        return cx.nbytes + cn.nbytes + 4 * (mean.numel() + rstd.numel()) + 2 * gu.numel()

    def backward(self, dy):
        """dx of the last forward pass from dy, a row for each of its rows, both
        of x's type; adds to the gradients."""
        if self._held is None:
            raise RuntimeError("backward takes what a forward pass holds, once")
        cx, cn, mean, rstd, gu, dtype, step = self._held
        T, K, F, dev = cx.rows, self.width, self.hidden, self.weight.device
        lddy = _pitch(dy, T, K, dev, (dtype,))
        self._held = None  # G and U are written over: held once, also by a pass that fails
        _read_here((cx.q, cx.e, cn.q, cn.e, mean, rstd, gu, _drawn(step)[1]), self._home)
        do = torch.empty((T, K), dtype=_BF16, device=dev)
        L.check(L.gemm_dropout_backward(T, K, dy, lddy, _TYPE[dtype], do, K, L.GEMM_TYPE_BF16, self.drop, self.seed,
                                        *_drawn(step)))
        ch = Checkpoint(T, F, dev)
        L.check(L.gemm_gated_down_backward(T, K, F, do, K, self.down, K, L.GEMM_B_ROW_MAJOR_KxN, gu, 2 * F, gu[:, F:],
                                           2 * F, ACTIVATIONS[self.act], gu, 2 * F, gu[:, F:], 2 * F, *ch.args))
        L.check(L.gemm_q8_weight_grad(T, F, K, *ch.args, do, K, self.ddown, K, self.ddown, K, L.GEMM_B_ROW_MAJOR_KxN,
                                      L.GEMM_TYPE_F32))
        L.check(L.gemm_q8_weight_grad(T, K, 2 * F, *cn.args, gu, 2 * F, self.dweight, 2 * F, self.dweight, 2 * F,
                                      L.GEMM_B_ROW_MAJOR_KxN, L.GEMM_TYPE_F32))
        # [dG dU] . W^T: W as stored is the transposed factor, column-major
        dn = torch.empty((T, K), dtype=_BF16, device=dev)
        G.check(G.gemm_bf16_f32acc_bf16(T, K, 2 * F, gu, 2 * F, self.weight, 2 * F, G.GEMM_B_COL_MAJOR_NxK, dn, K))
        # layer_norm'(dn) stays float32 until dy has been added (dropout's call with a
        # share of 0 is that sum), so that a bf16 dx is rounded once
        dl = torch.empty((T, K), device=dev)
        dgamma, dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        L.check(L.gemm_layernorm_backward(T, K, None, 0, L.GEMM_TYPE_F32, *cx.args, self.gamma, L.GEMM_TYPE_F32, mean,
                                          rstd, dn, K, L.GEMM_TYPE_BF16, dl, K, L.GEMM_TYPE_F32, dgamma, dbeta))
        self.dgamma += dgamma
        self.dbeta += dbeta
        dx = dl if dtype == torch.float32 else torch.empty((T, K), dtype=dtype, device=dev)
        L.check(L.gemm_dropout_forward(T, K, dl, K, L.GEMM_TYPE_F32, dy, lddy, dx, K, _TYPE[dtype], 0.0, 0, 0))
        return dx


def train(tokens, width, hidden, steps, act="silu", drop=0.0, report=print):
    """Losses of `steps` steps of gradient descent towards a fixed block."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    teacher = FeedForwardBlock(width, hidden, act, 0.0, gen, seed=0)
    block = FeedForwardBlock(width, hidden, act, drop, gen, seed=0)
    masters = [block.weight.float(), block.down.float()]
    losses = []
    for step in range(steps):
        x = torch.randn((tokens, width), device="cuda", generator=gen).to(_BF16)
        target = teacher.forward(x)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        block.zero_grad()
        y = block.forward(x)
        held = block.held_bytes
        diff = y.float() - target.float()
        block.backward((diff * (2 / tokens)).to(_BF16))
        # steps of a fixed length per weight, as the gradients' scale changes with the shape
        for master, grad, weight in zip(masters, (block.dweight, block.ddown), (block.weight, block.down)):
            master -= 0.1 * master.norm() / grad.norm().clamp(min=1e-20) * grad
            weight.copy_(master)
        end.record()
        losses.append(float(diff.square().mean()))
        report(f"step {step:3d}  loss {losses[-1]:.5f}  {start.elapsed_time(end):7.3f} ms  held between the passes "
               f"{held / 2**20:.1f} MiB (in full: {2 * tokens * (2 * width + 3 * hidden) / 2**20:.1f} MiB)")
    G.check(G.gemm_device_status())
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=11008)
    ap.add_argument("--act", choices=ACTIVATIONS, default="silu")
    ap.add_argument("--drop", type=float, default=0.1)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    train(a.tokens, a.width, a.hidden, a.steps, a.act, a.drop)


if __name__ == "__main__":
    main()
