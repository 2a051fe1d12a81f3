"""A residual block around the selective scan, trained and served with the library's operators.

    r += x;  n = norm(r);  [z | v | B | C | delta] = n W_in^T;  [u | B | C] = conv([v | B | C]);
    y = scan(u, delta, A, B, C) * silu(z);  out = norm(y) W_out^T       (out is the next block's x)

A gradient step keeps the residual stream in 32 bits and everything else in bf16, the scan's states of every `stretch`-th step
only; its two projections are plain matrix products.  Serving takes the projections in 8-bit integers, the norms in front of them writing
their rows in 8 bits with a scale each; prompts of unequal lengths, then single tokens on a pool of states.

``python -m paper_1606_03401_amd.selective`` trains a small block on a synthetic task, quantises it and serves it.
"""
from __future__ import annotations

import dataclasses
import time
from typing import Optional

import torch

from . import binding as mb
from .optimiser import AdamW

EPS = 1e-5


@dataclasses.dataclass
class Sizes:
    width: int          # of the residual stream
    inner: int          # channels of the scan
    N: int = 16         # states per channel
    groups: int = 1     # groups of channels that share B and C
    taps: int = 4
    stretch: int = 64

    @property
    def shared(self) -> int:
        return self.groups * self.N

    @property
    def mixed(self) -> int:
        """Channels of the convolution: v, B and C."""
        return self.inner + 2 * self.shared

    @property
    def projected(self) -> int:
        return 2 * self.inner + self.mixed


def make_weights(s: Sizes, seed: int = 0, device: str = "cuda:0") -> dict:
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *shape, k: torch.randn(shape, generator=g, device=device) * k  # noqa: E731
    first = torch.exp(torch.empty(s.inner, device=device).uniform_(-6.9, -2.3, generator=g))     # steps of 0.001 to 0.1
    return {"norm": torch.ones(s.width, device=device), "W_in": normal(s.projected, s.width, k=s.width ** -0.5),
            "conv": normal(s.mixed, s.taps, k=s.taps ** -0.5), "conv_bias": torch.zeros(s.mixed, device=device),
            "A": -torch.arange(1, s.N + 1, device=device, dtype=torch.float32).repeat(s.inner, 1),
            "skip": torch.ones(s.inner, device=device), "delta_bias": torch.log(torch.expm1(first)),
            "norm_out": torch.ones(s.inner, device=device), "W_out": normal(s.width, s.inner, k=s.inner ** -0.5)}


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


class Training:
    """Forward and backward of one block at fixed sizes; buffers are allocated once."""

    def __init__(self, s: Sizes, t: int, B: int, device: str = "cuda:0"):
        self.s, self.t, self.B = s, t, B
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=device)  # noqa: E731
        M, f32 = t * B, torch.float32
        self.norm = mb.make_norm_desc(M, s.width, mb.BF16, mb.FP32, mb.BF16, EPS)
        self.norm_out = mb.make_norm_desc(M, s.inner, mb.BF16, mb.BF16, mb.BF16, EPS)
        self.conv = mb.make_conv_desc(t, B, s.mixed, s.taps, mb.BF16, 1)
        self.scan = mb.make_scan_desc(t, B, s.inner, s.N, s.groups, mb.BF16, 1, s.stretch)
        self.r, self.n, self.rstd = new(M, s.width, dtype=f32), new(M, s.width), new(M, dtype=f32)
        self.p, self.c, self.y = new(t, B, s.projected), new(t, B, s.mixed), new(t, B, s.inner)
        self.m, self.rstd_out = new(M, s.inner), new(M, dtype=f32)
        self.dy, self.dc, self.dp = new(t, B, s.inner), new(t, B, s.mixed), new(t, B, s.projected)
        self.dx, self.dr = new(M, s.width), new(M, s.width, dtype=f32)
        self.states = _bytes(mb.mebptt_scan_state_bytes(self.scan), device)
        self.ws = _bytes(max(mb.mebptt_scan_workspace_bytes(self.scan, True), mb.mebptt_conv_workspace_bytes(self.conv),
                             mb.mebptt_norm_workspace_bytes(self.norm), mb.mebptt_norm_workspace_bytes(self.norm_out)), device)

    def _split(self, p):
        """z, [v | B | C] and delta as column blocks of the projection, read and written in place."""
        return p[..., :self.s.inner], p[..., self.s.inner:self.s.inner + self.s.mixed], p[..., self.s.inner + self.s.mixed:]

    def _conv_split(self, c):
        """u, B and C as column blocks of the convolution's output."""
        D, S = self.s.inner, self.s.shared
        return c[..., :D], c[..., D:D + S], c[..., D + S:]

    def forward(self, w: dict, x, residual):
        """x [t, B, width] bf16 and the residual stream [t, B, width] float32 -> out [t, B, width] bf16; the new residual stream is self.r."""
        s, M = self.s, self.t * self.B
        mb.mebptt_norm_forward(self.norm, x.reshape(M, s.width), residual.reshape(M, s.width), w["norm"], self.n, None, self.r, self.rstd)
        torch.mm(self.n, w["W_in"].bfloat16().t(), out=self.p.view(M, s.projected))
        z, mixed, delta = self._split(self.p)
        mb.mebptt_conv_forward(self.conv, mixed, w["conv"], w["conv_bias"], None, None, self.c)
        u, Bm, Cm = self._conv_split(self.c)
        mb.mebptt_scan_forward(self.scan, u, delta, w["A"], Bm, Cm, w["skip"], z, w["delta_bias"], None, None, self.y, None, self.states, self.ws)
        mb.mebptt_norm_forward(self.norm_out, self.y.view(M, s.inner), None, w["norm_out"], self.m, None, None, self.rstd_out)
        return torch.mm(self.m, w["W_out"].bfloat16().t()).view(self.t, self.B, s.width)

    def backward(self, w: dict, dout, dr_out=None):
        """dout: gradient of `out`, dr_out: of the new residual stream (None: zero).  Returns (gradients of the weights, dx bf16, dresidual
        float32)."""
        s, M = self.s, self.t * self.B
        g = {k: torch.empty_like(v) for k, v in w.items()}
        dout = dout.reshape(M, s.width)
        g["W_out"] = torch.mm(dout.t(), self.m).float()
        dm = torch.mm(dout, w["W_out"].bfloat16())
        y, dy = self.y.view(M, s.inner), self.dy.view(M, s.inner)
        mb.mebptt_norm_backward(self.norm_out, y, w["norm_out"], self.rstd_out, dm, None, dy, None, g["norm_out"], self.ws)
        z, mixed, delta = self._split(self.p)
        dz, dmixed, ddelta = self._split(self.dp)
        u, Bm, Cm = self._conv_split(self.c)
        du, dB, dC = self._conv_split(self.dc)
        mb.mebptt_scan_backward(self.scan, u, delta, w["A"], Bm, Cm, w["skip"], z, w["delta_bias"], None, None, self.dy, None, self.states,
                                du, ddelta, g["A"], dB, dC, g["skip"], dz, g["delta_bias"], None, self.ws)
        mb.mebptt_conv_backward(self.conv, mixed, w["conv"], w["conv_bias"], None, None, self.dc, None, dmixed, g["conv"], g["conv_bias"], None,
                                self.ws)
        dp = self.dp.view(M, s.projected)
        g["W_in"] = torch.mm(dp.t(), self.n).float()
        dn = torch.mm(dp, w["W_in"].bfloat16())
        mb.mebptt_norm_backward(self.norm, self.r, w["norm"], self.rstd, dn, None if dr_out is None else dr_out.reshape(M, s.width), self.dx,
                                self.dr, g["norm"], self.ws)
        shape = (self.t, self.B, s.width)
        return g, self.dx.view(shape), self.dr.view(shape)


def quantise(w: torch.Tensor):
    """(8-bit rows, their scales) of a weight matrix."""
    scale = w.abs().amax(1) / 127.0
    return torch.round(w / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.int8), scale


class Serving:
    """One block with 8-bit projections: prompts, then single tokens of sequences whose states live in a pool of `slots`."""

    def __init__(self, s: Sizes, w: dict, slots: int, device: str = "cuda:0"):
        self.s, self.w, self.dev = s, w, device
        (self.W_in, self.s_in), (self.W_out, self.s_out) = quantise(w["W_in"]), quantise(w["W_out"])
        # a row behind the pool's last slot takes the states of sequences that have none
        self._conv_rows = torch.zeros((slots + 1, s.taps - 1, s.mixed), dtype=torch.bfloat16, device=device)
        self._scan_rows = torch.zeros((slots + 1, s.inner, s.N), device=device)
        self.slots, self.conv_states, self.scan_states = slots, self._conv_rows[:slots], self._scan_rows[:slots]
        self.kept = {}

    def _buffers(self, t: int, B: int) -> dict:
        """What a call of these sizes needs."""
        s, M, f32 = self.s, t * B, torch.float32
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=self.dev)  # noqa: E731
        k = {"norm": mb.make_norm_desc(M, s.width, mb.BF16, mb.FP32, mb.INT8, EPS), "norm_out": mb.make_norm_desc(M, s.inner, mb.BF16, mb.BF16, mb.INT8, EPS),
             "product": mb.make_int8_desc(M, s.projected, s.width, mb.BF16), "product_out": mb.make_int8_desc(M, s.width, s.inner, mb.BF16),
             "conv": mb.make_conv_desc(t, B, s.mixed, s.taps, mb.BF16, 1), "scan": mb.make_scan_desc(t, B, s.inner, s.N, s.groups, mb.BF16, 1),
             "n": new(M, s.width, dtype=torch.int8), "n_scale": new(M, dtype=f32), "r": new(M, s.width, dtype=f32), "p": new(t, B, s.projected),
             "c": new(t, B, s.mixed), "y": new(t, B, s.inner), "m": new(M, s.inner, dtype=torch.int8), "m_scale": new(M, dtype=f32),
             "out": new(M, s.width)}
        k["ws"] = _bytes(max(mb.mebptt_scan_workspace_bytes(k["scan"], False), mb.mebptt_int8_workspace_bytes(k["product"]),
                             mb.mebptt_int8_workspace_bytes(k["product_out"])), self.dev)
        return k

    def _in(self, k: dict, x, residual):
        s, w = self.s, self.w
        M = x.numel() // s.width
        mb.mebptt_norm_forward(k["norm"], x.reshape(M, s.width), residual.reshape(M, s.width), w["norm"], k["n"], k["n_scale"], k["r"])
        mb.mebptt_int8_product(k["product"], k["n"], k["n_scale"], self.W_in, self.s_in, None, k["p"].view(M, s.projected), k["ws"])
        D = s.inner
        p, c = k["p"], k["c"]
        return (p[..., :D], p[..., D:D + s.mixed], p[..., D + s.mixed:]), (c[..., :D], c[..., D:D + s.shared], c[..., D + s.shared:])

    def _out(self, k: dict, shape):
        s, w = self.s, self.w
        M = k["out"].shape[0]
        mb.mebptt_norm_forward(k["norm_out"], k["y"].view(M, s.inner), None, w["norm_out"], k["m"], k["m_scale"])
        mb.mebptt_int8_product(k["product_out"], k["m"], k["m_scale"], self.W_out, self.s_out, None, k["out"], k["ws"])
        return k["out"].view(shape), k["r"].view(shape)

    def prompt(self, x, residual, index, lengths=None):
        """x, residual [t, B, width]; sequence b starts in slot index[b]; one whose index is no slot is passed over (its out is zero).  Returns (out,
        the new residual stream), the caller's own: prompts come in any length, so nothing is kept of a call."""
        t, B, _ = x.shape
        s, k, w = self.s, self._buffers(t, B), self.w
        conv_last = torch.empty((B, s.taps - 1, s.mixed), dtype=torch.bfloat16, device=self.dev)
        h = torch.empty((B, s.inner, s.N), device=self.dev)
        there = (index >= 0) & (index < self.slots)
        lengths = torch.where(there, t if lengths is None else lengths, 0).to(torch.int32)
        (z, mixed, delta), (u, Bm, Cm) = self._in(k, x, residual)
        mb.mebptt_conv_forward(k["conv"], mixed, w["conv"], w["conv_bias"], lengths, None, k["c"], conv_last)
        mb.mebptt_scan_forward(k["scan"], u, delta, w["A"], Bm, Cm, w["skip"], z, w["delta_bias"], lengths, None, k["y"], h, None, k["ws"])
        at = torch.where(there, index, self.slots).long()
        self._conv_rows[at], self._scan_rows[at] = conv_last, h
        return self._out(k, x.shape)

    def token(self, x, residual, index: Optional[torch.Tensor] = None):
        """x, residual [B, width], one token each; a sequence whose index is no slot is passed over.  Returns (out, the new residual stream):
        buffers of this object, made once per batch size and stream, so that a captured call finds them in place."""
        B, w = x.shape[0], self.w
        key = (B, torch.cuda.current_stream(self.dev).cuda_stream)
        if key not in self.kept:
            self.kept[key] = self._buffers(1, B)
        k = self.kept[key]
        (z, mixed, delta), (u, Bm, Cm) = self._in(k, x, residual)
        mb.mebptt_conv_step(k["conv"], mixed[0], w["conv"], w["conv_bias"], self.conv_states, index, k["c"][0], self.conv_states)
        mb.mebptt_scan_step(k["scan"], u[0], delta[0], w["A"], Bm[0], Cm[0], w["skip"], z[0], w["delta_bias"], self.scan_states, index, k["y"][0],
                            self.scan_states)
        return self._out(k, x.shape)


def train(s: Sizes, t: int, B: int, steps: int, rate: float = 0.3, seed: int = 0, adamw: int = 0):
    """Gradient descent on a task that needs memory: out of a step is to be the input of eight steps before.  adamw 32 or 8: AdamW instead, with states of so many
    bits.  Returns (weights, the losses)."""
    w = make_weights(s, seed)
    run, losses = Training(s, t, B), []
    if adamw:
        into = {k: torch.empty_like(v) for k, v in w.items()}
        opt = AdamW(list(w.values()), list(into.values()), rate, bits=adamw, clip=1.0, no_decay=[not k.startswith("W") for k in w], seed=seed)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed + 1)
    for _ in range(steps):
        x = torch.randn((t, B, s.width), generator=g, device="cuda:0").bfloat16()
        target = torch.zeros_like(x)
        target[8:] = x[:-8]
        out = run.forward(w, x, torch.zeros_like(x, dtype=torch.float32))
        err = out.float() - target.float()
        losses.append(float((err * err).mean()))
        grads, _, _ = run.backward(w, (2.0 / err.numel() * s.width * err).bfloat16())
        if adamw:
            for k, v in grads.items():
                into[k].copy_(v)
            opt.step()
        else:
            for k, v in grads.items():
                w[k] -= rate * v / (1.0 + v.norm())
        w["A"].clamp_(max=-1e-3)
    return w, losses


def main() -> None:
    s = Sizes(width=256, inner=512, N=16)
    t0 = time.time()
    w, losses = train(s, t=256, B=32, steps=60)
    print(f"trained 60 steps of 256 x 32 in {time.time() - t0:.1f} s: loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    B, t, more = 6, 48, 8
    serve = Serving(s, w, slots=B)
    x = torch.randn((t + more, B, s.width), device="cuda:0").bfloat16()
    zero = torch.zeros_like(x, dtype=torch.float32)
    index = torch.arange(B, dtype=torch.int32, device="cuda:0")
    whole = serve.prompt(x, zero, index)[0].clone()
    serve.prompt(x[:t], zero[:t], index)
    worst = 0.0
    for i in range(t, t + more):
        out, _ = serve.token(x[i], zero[i], index)
        worst = max(worst, float((out.float() - whole[i].float()).abs().max() / whole.float().abs().max()))
    print(f"8 tokens after a prompt of {t} differ from a prompt of {t + more} by {worst:.1e} of the largest value")


if __name__ == "__main__":
    main()
