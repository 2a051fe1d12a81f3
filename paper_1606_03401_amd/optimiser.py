"""AdamW over all tensors of a model, however many, in one launch (and two for the norm of all gradients), with its states in 32 or 8 bits.

Owns the states and what the library's calls need; every tensor and gradient stays where it is, so that a step can be captured into a graph.  Rate and
step count live on the GPU: set `rate` between steps (or replays), the count goes on by itself.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as mb


class AdamW:
    """params float32, grads float32 or bfloat16 (written by the caller before each step); copies: bfloat16 tensors that receive the new
    parameters (entries may be None); no_decay: truth values; clip: limit of the norm of all gradients together."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], rate: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, decay: float = 0.01, bits: int = 32, clip: Optional[float] = None, copies=None, no_decay=None, seed: int = 0):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        params, dev = list(params), params[0].device
        self.bits, self.clip = bits, clip
        kind = torch.uint8 if bits == 8 else torch.float32
        self.m, self.v = ([torch.zeros(p.shape, dtype=kind, device=dev) for p in params] for _ in range(2))
        scales = lambda: [torch.zeros(-(-p.numel() // 256), device=dev) for p in params] if bits == 8 else None  # noqa: E731
        self.m_scale, self.v_scale = scales(), scales()
        self.tensors = mb.make_adamw_tensors(params, grads, self.m, self.v, self.m_scale, self.v_scale, copies, no_decay)
        room = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device=dev)  # noqa: E731
        self.table, self.ws = room(mb.mebptt_adamw_table_bytes(self.tensors)), room(mb.mebptt_adamw_workspace_bytes(self.tensors))
        self.desc = mb.make_adamw_desc(rate, beta1, beta2, eps, decay, 1, seed)
        self.rate = torch.full((1,), rate, device=dev)
        self.count = torch.zeros(1, dtype=torch.int64, device=dev)
        self.norm = torch.zeros(2, device=dev)          # of the last step's gradients, and the factor that limited it
        mb.mebptt_adamw_prepare(self.tensors, self.table)

    def step(self) -> None:
        """One step on the current stream.  With a clip, gradients whose norm is not finite change nothing, and the step does not count."""
        if self.clip is not None:
            mb.mebptt_adamw_norm(self.tensors, self.table, self.clip, self.norm, self.ws)
            self.count += self.norm[1:] == self.norm[1:]        # (the factor is NaN then)
        else:
            self.count += 1
        mb.mebptt_adamw_step(self.desc, self.tensors, self.table, self.norm[1:] if self.clip is not None else None, self.rate, self.count)

    def states(self):
        """(m, v) of every tensor in float32, to be looked at.  A checkpoint keeps what steps go on from, as it is: `m`, `v`, `m_scale`, `v_scale` and `count`, copied into a new object's."""
        if self.bits == 32:
            return [m.clone() for m in self.m], [v.clone() for v in self.v]

        def wide(codes, scale, signed):
            out = torch.empty(codes.shape, device=codes.device)
            mb.mebptt_adamw_unpack(codes, scale, signed, out)
            return out
        return [wide(*x, True) for x in zip(self.m, self.m_scale)], [wide(*x, False) for x in zip(self.v, self.v_scale)]
