"""The gated delta rule without an eps: keys and queries divided by their own length alone.  Steps behind a sequence's end have no length, and nothing of theirs may reach
the others of their chunk of 64.  Inputs, tolerances and the float64 formulas are those of test_gpu_delta.py."""
import numpy as np
import pytest
import torch
from placed import DEV, down, near
from test_gpu_delta import CODE, _Call

from oracle import delta as od
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu


class _NoEps(_Call):
    def __init__(self, *size, **kw):
        super().__init__(*size, **kw)
        self.desc.eps = 0.0

    def want(self, back):
        t, B, Hk, H, dk, dv = self.size
        with np.errstate(all="ignore"):      # (the formulas divide by the lengths of steps that do not count, too)
            return od.delta(*(down(x) for x in (self.q, self.k, self.v, self.a, self.b, self.A, self.a_bias)), Hk, H, np.float32(self.scale), self.activate,
                            self.normalise, 0.0, self.lengths, down(self.h0), down(self.dy) if back else None, down(self.dh))


def _run(*size, **kw):
    c = _NoEps(*size, **kw)
    c.outputs()
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size", [(1, 2, 1, 1, 16, 16), (64, 1, 1, 1, 32, 32), (65, 2, 1, 2, 32, 48), (100, 2, 2, 2, 128, 128), (100, 2, 2, 4, 21, 13), (130, 1, 1, 1, 64, 200)])
def test_lengths_that_are_no_whole_chunks(size, dtype):
    _run(*size, dtype=dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("t,stretch,lengths", [(100, 64, [100, 0, 1, 64, 65]), (200, 128, [3, 200, 0, 127, 129])])
@pytest.mark.parametrize("dk", [24, 21])
def test_sequences_of_unequal_lengths(dk, t, stretch, lengths, dtype):
    _run(t, 5, 1, 2, dk, 40, dtype=dtype, lengths=lengths, stretch=stretch)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_segments(dtype):
    """25 chunks and more of one sequence, the last one in part; another one that ends early."""
    _run(1630, 2, 1, 1, 32, 16, dtype=dtype, lengths=[1630, 701], stretch=256)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_tokens_go_on_where_a_prompt_ended(dtype):
    """Against the formulas over all steps.  (In bf16 each is a rounding off, as everywhere.)"""
    t, more = 70, 3
    c = _NoEps(t + more, 2, 1, 2, 40, 24, dtype=dtype)
    y, h = c.want(False)
    desc = mb.make_delta_desc(t, 2, 1, 2, 40, 24, CODE[dtype], 1, 1, 64, c.scale, 0.0)
    one = mb.make_delta_desc(1, 2, 1, 2, 40, 24, CODE[dtype], 1, 1, 0, c.scale, 0.0)
    c.outputs(False)
    out, state = torch.empty((t, 2, 48), dtype=c.T, device=DEV), torch.empty_like(c.h)
    mb.mebptt_delta_forward(desc, c.q[:t], c.k[:t], c.v[:t], c.a[:t], c.b[:t], c.A, c.a_bias, None, c.h0, out, state, None, c.ws)
    near(out, y[:t], "prompt")
    token = torch.empty((2, 48), dtype=c.T, device=DEV)
    for s in range(t, t + more):
        mb.mebptt_delta_step(one, c.q[s], c.k[s], c.v[s], c.a[s], c.b[s], c.A, c.a_bias, state, None, token, state)
        near(token, y[s], "token")
    near(state, h, "state")
