"""The gated delta rule with inputs of bf16: what has 32 bits on the way (the products of queries and keys, of gradients and values, the values themselves) keeps 24 of them in the matrix
products.  Seen where a result is what little is left of terms that cancel: a step's y is a sum of four products, dq of two, that were chosen to add up to
next to nothing, so that the rounding of the result itself is next to nothing too.

Tolerances, relative to the terms' sizes.  An operand of three bf16 parts is exact to 2^-26; what is left out of a product of two of them is another 2^-26.  Each term has been
rounded up to four times on its way (its factors, beta, R), each of its six products of parts is added with one more rounding: ten independent ones of 2^-24 at
most, 2^-25.8 in the mean square, make 2^-24.1; a factor of four for how the matrix unit orders its sums: 2^-22 in the mean square, 2^-20 for one.  With 16 bits each operand
alone would be off by 2^-18, 2^-19.6 in the mean square."""
import numpy as np
import pytest
import torch
from placed import DEV, down, room, up

from oracle import delta as od
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _round(x):
    return up(x, BF16).double().cpu().numpy()


def _cancel(rng, d):
    """Four coefficients in bf16 whose sum of products with d [.., 4] is next to nothing; the first is drawn."""
    c = np.zeros_like(d)
    c[..., 0] = _round(rng.uniform(1, 2, d.shape[:-1]))
    for j in (1, 2, 3):
        c[..., j] = _round(-(c[..., :j] * d[..., :j]).sum(-1) / d[..., j])
    return c


def _call(q, k, v, b, dy, scale):
    """(y, dq) of one head without decay, norms and a state before."""
    t, B, dk = q.shape
    dv = v.shape[2]
    desc = mb.make_delta_desc(t, B, 1, 1, dk, dv, mb.BF16, 0, 0, 64, scale)
    ins = [up(x, BF16) for x in (q, k, v, b, dy)]
    outs = [torch.empty_like(ins[i]) for i in (2, 0, 1, 2, 3)]       # y, dq, dk, dv, db
    states, ws = room(mb.mebptt_delta_state_bytes(desc)), room(mb.mebptt_delta_workspace_bytes(desc, True))
    q, k, v, b, dy = ins
    mb.mebptt_delta_forward(desc, q, k, v, None, b, None, None, None, None, outs[0], None, states, ws)
    mb.mebptt_delta_backward(desc, q, k, v, None, b, None, None, None, None, dy, None, states, *outs[1:4], None, outs[4], None, None, None, ws)
    want_y, _, d = od.delta(*(down(x) for x in (q, k, v)), None, down(b), None, None, 1, 1, np.float32(scale), False, False, 0.0, dy=down(dy))
    return down(outs[0]), want_y, down(outs[1]), d["dq"]


def _close(got, want, terms):
    err = np.maximum(np.abs(got - want) - 2.0 ** -8 * np.abs(want), 0) / terms
    assert (np.abs(want) < 2.0 ** -14 * terms).mean() > 0.9        # (they do cancel)
    assert np.sqrt((err ** 2).mean()) <= 2.0 ** -22 and err.max() <= 2.0 ** -20, (np.log2(np.sqrt((err ** 2).mean())), np.log2(err.max()))


@pytest.mark.parametrize("B", [2, 150])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 48), (64, 128)])
def test_y_of_terms_that_cancel(dk, dv, B):
    """Keys are unit vectors, each at right angles to those of 31 steps before it, so that step i answers with the values of steps i - 3 .. i, one by one."""
    rng, t, scale = np.random.default_rng(dk + dv + B), 32, 0.7
    k = np.zeros((t, B, dk))
    k[np.arange(t), :, np.arange(t)] = 1.0
    v, b = _round(rng.uniform(1, 2, (t, B, dv)) * rng.choice([-1, 1], (t, B, dv))), _round(rng.uniform(0.5, 1, (t, B, 1)))
    q, rows, cols = np.zeros((t, B, dk)), np.arange(3, t), np.arange(3, t) % dv
    U = (b * v)[rows[:, None] - np.arange(4), :, cols[:, None]]         # [rows, 4, B]
    c = _cancel(rng, U.transpose(0, 2, 1))
    for j in range(4):
        q[rows, :, rows - j] = c[..., j]
    y, want, _, _ = _call(q, k, v, b, np.zeros((t, B, dv)), scale)
    terms = scale * np.abs(c * U.transpose(0, 2, 1)).sum(-1)
    _close(y[rows, :, cols], want[rows, :, cols], terms)


@pytest.mark.parametrize("B", [2, 150])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 48), (128, 128)])
def test_dq_of_terms_that_cancel(dk, dv, B):
    """Steps 2 p and 2 p + 1 have keys along one axis, so that dq along it is a difference of two products of dy and values."""
    rng, t, scale = np.random.default_rng(dk + dv + B), 48, 0.7
    k, p, axis = np.zeros((t, B, dk)), np.arange(t // 2), np.arange(t // 2)
    other = _round(rng.uniform(0.5, 1, (t // 2, B)))
    k[2 * p, :, axis], k[2 * p + 1, :, axis] = 1.0, -other
    v, b = _round(rng.uniform(1, 2, (t, B, dv)) * rng.choice([-1, 1], (t, B, dv))), _round(rng.uniform(0.5, 1, (t, B, 1)))
    first = b[2 * p] * v[2 * p]                                          # beta R of each pair
    second = b[2 * p + 1] * (v[2 * p + 1] + other[..., None] * first)
    D = first - other[..., None] * second
    dy, i = np.zeros((t, B, dv)), np.arange(2, t)
    at = (i - 2) // 2                                                     # step i looks at the pair before its own
    for s, pair in zip(i, at):
        dy[s, :, :4] = _cancel(rng, D[pair][:, :4])
    _, _, dq, want = _call(np.zeros((t, B, dk)), k, v, b, dy, scale)
    # (the products that dP's two values are sums of: each has been rounded, also where the sum is smaller)
    terms = scale * (np.abs(dy[i, :, :4] * first[at][..., :4]).sum(-1) + np.abs(dy[i, :, :4] * second[at][..., :4]).sum(-1) * np.abs(other[at]))
    _close(dq[i, :, axis[at]], want[i, :, axis[at]], terms)
