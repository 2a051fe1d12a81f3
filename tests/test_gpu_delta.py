"""GPU parity of the gated delta rule with the float64 formulas, through the C ABI's binding: lengths from none to several chunks of 64 steps, sizes of one and odd
ones, heads shared by several, both types, strided and unaligned rows, sequences of none and one with NaN in what lies beyond them, states in and out
and in place, long sequences cut into segments, stretches one and several at a time, pools with sequences that have no slot.

Tolerances.  A chunk's values come out of four products one after another (the state by k, T, P or k, and back into the state), each a sum of at most 128 terms
whose operands keep 24 bits and whose roundings in 32 bits add up like a random walk: 4 sqrt(128) 2^-25 = 2^-19.5 of the terms, which T, the inverse of a
triangle of products of unit vectors, enlarges at most a few times for keys that were drawn: 2^-17 of the norm, 8 times that for a single value.  Gradients of a
come out of differences of sums over pairs of steps, added up over 64 steps: 8 times as much; their sums over all steps are measured against the sum of
magnitudes.  A gradient through the norm of q or k is what is left of one after its part along q or k is taken away, f (m - n (m.n)): each of the two
terms has been rounded, so that their sizes count and not what is left (of one value: f m eps / (x^2 + eps)).  An output of bf16 adds one rounding."""
import numpy as np
import pytest
import torch
from placed import DEV, NAN, TORCH, Placed, down, near, room, up

from oracle import delta as od
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

CODE = {"fp32": mb.FP32, "bf16": mb.BF16}
EPS = 1e-6


class _Call:
    """Inputs and outputs of one call, and what they should be."""

    def __init__(self, t, B, Hk, H, dk, dv, dtype, seed=0, layout="plain", decay=True, activate=True, normalise=True, lengths=None, state=True, stretch=64, scale=None):
        self.size, self.T, self.lengths = (t, B, Hk, H, dk, dv), TORCH[dtype], lengths
        m = self.m = Placed(seed + 31 * t + dk, layout)
        unit = 1.0 if normalise else dk ** -0.5
        T = self.T
        self.q, self.k, self.v = m.normal((t, B, Hk * dk), unit, T), m.normal((t, B, Hk * dk), unit, T), m.normal((t, B, H * dv), 1.0, T)
        if activate:
            self.b = m.normal((t, B, H), 1.0, T)
            self.a = m.normal((t, B, H), 0.5, T) if decay else None
        else:
            self.b = m.place(up(m.rng.random((t, B, H)), T))
            self.a = m.place(up(-0.2 * m.rng.random((t, B, H)), T)) if decay else None
        both = decay and activate
        self.A, self.a_bias = (up(-np.exp(m.rng.random(H) * 2.5)) if both else None), (up(m.rng.standard_normal(H) - 3.0) if both else None)
        self.h0 = up(m.rng.standard_normal((B, H, dk, dv)) * 0.3) if state else None
        self.dy, self.dh = m.normal((t, B, H * dv), 0.1, T), (up(m.rng.standard_normal((B, H, dk, dv)) * 0.1) if state else None)
        self.scale = dk ** -0.5 if scale is None else scale
        self.desc = mb.make_delta_desc(t, B, Hk, H, dk, dv, CODE[dtype], int(activate), int(normalise), stretch, self.scale, EPS)
        self.activate, self.normalise = activate, normalise
        if lengths is not None:
            for x in (self.q, self.k, self.v, self.b, self.a, self.dy):
                if x is not None:
                    for i, n in enumerate(lengths):
                        x[max(n, 0):, i] = NAN
        self.ends = None if lengths is None else up(np.asarray(lengths), torch.int32)

    def want(self, back):
        t, B, Hk, H, dk, dv = self.size
        with np.errstate(invalid="ignore"):
            return od.delta(*(down(x) for x in (self.q, self.k, self.v, self.a, self.b, self.A, self.a_bias)), Hk, H, np.float32(self.scale), self.activate,
                            self.normalise, EPS, self.lengths, down(self.h0), down(self.dy) if back else None, down(self.dh))

    def given(self):
        return self.desc, self.q, self.k, self.v, self.a, self.b, self.A, self.a_bias, self.ends, self.h0

    def outputs(self, back=True):
        t, B, Hk, H, dk, dv = self.size
        e, T = self.m.empty, self.T
        self.y, self.h = e((t, B, H * dv), T), torch.full((B, H, dk, dv), NAN, device=DEV)
        self.states = room(mb.mebptt_delta_state_bytes(self.desc)) if back else None
        self.ws = room(mb.mebptt_delta_workspace_bytes(self.desc, back))
        self.dq, self.dk, self.dv, self.db = e((t, B, Hk * dk), T), e((t, B, Hk * dk), T), e((t, B, H * dv), T), e((t, B, H), T)
        self.da = e((t, B, H), T) if self.a is not None else None
        self.dA, self.da_bias = (torch.full((H,), NAN, device=DEV) if self.A is not None else None for _ in range(2))
        self.dh0 = torch.full((B, H, dk, dv), NAN, device=DEV)

    def forward(self, **more):
        mb.mebptt_delta_forward(*self.given(), self.y, self.h, self.states, self.ws, **more)

    def backward(self, **more):
        mb.mebptt_delta_backward(*self.given(), self.dy, self.dh, self.states, self.dq, self.dk, self.dv, self.da, self.db, self.dA, self.da_bias,
                                 self.dh0, self.ws, **more)

    def check(self, back=True):
        w = self.want(back)
        near(self.y, w[0], "y")
        near(self.h, w[1], "h_out")
        if back:
            d = w[2]
            for n in ("dq", "dk", "dv", "db", "dh0"):
                near(getattr(self, n), d[n], n, d.get(n + "_terms"))
            if self.a is not None:
                near(self.da, d["da"], "da", bits=14)
            if self.A is not None:
                near(self.dA, d["dA"], "dA", d["dA_terms"], bits=14)
                near(self.da_bias, d["da_bias"], "da_bias", d["da_bias_terms"], bits=14)
        assert self.m.clean()


def _run(*size, **kw):
    c = _Call(*size, **kw)
    c.outputs()
    c.forward()
    c.backward()
    c.check()
    return c


SIZES = [(1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 5, 3), (63, 1, 1, 1, 16, 16), (64, 2, 2, 2, 32, 32), (65, 1, 1, 3, 33, 17), (130, 3, 2, 4, 128, 128), (200, 2, 1, 1, 50, 75),
         (129, 1, 3, 3, 64, 65), (70, 1, 1, 2, 127, 255), (128, 1, 1, 1, 128, 256)]


@pytest.mark.parametrize("layout", ["plain", "odd", "batch"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(size, dtype, layout):
    _run(*size, dtype, layout=layout)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kw", [dict(decay=False), dict(normalise=False), dict(activate=False), dict(activate=False, decay=False, normalise=False), dict(state=False),
                                dict(stretch=128), dict(stretch=1 << 20), dict(scale=1.0)])
def test_what_may_be_left_out(kw, dtype):
    _run(150, 2, 2, 4, 40, 24, dtype, **kw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("t,stretch,lengths", [(200, 64, [0, 1, 64, 65, 200, 199]), (200, 128, [200, 0, 128, 300, -5, 127]), (70, 64, [0, 0, 0, 1, 70, 64])])
def test_lengths(t, stretch, lengths, dtype):
    c = _run(t, 6, 1, 2, 24, 40, dtype, lengths=lengths, stretch=stretch)
    for i, n in enumerate(lengths):
        for x in (c.y, c.dq, c.dk, c.dv, c.da, c.db):
            assert not bool(x[max(n, 0):, i].any())
    assert torch.equal(c.h[0], c.h0[0]) == (lengths[0] == 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_lengths_of_rows_that_are_copied(dtype):
    _run(100, 3, 1, 2, 21, 13, dtype, lengths=[100, 65, 0])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size,kw", [((1600, 1, 1, 1, 32, 16), dict()), ((1700, 2, 1, 2, 50, 70), dict(lengths=[1700, 900])), ((1600, 1, 2, 2, 128, 128), dict(state=False)),
                                     ((2100, 1, 1, 1, 64, 64), dict(decay=False))])
def test_long_sequences_in_segments(size, kw, dtype):
    """Few sequences of 25 chunks and more: the time axis is cut.  The state behind them may be where the one before them was."""
    c = _Call(*size, dtype, stretch=256, **kw)
    c.outputs()
    c.forward()
    c.backward()
    c.check()
    if c.h0 is not None:
        y, h = c.y.clone(), c.h.clone()
        c.y.fill_(NAN)
        mb.mebptt_delta_forward(*c.given(), c.y, c.h0, None, c.ws)
        assert torch.equal(c.y, y) and torch.equal(c.h0, h)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H", [2, 4])
@pytest.mark.parametrize("some", [True, False])
def test_more_chunks_than_compute_units(some, H, dtype):
    """Workgroups that take several chunks one after another, with chunks behind a sequence's end first, last and between those with steps; and none with steps."""
    B = 90
    lengths = [0] * 9 + [int(n) for n in np.random.default_rng(4).integers(-40, 190, B - 18)] + [190] * 4 + [0] * 5 if some else [0] * B
    _run(190, B, 2, H, 20, 12, dtype, lengths=lengths, stretch=256)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size,some", [((130, 700, 1, 3, 9, 6), True), ((130, 700, 3, 3, 16, 8), False), ((4500, 16, 2, 4, 16, 8), True)])
def test_several_launches(size, some, dtype):
    """More chunks than a call holds the records of at once: the state goes from launch to launch, of whole chunks and of segments."""
    lengths = [int(n) for n in np.random.default_rng(5).integers(-20, size[0] + 60, size[1])] if some else None
    _run(*size, dtype, lengths=lengths, stretch=128)


@pytest.mark.parametrize("stretch", [64, 128, 256, 512])
def test_stretches_give_the_same_gradients(stretch):
    """Whatever is kept, and however much of it is recomputed at a time."""
    first = _run(400, 2, 1, 2, 64, 32, "bf16", stretch=1 << 20)
    c = _run(400, 2, 1, 2, 64, 32, "bf16", stretch=stretch)
    for n in ("dq", "dk", "dv", "da", "db", "dA", "da_bias", "dh0"):
        assert torch.equal(getattr(c, n), getattr(first, n)), n


def test_gradients_where_they_were():
    """dh0 over dh_out; gradients that nobody wants."""
    c = _run(90, 2, 1, 2, 20, 20, "fp32")
    want, da = c.dh0.clone(), c.da.clone()
    c.da.fill_(NAN)
    mb.mebptt_delta_backward(*c.given(), c.dy, c.dh, c.states, c.dq, c.dk, c.dv, c.da, c.db, None, None, c.dh, c.ws)
    assert torch.equal(c.dh, want) and torch.equal(c.da, da)
    mb.mebptt_delta_backward(*c.given(), c.dy, None, c.states, c.dq, c.dk, c.dv, c.da, c.db, None, c.da_bias, None, c.ws)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_no_steps_and_no_sequences(dtype):
    c = _Call(0, 2, 1, 2, 8, 8, dtype)
    c.outputs()
    c.forward()
    c.backward()
    assert torch.equal(c.h, c.h0) and torch.equal(c.dh0, c.dh) and not bool(c.dA.any()) and not bool(c.da_bias.any())
    c = _Call(5, 0, 1, 2, 8, 8, dtype)
    c.outputs()
    c.forward()
    c.backward()
    assert not bool(c.dA.any()) and not bool(c.da_bias.any())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_steps_that_forget_everything(dtype):
    """Decays of minus infinity, and so strong ones that their sums have few bits left: what stands behind them is as exact as elsewhere."""
    c = _Call(130, 1, 1, 2, 32, 32, dtype, activate=False, state=True)
    c.a[3] = -float("inf")
    c.a[40] = -5000.0
    c.a[70, :, 0] = -1e30
    c.outputs()
    c.forward()
    c.backward()
    c.a[3] = c.a[40] = c.a[70, :, 0] = -1000.0      # (the formulas' own zero)
    c.check()


def test_another_head_stays_clean():
    """A value that is not finite reaches its own head of its own sequence, and nothing behind the chunk before it."""
    c = _Call(200, 2, 2, 4, 32, 32, "bf16")
    c.v[150, 1, 32 + 5] = float("inf")      # head 1 of sequence 1
    c.outputs()
    c.forward()
    c.backward()
    y = c.y.view(200, 2, 4, 32)
    assert bool(y[:128].isfinite().all()) and bool(y[:, 0].isfinite().all()) and bool(y[:, 1, [0, 2, 3]].isfinite().all())
    assert not bool(y[150:, 1, 1, 5].isfinite().any()) and bool(c.dq[:, 0].isfinite().all()) and bool(c.dv.view(200, 2, 4, 32)[:, 1, [0, 2, 3]].isfinite().all())


def test_gradients_against_differences():
    """The forward call itself, in 32 bits, along random directions."""
    c = _run(140, 1, 1, 2, 24, 24, "fp32", decay=True)
    loss = lambda: float((c.y.double() * c.dy.double()).sum() + (c.h.double() * c.dh.double()).sum())  # noqa: E731
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    for x, d in ((c.q, c.dq), (c.k, c.dk), (c.v, c.dv), (c.a, c.da), (c.b, c.db), (c.A, c.dA), (c.a_bias, c.da_bias), (c.h0, c.dh0)):
        way = torch.randn(x.shape, generator=g, device=DEV)
        way *= 1e-2 * x.norm() / way.norm()
        want, old = float((d.double() * way.double()).sum()), x.clone()
        got = 0.0
        for s in (1, -1):
            x.copy_(old + s * way)
            c.forward()
            got += s * loss() / 2
        x.copy_(old)
        # a step of 1 % of the norm: the third derivative's share is about 1e-4 of the gradient's size along it
        assert abs(got - want) <= 3e-3 * (abs(want) + float(d.norm() * way.norm()) * 0.05), (got, want)


# ---- single tokens ---------------------------------------------------------------------------------


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,Hk,H,dk,dv,kw", [(1, 1, 1, 1, 1, {}), (3, 2, 4, 20, 24, {}), (2, 1, 2, 128, 128, {}), (2, 1, 1, 37, 51, dict(decay=False)), (1, 2, 2, 128, 256, {}),
                                             (2, 1, 3, 64, 64, dict(normalise=False)), (2, 1, 1, 100, 250, dict(activate=False))])
def test_single_tokens(B, Hk, H, dk, dv, kw, dtype, layout):
    c = _Call(1, B, Hk, H, dk, dv, dtype, layout=layout, state=True, **kw)
    slots = B + 2
    pool, index = torch.randn((slots, H, dk, dv), device=DEV), torch.randperm(slots, device=DEV)[:B].to(torch.int32)
    pool[index.long()] = c.h0
    out, y = torch.full_like(pool, 7.0), c.m.empty((B, H * dv), c.T)
    row = lambda x: None if x is None else x[0]  # noqa: E731
    args = (c.desc, row(c.q), row(c.k), row(c.v), row(c.a), row(c.b), c.A, c.a_bias)
    mb.mebptt_delta_step(*args, pool, index, y, out)
    want_y, want_h = c.want(False)
    near(y, want_y[0], "y")
    near(out[index.long()], want_h, "state")
    rest = [i for i in range(slots) if i not in index.tolist()]
    assert bool((out[rest] == 7.0).all()) and c.m.clean()
    # in place; a sequence without a slot
    before, first = pool.clone(), y.clone()
    index[0] = -1 if B % 2 else slots
    mb.mebptt_delta_step(*args, pool, index, y, pool)
    assert not bool(y[0].any()) and torch.equal(y[1:], first[1:])
    for b in range(1, B):
        assert torch.equal(pool[int(index[b])], out[int(index[b])])
    others = [i for i in range(slots) if i not in index[1:].tolist()]
    assert torch.equal(pool[others], before[others])
    # by their own number
    mb.mebptt_delta_step(*args, c.h0, None, y, c.h0)
    near(c.h0, want_h, "state")


def test_tokens_go_on_where_a_prompt_ended():
    c = _Call(100, 2, 1, 2, 48, 40, "fp32")
    c.outputs()
    c.forward()
    short = mb.make_delta_desc(90, 2, 1, 2, 48, 40, mb.FP32, 1, 1, 64, c.scale, EPS)
    cut = lambda x: x[:90]  # noqa: E731
    y, h = torch.empty((90, 2, 80), device=DEV), torch.empty_like(c.h)
    mb.mebptt_delta_forward(short, cut(c.q), cut(c.k), cut(c.v), cut(c.a), cut(c.b), c.A, c.a_bias, None, c.h0, y, h, None, c.ws)
    near(y, down(c.y[:90]), "prompt")
    one = mb.make_delta_desc(1, 2, 1, 2, 48, 40, mb.FP32, 1, 1, 0, c.scale, EPS)
    out = torch.empty((2, 80), device=DEV)
    for s in range(90, 100):
        mb.mebptt_delta_step(one, c.q[s], c.k[s], c.v[s], c.a[s], c.b[s], c.A, c.a_bias, h, None, out, h)
        near(out, down(c.y[s]), "token")
    near(h, down(c.h), "state")


# ---- streams and graphs ----------------------------------------------------------------------------


def test_another_stream_and_a_graph():
    c = _run(300, 2, 1, 2, 64, 64, "bf16", lengths=[300, 170])
    names = ("y", "h", "dq", "dk", "dv", "da", "db", "dA", "da_bias", "dh0")
    want = {n: getattr(c, n).clone() for n in names}

    def wipe():
        for n in names:
            getattr(c, n).fill_(NAN)
        c.ws.fill_(0xFF)
        c.states.fill_(0xFF)
    side = torch.cuda.Stream()
    wipe()
    side.wait_stream(torch.cuda.current_stream())
    c.forward(stream=side.cuda_stream)
    c.backward(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(getattr(c, n), want[n]) for n in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for _ in range(3):
        wipe()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(c, n), want[n]) for n in names)
    v = c.v.clone()
    c.v.mul_(0.5)
    graph.replay()
    half = {n: getattr(c, n).clone() for n in names}
    wipe()
    c.forward()
    c.backward()
    assert all(torch.equal(getattr(c, n), half[n]) for n in names) and not torch.equal(half["y"], want["y"])
    c.v.copy_(v)


def test_inputs_still_on_their_way():
    """Inputs written on the call's own stream just before it."""
    c = _Call(200, 2, 1, 2, 32, 32, "bf16")
    c.outputs()
    side = torch.cuda.Stream()
    q = c.q.clone()
    c.q.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        c.q.copy_(q)
        c.forward()
        c.backward()
    side.synchronize()
    c.check()
