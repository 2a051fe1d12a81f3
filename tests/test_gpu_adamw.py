"""GPU parity of AdamW over many tensors with the float64 formulas, through the C ABI's binding: tensors of none, one and odd numbers of values, at any alignment, states
in 32 and 8 bits side by side, gradients of both types, factors that are not finite, rates and steps read on the GPU, captured and replayed.

Tolerances.  A new state: three roundings of 2^-24 each of its terms, 2^-22 of the larger one.  A parameter: its update is off by a few roundings of what m's
terms would make of it, and the sum by one, 2^-21 of the parameter and that together.  A code of 8 bits is one of the two neighbours of a value that is itself off by 2^-22 and of a scale
off by 2^-23: what it stands for lies between them, 2^-20 more to either side."""
import numpy as np
import pytest
import torch
from placed import DEV, NAN, TORCH, down, room, up

from oracle import delta as od
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

SIZES = [1, 7, 255, 256, 257, 0, 1000, 4095, 4096, 4097, 12345, 33]
SET = dict(rate=1e-2, beta1=0.9, beta2=0.98, eps=1e-8, decay=0.1, step=3, seed=77)


class _Tensors:
    """Lists of tensors in buffers with room between them, 0xFF where nobody is to write."""

    def __init__(self, sizes, grad="fp32", bits=32, copy=True, shift=0, seed=0, no_decay=None):
        rng = self.rng = np.random.default_rng(seed)
        self.sizes, self.bits, self.outer = sizes, bits, []
        s = lambda n: 10.0 ** rng.uniform(-4, 0, n)  # noqa: E731

        def place(a, dtype):
            t = up(a, dtype)
            size = t.numel() * t.element_size()
            b = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
            at = 16 + shift * t.element_size()
            view = b[at:at + size].view(dtype)
            view.copy_(t)
            self.outer.append((b, at, size))
            return view
        f32 = torch.float32
        self.p = [place(rng.standard_normal(n), f32) for n in sizes]
        self.g = [place(rng.standard_normal(n) * s(n), TORCH[grad]) for n in sizes]
        blocks = [-(-n // 256) for n in sizes]
        if bits == 32:
            self.m, self.v = [place(rng.standard_normal(n) * s(n), f32) for n in sizes], [place(s(n) ** 2, f32) for n in sizes]
            self.ms = self.vs = None
        else:
            self.m, self.v = ([place(rng.integers(0, 256, n), torch.uint8) for n in sizes] for _ in range(2))
            self.ms, self.vs = ([place(s(n), f32) for n in blocks] for _ in range(2))
        self.copies = [place(np.zeros(n), torch.bfloat16) for n in sizes] if copy else None
        self.flags = no_decay or [False] * len(sizes)
        self.args = mb.make_adamw_tensors(self.p, self.g, self.m, self.v, self.ms, self.vs, self.copies, self.flags)
        self.table = room(mb.mebptt_adamw_table_bytes(self.args))
        mb.mebptt_adamw_prepare(self.args, self.table)

    def state(self):
        """(p, g, m, v) of every tensor in 64 bits."""
        if self.bits == 32:
            return [tuple(down(x[i]) for x in (self.p, self.g, self.m, self.v)) for i in range(len(self.sizes))]
        return [(down(self.p[i]), down(self.g[i]), od.values8(self.m[i].cpu().numpy(), down(self.ms[i]), True), od.values8(self.v[i].cpu().numpy(), down(self.vs[i]), False))
                for i in range(len(self.sizes))]

    def clean(self):
        return all(bool((b[:at] == 0xFF).all()) and bool((b[at + n:] == 0xFF).all()) for b, at, n in self.outer)


def _check(t, before, factor=1.0, **kw):
    h = {**SET, **kw}
    for i, (p, g, m, v) in enumerate(before):
        decay = 0.0 if t.flags[i] else h["decay"]
        want_p, want_m, want_v = od.adamw(p, g * factor, m, v, h["rate"], h["beta1"], h["beta2"], h["eps"], decay, h["step"])
        got = down(t.p[i])
        terms_m, terms_v = np.abs(h["beta1"] * m) + np.abs((1 - h["beta1"]) * g * factor), want_v
        # the two terms of m may nearly cancel; their roundings stay
        move = h["rate"] * terms_m / (1 - h["beta1"] ** h["step"]) / (np.sqrt(want_v / (1 - h["beta2"] ** h["step"])) + h["eps"])
        assert (np.abs(got - want_p) <= 2.0 ** -21 * (np.abs(p) + move) + 1e-30).all(), i
        if t.copies is not None:
            assert torch.equal(t.copies[i], t.p[i].to(torch.bfloat16))
        if t.bits == 32:
            assert (np.abs(down(t.m[i]) - want_m) <= 2.0 ** -22 * terms_m + 1e-38).all(), i
            assert (np.abs(down(t.v[i]) - want_v) <= 2.0 ** -22 * terms_v + 1e-38).all(), i
            continue
        for codes, scale, want, terms, signed in ((t.m[i], t.ms[i], want_m, terms_m, True), (t.v[i], t.vs[i], want_v, terms_v, False)):
            if not want.size:
                continue
            top, low, high = od.neighbours8(want, signed)
            assert (np.abs(down(scale) - top) <= 2.0 ** -20 * np.maximum(top, np.pad(terms, (0, -terms.size % 256)).reshape(-1, 256).max(1))).all()
            got = od.values8(codes.cpu().numpy(), down(scale), signed)
            slack = 2.0 ** -20 * np.maximum(np.abs(high), terms) + 1e-38
            assert (got >= np.minimum(low, high) - slack).all() and (got <= np.maximum(low, high) + slack).all(), i
    assert t.clean()


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_step(bits, grad, shift):
    t = _Tensors(SIZES, grad, bits, shift=shift, no_decay=[i % 3 == 0 for i in range(len(SIZES))])
    before = t.state()
    mb.mebptt_adamw_step(mb.make_adamw_desc(**SET), t.args, t.table)
    _check(t, before)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    rng = np.random.default_rng(3)
    t = _Tensors([int(n) for n in rng.integers(0, 600, 130)] + [70000], "bf16", bits, copy=False)
    before = t.state()
    mb.mebptt_adamw_step(mb.make_adamw_desc(**SET), t.args, t.table)
    _check(t, before)


def test_states_from_nothing():
    """States of zeros, a first step; a gradient of zeros leaves them so."""
    for bits in (32, 8):
        t = _Tensors([300, 300], bits=bits)
        for x in t.m + t.v + (t.ms + t.vs if bits == 8 else []):
            x.zero_()
        t.g[1].zero_()
        before = t.state()
        mb.mebptt_adamw_step(mb.make_adamw_desc(**{**SET, "step": 1}), t.args, t.table)
        _check(t, before, step=1)
        assert not bool(t.m[1].any()) and not bool(t.v[1].any())


def test_the_mean_is_kept():
    """Many steps of a v that changes by less than a code's step each time: rounded to the nearest it would never move.  4096 values of one
    start and one gradient: after 200 steps their mean has gone where 64 bits go, within four deviations of a mean of so many (each step's rounding
    adds at most a quarter of a step squared: 200 (1/8)^2 / 4 of the value squared, times the share that moves, 0.02 / (1/8))."""
    n, steps, beta2 = 4096, 200, 0.98
    t = _Tensors([n], bits=8)
    t.p[0].zero_()
    t.g[0].fill_(1.0)
    t.m[0].zero_()
    t.v[0].fill_((31 << 3) - 8 * 2)           # 1/4 of the scale
    t.ms[0].zero_()
    t.vs[0].fill_(1.0)
    want = 0.25
    for k in range(steps):
        mb.mebptt_adamw_step(mb.make_adamw_desc(rate=0.0, beta1=0.9, beta2=beta2, decay=0.0, step=k + 1, seed=5), t.args, t.table)
        want = beta2 * want + (1 - beta2)
    got = od.values8(t.v[0].cpu().numpy(), down(t.vs[0]), False).mean()
    assert abs(got - want) <= 4 * np.sqrt(200 / 256 * 0.16) / np.sqrt(n) * want + 1e-3, (got, want)


def test_the_same_call_gives_the_same_bits_and_another_step_others():
    runs = []
    for step in (3, 3, 4):
        t = _Tensors([5000], bits=8, seed=9)
        mb.mebptt_adamw_step(mb.make_adamw_desc(**{**SET, "step": step}), t.args, t.table)
        runs.append(t)
    a, b, c = runs
    assert torch.equal(a.m[0], b.m[0]) and torch.equal(a.v[0], b.v[0]) and torch.equal(a.p[0], b.p[0])
    assert 0.2 < float((a.m[0] != c.m[0]).float().mean()) < 0.8


@pytest.mark.parametrize("bits", [32, 8])
def test_factors(bits):
    t = _Tensors(SIZES, bits=bits)
    before = t.state()
    f = torch.tensor([0.25], device=DEV)
    mb.mebptt_adamw_step(mb.make_adamw_desc(**SET), t.args, t.table, f)
    _check(t, before, factor=0.25)
    for bad in (NAN, float("inf")):
        f.fill_(bad)
        old = [x.clone() for x in t.p + t.m + t.v]
        mb.mebptt_adamw_step(mb.make_adamw_desc(**SET), t.args, t.table, f)
        assert all(torch.equal(x, y) for x, y in zip(t.p + t.m + t.v, old))


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm(grad, shift):
    t = _Tensors(SIZES + [500000], grad, shift=shift)
    out, ws = torch.full((2,), NAN, device=DEV), room(mb.mebptt_adamw_workspace_bytes(t.args))
    norm = np.sqrt(sum((down(g) ** 2).sum() for g in t.g))
    for limit in (0.5 * norm, 2.0 * norm, float("inf")):
        mb.mebptt_adamw_norm(t.args, t.table, limit, out, ws)
        got = out.tolist()
        assert abs(got[0] - norm) <= 2.0 ** -23 * norm and abs(got[1] - min(1.0, limit / norm)) <= 2.0 ** -22
    t.g[0].fill_(1e30)                       # its square leaves fp32
    mb.mebptt_adamw_norm(t.args, t.table, 1.0, out, ws)
    assert abs(out[0].item() / 1e30 - (1 if grad == "fp32" else float(torch.tensor(1e30).bfloat16()) / 1e30)) < 1e-3 and 0 < out[1].item() < 2e-30
    for bad in (NAN, float("inf")):
        t.g[3][5] = bad
        mb.mebptt_adamw_norm(t.args, t.table, 1.0, out, ws)
        assert not np.isfinite(out[0].item()) and np.isnan(out[1].item())
    none = _Tensors([0])
    mb.mebptt_adamw_norm(none.args, none.table, 1.0, out, ws)
    assert out.tolist() == [0.0, 1.0]


@pytest.mark.parametrize("signed", [True, False])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [0, 1, 255, 256, 1000, 70001])
def test_unpack(n, dtype, signed):
    rng = np.random.default_rng(n)
    codes, scale = up(rng.integers(0, 256, n), torch.uint8), up(10.0 ** rng.uniform(-3, 3, -(-n // 256)))
    out = torch.full((n + 1,), NAN, dtype=TORCH[dtype], device=DEV)
    mb.mebptt_adamw_unpack(codes, scale, signed, out[:n])
    want = od.values8(codes.cpu().numpy(), down(scale), signed)
    assert torch.equal(out[:n], up(np.asarray(want, np.float32)).to(TORCH[dtype])) and bool(out[n].isnan())


def test_a_captured_step_goes_on():
    """Rate and step are read when the step runs: a replayed graph is a training loop's body."""
    a, b = (_Tensors([1000, 77], bits=8, seed=4) for _ in range(2))
    rate, step = torch.zeros(1, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    norm, ws = torch.zeros(2, device=DEV), room(mb.mebptt_adamw_workspace_bytes(a.args))
    desc = mb.make_adamw_desc(**SET)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.mebptt_adamw_norm(a.args, a.table, 1.0, norm, ws)
        mb.mebptt_adamw_step(desc, a.args, a.table, norm[1:], rate, step)
    for k in range(1, 4):
        rate.fill_(0.01 / k)
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        mb.mebptt_adamw_norm(b.args, b.table, 1.0, norm, ws)
        mb.mebptt_adamw_step(mb.make_adamw_desc(**{**SET, "rate": 0.01 / k, "step": k}), b.args, b.table, norm[1:])
        assert all(torch.equal(x, y) for x, y in zip(a.p + a.m + a.v + a.ms + a.vs, b.p + b.m + b.v + b.ms + b.vs)), k


def test_lists_that_do_not_fit():
    t = _Tensors([10, 20])
    for kw in (dict(grads=t.g[:1]), dict(m=[t.m[0], t.v[0]]), dict(m=[None, t.m[1]]), dict(v=[t.v[0].cpu(), t.v[1]]), dict(copies=[None, t.p[1]])):
        with pytest.raises(ValueError):
            mb.make_adamw_tensors(**{**dict(params=t.p, grads=t.g, m=t.m, v=t.v), **kw})
    s = _Tensors([300], bits=8)
    with pytest.raises(ValueError):
        mb.make_adamw_tensors(s.p, s.g, s.m, s.v, [s.ms[0][:1]], s.vs)
    with pytest.raises(ValueError):
        mb.make_adamw_tensors([], [], [], [])


def _mix(x):
    x = (x ^ (x >> np.uint32(17))) * np.uint32(0x2C9277B5)
    x = (x ^ (x >> np.uint32(14))) * np.uint32(0x5851F42D)
    return x ^ (x >> np.uint32(16))


def _values32(code, scale, signed):
    low = code.astype(np.uint32) & np.uint32(127) if signed else code.astype(np.uint32)
    size = np.where(low > 0, ((low + np.uint32((112 if signed else 96) << 3)) << np.uint32(20)).view(np.float32) * scale, np.float32(0))
    return np.where(signed & (code >= 128), -size, size)


def _codes32(x, scale, bits, signed):
    u = np.where(scale > 0, np.abs(x) / np.where(scale > 0, scale, np.float32(1)), np.abs(x)).astype(np.float32)
    bits16 = bits >> np.uint32(16) if signed else bits & np.uint32(0xFFFF)
    code = ((u.view(np.uint32) + (bits16 << np.uint32(4))) >> np.uint32(20)).astype(np.int64) - ((112 if signed else 96) << 3)
    if not signed:
        return np.where(u > 0, np.clip(code, 1, 255), 0)
    least = np.float32(1.125 * 2.0 ** -15)
    c = np.where(u < least, u * (np.float32(65536.0) / least) > bits16.astype(np.float32), np.clip(code, 1, 127))
    return np.where((x < 0) & (c > 0), c + 128, c)


def test_codes_bit_by_bit():
    """States in 8 bits are what operations with one rounding each make of them, whatever the size of the values: from squares that vanish in 32 bits over blocks
    whose scales have no normal reciprocal to squares near the type's end.  (Every operation here is numpy's in 32 bits, so equality is exact.)"""
    powers = [0, -20, -40, -58, -62, -66, -72, 20, 40, 50, 56, 60]
    t = _Tensors([70001 if i < 2 else 3001 for i in range(len(powers))], bits=8, copy=False, seed=9)
    for i, e in enumerate(powers):
        t.g[i].mul_(2.0 ** e)
        t.ms[i].mul_(2.0 ** e)
        t.vs[i].mul_(max(2.0 ** (2 * e), 2.0 ** -149))
    before = [[x[i].cpu().numpy().copy() for x in (t.g, t.m, t.v, t.ms, t.vs)] for i in range(len(powers))]
    mb.mebptt_adamw_step(mb.make_adamw_desc(**SET), t.args, t.table)
    first, f = 0, np.float32
    with np.errstate(over="ignore"):
        for i, (g, m, v, ms, vs) in enumerate(before):
            n, blocks = g.size, ms.size
            of = np.arange(n) // 256
            key = _mix(np.uint32(SET["seed"]) + np.uint32(SET["step"]) * np.uint32(0x632BE5AB) + (first + np.arange(blocks)).astype(np.uint32) * np.uint32(0x9E3779B9))
            bits = _mix(key[of] + (np.arange(n) % 256).astype(np.uint32) * np.uint32(0x85157AF5))
            first += blocks
            new_m = f(SET["beta1"]) * _values32(m, ms[of], True) + f(1 - SET["beta1"]) * g
            new_v = f(SET["beta2"]) * _values32(v, vs[of], False) + f(1 - SET["beta2"]) * (g * g)
            for x, codes, scale, signed in ((new_m, t.m[i], t.ms[i], True), (new_v, t.v[i], t.vs[i], False)):
                top = np.pad(np.abs(x), (0, -n % 256)).reshape(-1, 256).max(1)
                s = top * (f(1.0) / f(1.875))
                assert np.array_equal(scale.cpu().numpy(), s), (powers[i], signed)
                assert np.array_equal(codes.cpu().numpy(), _codes32(x, s[of], bits, signed)), (powers[i], signed)
    assert t.clean()
