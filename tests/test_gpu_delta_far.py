"""Offsets that leave 32 bits, in the operators around the gated delta rule: steps 2^23 values apart, a pool of states of over 2^31 values, rows 2^26 values apart, a tensor of
over 2^31 values.  Only what a call reads is filled in; results are those of the same values side by side."""
import pytest
import torch
from placed import DEV, room

from oracle import delta as od
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu


def _far(t, base, at, strides):
    """A copy of `t` in `base`, its first value at `at`, with the given strides of all dimensions but the last."""
    view = base.as_strided(t.shape, (*strides, 1), at)
    view.copy_(t)
    return view


def test_steps_far_apart():
    t, B, Hk, H, dk, dv, gap = 300, 2, 1, 2, 40, 24, 1 << 23
    T, g = torch.bfloat16, torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    given = [r(t, B, Hk * dk).to(T), r(t, B, Hk * dk).to(T), r(t, B, H * dv).to(T), r(t, B, H).to(T), r(t, B, H).to(T)]   # q, k, v, a, b
    dy, A, bias, h0, dh = (r(t, B, H * dv) * 0.1).to(T), -torch.rand(H, generator=g, device=DEV) - 0.1, r(H) - 3, r(B, H, dk, dv) * 0.3, r(B, H, dk, dv) * 0.1
    desc = mb.make_delta_desc(t, B, Hk, H, dk, dv, mb.BF16, 1, 1, 64, dk ** -0.5)
    shapes = [(t, B, H * dv), (t, B, Hk * dk), (t, B, Hk * dk), (t, B, H * dv), (t, B, H), (t, B, H)]                        # y, dq, dk, dv, da, db
    base = torch.empty((t - 1) * gap + (1 << 14), dtype=T, device=DEV)                                                     # (5 GB)
    results = []
    for far in (False, True):
        place = iter(range(0, 1 << 14, 512))
        put = (lambda x: _far(x, base, next(place), (gap, 200))) if far else (lambda x: x)
        q, k, v, a, b = (put(x) for x in given)
        out = [put(torch.full(s, float("nan"), dtype=T, device=DEV)) for s in shapes]
        h, dA, da_bias, dh0 = torch.empty_like(h0), torch.empty_like(A), torch.empty_like(A), torch.empty_like(h0)
        states, ws = room(mb.mebptt_delta_state_bytes(desc)), room(mb.mebptt_delta_workspace_bytes(desc, True))
        mb.mebptt_delta_forward(desc, q, k, v, a, b, A, bias, None, h0, out[0], h, states, ws)
        mb.mebptt_delta_backward(desc, q, k, v, a, b, A, bias, None, h0, put(dy), dh, states, *out[1:], dA, da_bias, dh0, ws)
        results.append([x.clone() for x in (*out, h, dA, da_bias, dh0)])
    for one, two in zip(*results):
        assert bool(torch.isfinite(one).all()) and torch.equal(one, two)


def test_a_large_pool():
    H, dk, dv = 2, 128, 128
    slots = (1 << 31) // (H * dk * dv) + 3                   # 8.6 GB
    pool, index = torch.empty((slots, H, dk, dv), device=DEV), torch.tensor([slots - 1, 1, slots - 2], dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    h, x = r(3, H, dk, dv) * 0.3, (r(3, H * dk), r(3, H * dk), r(3, H * dv), r(3, H), r(3, H), -torch.ones(H, device=DEV), None)
    pool[index.long()] = h
    desc = mb.make_delta_desc(1, 3, H, H, dk, dv, mb.FP32, 1, 1, 0, dk ** -0.5)
    y, far_y = torch.empty((3, H * dv), device=DEV), torch.empty((3, H * dv), device=DEV)
    mb.mebptt_delta_step(desc, *x, h, None, y, h)
    mb.mebptt_delta_step(desc, *x, pool, index, far_y, pool)
    assert torch.equal(y, far_y) and torch.equal(pool[index.long()], h)


@pytest.mark.parametrize("group", [264, 33])
def test_rows_far_apart(group):
    rows, width, ld = 40, 264, 1 << 26
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda: torch.randn((rows, width), generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    given, w = [r() for _ in range(5)], torch.rand((2, width), generator=g, device=DEV) + 0.5      # x, z, residual, dy, dresidual_out
    desc = mb.make_join_desc(rows, width, group, mb.BF16, mb.BF16, 0.5, 1e-5)
    base = torch.empty((rows - 1) * ld + (1 << 14), dtype=torch.bfloat16, device=DEV)             # (5 GB)
    results = []
    for far in (False, True):
        place = iter(range(0, 1 << 14, 512))
        put = (lambda t: _far(t, base, next(place), (ld,))) if far else (lambda t: t)
        x, z, residual, dy, dout = (put(t) for t in given)
        y, out, dx, dz, dres = (put(torch.full_like(given[0], float("nan"))) for _ in range(5))
        rstd, rn, dw, dwn = torch.empty((rows, width // group), device=DEV), torch.empty(rows, device=DEV), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
        mb.mebptt_join_forward(desc, x, z, w[0], residual, w[1], y, out, rstd, rn)
        mb.mebptt_join_backward(desc, x, z, w[0], out, w[1], rstd, rn, dy, dout, dx, dz, dw, dres, dwn, room(mb.mebptt_join_workspace_bytes(desc)))
        results.append([t.clone() for t in (y, out, dx, dz, dres, rstd, rn, dw, dwn)])
    for one, two in zip(*results):
        assert bool(torch.isfinite(one).all()) and torch.equal(one, two)


def test_a_tensor_of_over_two_to_the_31_values():
    """Its last values, around a piece's end, as the formula has them: within a few roundings of 2^-24 (as in the tests of ordinary sizes)."""
    n, last = (1 << 31) + 5000, 6000
    big = [torch.empty(n, device=DEV) for _ in range(4)]     # p, g, m, v: 34 GB
    g = torch.Generator(device=DEV).manual_seed(4)
    for t in big:
        t[-last:] = torch.rand(last, generator=g, device=DEV) + 0.5
    before = [t[-last:].double().cpu().numpy() for t in big]
    args = mb.make_adamw_tensors(*([t] for t in big))
    table = room(mb.mebptt_adamw_table_bytes(args))
    mb.mebptt_adamw_prepare(args, table)
    mb.mebptt_adamw_step(mb.make_adamw_desc(1e-2, 0.9, 0.98, 1e-8, 0.1, 3), args, table)
    want = od.adamw(*before, 1e-2, 0.9, 0.98, 1e-8, 0.1, 3)
    for t, x in zip((big[0], big[2], big[3]), want):
        assert (abs(t[-last:].double().cpu().numpy() - x) <= 2.0 ** -20 * abs(x)).all()
