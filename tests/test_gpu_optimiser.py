"""AdamW's object: a step that its clip refuses has not been taken, whatever comes after it; steps go on from what a checkpoint kept."""
import pytest
import torch
from placed import DEV, NAN

from paper_1606_03401_amd.optimiser import AdamW

pytestmark = pytest.mark.gpu

SIZES = [(40, 30), (257,), (1,), (5000,)]


def _made(bits):
    g = torch.Generator(device=DEV).manual_seed(2)
    params = [torch.randn(s, generator=g, device=DEV) for s in SIZES]
    given = [[torch.randn(s, generator=g, device=DEV) for s in SIZES] for _ in range(3)]
    grads = [torch.zeros(s, device=DEV) for s in SIZES]
    copies = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in SIZES]
    return AdamW(params, grads, 1e-2, bits=bits, clip=1.0, copies=copies, seed=4), params, grads, given, copies


def _everything(opt, params, copies):
    scales = (opt.m_scale + opt.v_scale) if opt.bits == 8 else []
    return [x.clone() for x in params + copies + opt.m + opt.v + scales + [opt.count]]


@pytest.mark.parametrize("replayed", [False, True])
@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf")])
@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_that_was_not_taken_does_not_count(bits, bad, replayed):
    (a, pa, ga, given, ca), (b, pb, gb, _, cb) = _made(bits), _made(bits)
    step = a.step
    if replayed:
        start = [(x, x.clone()) for x in pa + ca + a.m + a.v + ((a.m_scale + a.v_scale) if bits == 8 else []) + [a.count, a.norm]]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a.step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.step()
        for x, was in start:
            x.copy_(was)
        step = graph.replay
    for k, grads in enumerate(given):
        for x, y, g in zip(ga, gb, grads):
            x.copy_(g)
            y.copy_(g)
        ga[3][17] = bad           # first a step that is refused, then the same one as it should be
        before = _everything(a, pa, ca)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(_everything(a, pa, ca), before)), k
        ga[3][17] = given[k][3][17]
        step()
        b.step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(_everything(a, pa, ca), _everything(b, pb, cb))), k
        assert int(a.count) == k + 1


@pytest.mark.parametrize("bits", [8, 32])
def test_without_a_clip_every_step_counts(bits):
    opt, params, grads, given, copies = _made(bits)
    opt.clip = None
    for k in range(3):
        opt.step()
        assert int(opt.count) == k + 1


@pytest.mark.parametrize("bits", [8, 32])
def test_steps_go_on_from_a_checkpoint(bits):
    """Bit by bit, also where values are rounded by chance."""
    (a, pa, ga, given, ca), (b, pb, gb, _, cb) = _made(bits), _made(bits)
    for k, grads in enumerate(given):
        if k == 2:
            for x, y in zip(pb + b.m + b.v, pa + a.m + a.v):
                x.copy_(y)
            for x, y in zip((b.m_scale + b.v_scale) if bits == 8 else [], (a.m_scale + a.v_scale) if bits == 8 else []):
                x.copy_(y)
            b.count.copy_(a.count)
        for x, y, g in zip(ga, gb, grads):
            x.copy_(g)
            y.copy_(g)
        a.step()
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(_everything(a, pa, ca), _everything(b, pb, cb)))
    for x, y in zip(sum(a.states(), []), sum(b.states(), [])):
        assert torch.equal(x, y)
