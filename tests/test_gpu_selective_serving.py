"""Serving the residual block around the selective scan in a batch whose sequences come and go."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _serving(slots, **kw):
    from paper_1606_03401_amd import selective as blk
    s = blk.Sizes(**{**dict(width=64, inner=96, N=16, groups=2, taps=4, stretch=16), **kw})
    return s, blk.Serving(s, blk.make_weights(s, 7), slots)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("lengths", [None, [19, 7, 19, 0]])
@pytest.mark.parametrize("wide", [False, True])
def test_a_prompt_passes_over_sequences_that_have_no_slot(lengths, wide):
    """An index before the pool or behind it, NaN in what comes with it: no slot but the others' own changes, the others' values are those of a
    batch in which everyone has a slot, and the sequence's own output is zero."""
    t, slots = 19, 5
    s, serve = _serving(slots)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn((t, 4, s.width), generator=g, device=DEV).bfloat16()
    res = torch.randn((t, 4, s.width), generator=g, device=DEV)
    lengths = None if lengths is None else _i32(*lengths)
    want = serve.prompt(x, res, _i32(3, 1, 2, 0), lengths)[0].clone()
    states = [p.clone() for p in (serve.conv_states, serve.scan_states)]
    for pool in (serve.conv_states, serve.scan_states):
        pool.copy_(torch.randn(pool.shape, generator=g, device=DEV))
    before = [p.clone() for p in (serve.conv_states, serve.scan_states)]
    x[:, 1:3] = float("nan")
    index = _i32(3, -1, slots, 0)
    out, _ = serve.prompt(x, res, index.long() if wide else index, lengths)
    assert torch.equal(out[:, [0, 3]], want[:, [0, 3]])
    assert bool((out[:, 1:3] == 0).all())
    for now, kept, was in zip((serve.conv_states, serve.scan_states), states, before):
        assert now.shape[0] == slots
        assert torch.equal(now[[0, 3]], kept[[0, 3]])
        assert torch.equal(now[[1, 2, 4]], was[[1, 2, 4]])


def test_prompts_of_many_lengths_leave_nothing_behind():
    s, serve = _serving(4)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    index = _i32(2, 0)

    def prompt(t):
        x = torch.randn((t, 2, s.width), generator=g, device=DEV).bfloat16()
        return serve.prompt(x, torch.zeros_like(x, dtype=torch.float32), index)

    prompt(30)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for t in range(1, 60):
        prompt(t)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before
    one, r = prompt(17)                       # the caller's own
    kept = one.clone(), r.clone()
    prompt(17)
    assert torch.equal(one, kept[0]) and torch.equal(r, kept[1])


def test_two_streams_serve_from_buffers_of_their_own():
    """Tokens of different sequences on two streams at once, the same batch size: every one's values are those of a call by itself."""
    s, serve = _serving(8)
    other = type(serve)(s, serve.w, 8)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    halves = [_i32(0, 1, 2, 3), _i32(4, 5, 6, 7)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    xs = [[torch.randn((4, s.width), generator=g, device=DEV).bfloat16() for _ in range(20)] for _ in halves]
    res = torch.randn((4, s.width), generator=g, device=DEV)
    want = [[other.token(x, res, at)[0].clone() for x in v] for v, at in zip(xs, halves)]
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(20):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k].append(serve.token(xs[k][i], res, halves[k])[0].clone())
    torch.cuda.synchronize()
    for k in (0, 1):
        assert all(torch.equal(a, b) for a, b in zip(got[k], want[k]))
    assert len({v["out"].data_ptr() for v in serve.kept.values()}) == 2
