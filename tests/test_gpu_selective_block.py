"""The residual block around the selective scan: a gradient step through all its operators against float64 autograd of the same formulas,
training that learns, prompts of unequal lengths and single tokens in 8 bits against each other, and a captured token step."""
import numpy as np
import pytest
import torch

from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu


def _sizes(**kw):
    from paper_1606_03401_amd import selective as blk
    return blk, blk.Sizes(**{**dict(width=64, inner=96, N=16, groups=2, taps=4, stretch=16), **kw})


def _reference(s, w, x, residual):
    """The block in float64 by the formulas, for autograd; inputs and weights as they are."""
    t, B, _ = x.shape
    norm = lambda v, k: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-5) * k  # noqa: E731
    silu = lambda v: v * torch.sigmoid(v)  # noqa: E731
    r = x + residual
    p = norm(r, w["norm"]) @ w["W_in"].t()
    D, S = s.inner, s.shared
    z, mixed, delta = p[..., :D], p[..., D:D + s.mixed], p[..., D + s.mixed:]
    rows = torch.cat([torch.zeros(s.taps - 1, B, s.mixed, dtype=torch.float64), mixed])
    c = silu(sum(rows[j:j + t] * w["conv"][:, j] for j in range(s.taps)) + w["conv_bias"])
    u, Bm, Cm = c[..., :D], c[..., D:D + S], c[..., D + S:]
    step = torch.nn.functional.softplus(delta + w["delta_bias"])
    wide = lambda m: m.view(B, s.groups, s.N).repeat_interleave(D // s.groups, 1)  # noqa: E731
    h, ys = torch.zeros(B, D, s.N, dtype=torch.float64), []
    for i in range(t):
        h = torch.exp(step[i][..., None] * w["A"]) * h + (step[i] * u[i])[..., None] * wide(Bm[i])
        ys.append(((h * wide(Cm[i])).sum(-1) + w["skip"] * u[i]) * silu(z[i]))
    return norm(torch.stack(ys), w["norm_out"]) @ w["W_out"].t(), r


def test_gradient_step_against_float64_autograd():
    """bf16 activations: every stored activation and gradient is rounded once, 2^-9 of itself, about ten times between a weight and its
    gradient; 5 % of a tensor's norm is more than five times what those add up to in the mean."""
    blk, s = _sizes()
    t, B = 40, 3
    w = blk.make_weights(s, 3)
    run = blk.Training(s, t, B)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    x = torch.randn((t, B, s.width), generator=g, device="cuda:0").bfloat16()
    res = torch.randn((t, B, s.width), generator=g, device="cuda:0")
    dout = torch.randn((t, B, s.width), generator=g, device="cuda:0").bfloat16()
    dr = torch.randn((t, B, s.width), generator=g, device="cuda:0")
    out = run.forward(w, x, res)
    grads, dx, dres = run.backward(w, dout, dr)
    ref_w = {k: v.double().cpu().requires_grad_() for k, v in w.items()}
    for k in ("W_in", "W_out"):       # as the products see them
        ref_w[k] = w[k].bfloat16().double().cpu().requires_grad_()
    rx, rres = x.double().cpu().requires_grad_(), res.double().cpu().requires_grad_()
    ref, r = _reference(s, ref_w, rx, rres)
    ((ref * dout.double().cpu()).sum() + (r * dr.double().cpu()).sum()).backward()
    pairs = {"out": (out, ref.detach()), "dx": (dx, rx.grad), "dresidual": (dres, rres.grad), **{k: (grads[k], ref_w[k].grad) for k in w}}
    for name, (got, want) in pairs.items():
        err = float((got.double().cpu() - want).norm() / want.norm())
        assert np.isfinite(err) and err < 0.05, (name, err)
    assert torch.equal(run.r.view(t, B, s.width), x.float() + res)


def test_training_lowers_the_loss():
    blk, s = _sizes(groups=1)
    _, losses = blk.train(s, t=64, B=16, steps=40)
    assert np.isfinite(losses).all() and np.mean(losses[-5:]) < 0.9 * np.mean(losses[:2]), (losses[0], losses[-1])


def _serving(slots):
    blk, s = _sizes()
    return blk, s, blk.Serving(s, blk.make_weights(s, 7), slots)


def test_tokens_go_on_where_prompts_of_unequal_lengths_end():
    """8 bits: a row's values move by up to half a step, 1 / 254 of the largest, where a tie falls the other way; the two ways round the
    same values otherwise, so 2 % of the largest output is allowed."""
    blk, s, serve = _serving(9)
    t, more, lengths = 21, 5, [21, 1, 13, 8]
    B = len(lengths)
    x = torch.randn((t + more, B, s.width), device="cuda:0").bfloat16()
    res = torch.randn((t + more, B, s.width), device="cuda:0")
    index = torch.tensor([4, 0, 8, 2], dtype=torch.int32, device="cuda:0")
    wholes = []
    for b, n in enumerate(lengths):
        out, r = serve.prompt(x[:n + more, b:b + 1], res[:n + more, b:b + 1], torch.tensor([6], device="cuda:0"))
        wholes.append((out[n:, 0].float().clone(), r[n:, 0].clone()))
    serve.prompt(x[:t], res[:t], index, torch.tensor(lengths, dtype=torch.int32, device="cuda:0"))
    spare = serve.scan_states[[1, 3, 5, 7]].clone()
    for i in range(more):
        at = [(n + i, b) for b, n in enumerate(lengths)]
        out, r = serve.token(torch.stack([x[a] for a in at]), torch.stack([res[a] for a in at]), index)
        for b in range(B):
            want, want_r = wholes[b]
            assert float((out[b].float() - want[i]).abs().max()) <= 0.02 * float(want.abs().max()), (i, b)
            assert torch.equal(r[b], want_r[i])
    assert torch.equal(serve.scan_states[[1, 3, 5, 7]], spare)


def test_captured_token_step_replays_as_the_eager_one():
    """A token of every sequence as one HIP graph, replayed with eager work in between; every replay against the eager call on
    states of its own."""
    blk, s, serve = _serving(4)
    other = blk.Serving(s, serve.w, 4)
    index = torch.tensor([3, 1, -1, 0], dtype=torch.int32, device="cuda:0")
    x, res = torch.zeros((4, s.width), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((4, s.width), device="cuda:0")
    serve.token(x, res, index)
    other.token(x, res, index)
    torch.cuda.synchronize()
    before = (serve.conv_states.clone(), serve.scan_states.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, r = serve.token(x, res, index)
    serve.conv_states.copy_(before[0])
    serve.scan_states.copy_(before[1])
    for i in range(6):
        x.copy_(torch.randn(x.shape, device="cuda:0"))
        res.copy_(torch.randn(res.shape, device="cuda:0"))
        graph.replay()
        want, want_r = other.token(x, res, index)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(r, want_r), i
        assert torch.equal(serve.scan_states, other.scan_states) and torch.equal(serve.conv_states, other.conv_states), i
        assert not torch.randn(3000, 3000, device="cuda:0").sum().isnan()


def test_captured_gradient_step_replays_as_the_eager_one():
    blk, s = _sizes()
    t, B = 40, 2
    w = blk.make_weights(s, 1)
    run, other = blk.Training(s, t, B), blk.Training(s, t, B)
    x, res = torch.zeros((t, B, s.width), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((t, B, s.width), device="cuda:0")
    dout = torch.zeros_like(x)
    run.forward(w, x, res)
    run.backward(w, dout)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run.forward(w, x, res)
        grads, dx, dr = run.backward(w, dout)
    for i in range(4):
        for a in (x, res, dout):
            a.copy_(torch.randn(a.shape, device="cuda:0"))
        graph.replay()
        want = other.forward(w, x, res)
        want_g, want_dx, want_dr = other.backward(w, dout)
        torch.cuda.synchronize()
        for k in ("norm", "conv", "conv_bias", "A", "skip", "delta_bias", "norm_out"):
            assert torch.allclose(grads[k], want_g[k], rtol=1e-5, atol=1e-6 * float(want_g[k].abs().max())), (i, k)
        assert torch.allclose(out.float(), want.float(), rtol=2e-2, atol=1e-3) and torch.allclose(dr, want_dr, rtol=2e-2, atol=1e-3), i
        assert mb.mebptt_last_error() is not None
