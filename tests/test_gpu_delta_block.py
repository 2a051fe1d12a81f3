"""The residual block around the gated delta rule and AdamW as they are used together: a gradient step through all operators against float64 autograd of the same
formulas, training with states of 8 and 32 bits, prompts and single tokens against each other, captured steps; AdamW on the gradients of an LSTM session."""
import numpy as np
import pytest
import torch

from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _sizes(**kw):
    from paper_1606_03401_amd import delta as blk
    return blk, blk.Sizes(**{**dict(width=64, heads=4, key_heads=2, dk=24, dv=32, stretch=64, scale=0.9), **kw})


def _reference(s, w, n, r):
    """The block in float64 by the formulas, for autograd."""
    t, B, _ = n.shape
    norm = lambda v, k: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-5) * k  # noqa: E731
    silu = lambda v: v * torch.sigmoid(v)  # noqa: E731
    p = n @ w["W_in"].t()
    at = s.mixed + s.values
    mixed, z, a, b = p[..., :s.mixed], p[..., s.mixed:at], p[..., at:at + s.heads], p[..., at + s.heads:]
    rows = torch.cat([torch.zeros(s.taps - 1, B, s.mixed, dtype=torch.float64), mixed])
    c = silu(sum(rows[j:j + t] * w["conv"][:, j] for j in range(s.taps)) + w["conv_bias"])
    unit = lambda m: m * torch.rsqrt(m.square().sum(-1, keepdim=True) + 1e-6)  # noqa: E731
    wide = lambda m: unit(m.view(t, B, s.key_heads, s.dk)).repeat_interleave(s.heads // s.key_heads, 2)  # noqa: E731
    q, k, v = wide(c[..., :s.keys]) * s.dk ** -0.5, wide(c[..., s.keys:2 * s.keys]), c[..., 2 * s.keys:].view(t, B, s.heads, s.dv)
    alpha, beta = torch.exp(w["A"] * torch.nn.functional.softplus(a + w["a_bias"])), torch.sigmoid(b)
    S, ys = torch.zeros(B, s.heads, s.dk, s.dv, dtype=torch.float64), []
    for i in range(t):
        S = alpha[i][..., None, None] * S
        e = v[i] - (S * k[i][..., None]).sum(2)
        S = S + k[i][..., None] * (beta[i][..., None] * e)[:, :, None]
        ys.append((S * q[i][..., None]).sum(2))
    y = torch.stack(ys)
    m = norm(y, w["head"].view(s.heads, s.dv)).flatten(2) * silu(z)
    total = s.scale * r + norm(m @ w["W_out"].t(), w["post"])
    return norm(total, w["norm"]), total


def test_gradient_step_against_float64_autograd():
    """bf16 activations: every stored activation and gradient is rounded once, 2^-9 of itself, about ten times between a weight and its
    gradient; 5 % of a tensor's norm is more than five times what those add up to in the mean."""
    blk, s = _sizes()
    t, B = 70, 3
    w = blk.make_weights(s, 3)
    w16 = {k: w[k].bfloat16() for k in blk.PROJECTIONS}
    run = blk.Training(s, t, B)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    normal = lambda: torch.randn((t, B, s.width), generator=g, device=DEV)  # noqa: E731
    n, r, dn, dr = normal().bfloat16(), normal(), normal().bfloat16(), normal()
    n_out, r_out = (x.clone() for x in run.forward(w, w16, n, r))
    grads, dn_in, dr_in = run.backward(w, w16, dn, dr)
    ref_w = {k: (w16[k] if k in w16 else w[k]).double().cpu().requires_grad_() for k in w}
    rn, rr = n.double().cpu().requires_grad_(), r.double().cpu().requires_grad_()
    want_n, want_r = _reference(s, ref_w, rn, rr)
    ((want_n * dn.double().cpu()).sum() + (want_r * dr.double().cpu()).sum()).backward()
    pairs = {"n": (n_out, want_n.detach()), "r": (r_out, want_r.detach()), "dn": (dn_in, rn.grad), "dr": (dr_in, rr.grad), **{k: (grads[k], ref_w[k].grad) for k in w}}
    for name, (got, want) in pairs.items():
        err = float((got.double().cpu() - want).norm() / want.norm())
        assert np.isfinite(err) and err < 0.05, (name, err)


@pytest.mark.parametrize("bits", [8, 32])
def test_training_runs(bits):
    blk, s = _sizes(key_heads=0)
    w, losses = blk.train(s, t=96, B=4, steps=6, bits=bits)
    assert np.isfinite(losses).all() and all(bool(v.isfinite().all()) for v in w.values())


@pytest.mark.parametrize("bits", [8, 32])
def test_the_scans_block_with_adamw(bits):
    from paper_1606_03401_amd import selective as blk
    w, losses = blk.train(blk.Sizes(width=64, inner=96, stretch=16), t=40, B=4, steps=5, rate=1e-3, adamw=bits)
    assert np.isfinite(losses).all() and all(bool(v.isfinite().all()) for v in w.values())


def test_tokens_go_on_where_prompts_of_unequal_lengths_end():
    """The same values in other orders: projections of one row and of many may be summed differently by the matrix library, and a bf16 rounding falls the other way
    here and there: 2^-8 of a value, through three more roundings; 2 % of the largest value."""
    blk, s = _sizes()
    serve = blk.Serving(s, blk.make_weights(s, 7), 9)
    t, more, lengths = 80, 5, [80, 1, 64, 8]
    B = len(lengths)
    n, r = torch.randn((t + more, B, s.width), device=DEV).bfloat16(), torch.randn((t + more, B, s.width), device=DEV)
    index = torch.tensor([4, 0, 8, 2], dtype=torch.int32, device=DEV)
    wholes = []
    for b, m in enumerate(lengths):
        _, out = serve.prompt(n[:m + more, b:b + 1], r[:m + more, b:b + 1], torch.tensor([6], device=DEV))
        wholes.append(out[m:, 0].clone())
    serve.prompt(n[:t], r[:t], index, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    spare = serve.delta_states[[1, 3, 5, 7]].clone()
    for i in range(more):
        at = [(m + i, b) for b, m in enumerate(lengths)]
        _, out = serve.token(torch.stack([n[a] for a in at]), torch.stack([r[a] for a in at]), index)
        for b in range(B):
            assert float((out[b] - wholes[b][i]).abs().max()) <= 0.02 * float(wholes[b].abs().max()), (i, b)
    assert torch.equal(serve.delta_states[[1, 3, 5, 7]], spare)


def test_captured_token_step_replays_as_the_eager_one():
    blk, s = _sizes()
    w = blk.make_weights(s, 7)
    serve, other = blk.Serving(s, w, 4), blk.Serving(s, w, 4)
    index = torch.tensor([3, 1, -1, 0], dtype=torch.int32, device=DEV)
    n, r = torch.zeros((4, s.width), dtype=torch.bfloat16, device=DEV), torch.zeros((4, s.width), device=DEV)
    serve.token(n, r, index)
    other.token(n, r, index)
    torch.cuda.synchronize()
    before = (serve.conv_states.clone(), serve.delta_states.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n_out, r_out = serve.token(n, r, index)
    serve.conv_states.copy_(before[0])
    serve.delta_states.copy_(before[1])
    for i in range(5):
        n.copy_(torch.randn(n.shape, device=DEV))
        r.copy_(torch.randn(r.shape, device=DEV))
        graph.replay()
        want_n, want_r = other.token(n, r, index)
        torch.cuda.synchronize()
        assert torch.equal(n_out, want_n) and torch.equal(r_out, want_r), i
        assert torch.equal(serve.delta_states, other.delta_states) and torch.equal(serve.conv_states, other.conv_states), i


def test_captured_training_step():
    """Forward, backward and AdamW as one graph, against eager steps of a block of its own."""
    blk, s = _sizes()
    t, B = 66, 2
    made = []
    for _ in range(2):
        w = blk.make_weights(s, 1)
        run = blk.Training(s, t, B)
        w16 = {k: w[k].bfloat16() for k in blk.PROJECTIONS}
        opt = blk.AdamW(list(w.values()), [run.g[k] for k in w], 1e-3, bits=8, clip=1.0, copies=[w16.get(k) for k in w])
        made.append((w, run, w16, opt))
    n, r, dr = torch.zeros((t, B, s.width), dtype=torch.bfloat16, device=DEV), torch.zeros((t, B, s.width), device=DEV), torch.zeros((t, B, s.width), device=DEV)
    zero = torch.zeros_like(n)

    def body(w, run, w16, opt):
        run.forward(w, w16, n, r)
        run.backward(w, w16, zero, dr)
        opt.step()
    for x in (n, r, dr):
        x.copy_(torch.randn(x.shape, device=DEV))
    for m in made:
        body(*m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(*made[0])
    for i in range(3):
        for x in (n, r, dr):
            x.copy_(torch.randn(x.shape, device=DEV))
        graph.replay()
        body(*made[1])
        torch.cuda.synchronize()
        for k in made[0][0]:
            # (the matrix library may sum differently under capture)
            assert torch.allclose(made[0][0][k], made[1][0][k], rtol=1e-2, atol=2e-3 * float(made[1][0][k].abs().max())), (i, k)
        assert int(made[0][3].count) == int(made[1][3].count) == i + 2


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_on_a_sessions_gradients(bits):
    """An LSTM's gradient step within a memory budget, and AdamW on what it wrote."""
    from oracle import delta as od
    from paper_1606_03401_amd import workloads as wl
    from paper_1606_03401_amd.optimiser import AdamW
    from paper_1606_03401_amd.session import Session
    w = wl.CONFIGS["cfg1"]
    sess = Session(w, wl.make_inputs(w))
    params, grads = [sess.W_ih, sess.W_hh, sess.b], [sess.dW_ih, sess.dW_hh, sess.db]
    opt = AdamW(params, grads, rate=1e-2, decay=0.1, bits=bits)
    before = [p.double().cpu().numpy() for p in params]
    sess.run()
    opt.step()
    torch.cuda.synchronize()
    m, v = opt.states()
    for i, p in enumerate(params):
        g = grads[i].double().cpu().numpy()
        want, wm, wv = od.adamw(before[i], g, 0 * g, 0 * g, 1e-2, 0.9, 0.999, 1e-8, 0.1, 1)
        assert np.abs(p.double().cpu().numpy() - want).max() <= 2.0 ** -20 * (np.abs(want).max() + 1e-2)
        near = 1 / 8 if bits == 8 else 2.0 ** -22       # a code's step
        scale = (np.abs(wm).max(), wv.max())
        for got, exact, top, floor in ((m[i], wm, scale[0], 2.0 ** -15), (v[i], wv, scale[1], 2.0 ** -31)):
            assert (np.abs(got.double().cpu().numpy() - exact) <= near * np.abs(exact) * 1.001 + 1.2 * floor * top).all()
    sess.run()
    opt.step()
    assert mb.mebptt_last_error() is not None and all(bool(p.isfinite().all()) for p in params)
