"""Pins of the float64 operators of the selective state space block: every backward formula against central differences, the
scan against its closed form for one step and for a constant decay, the convolution against numpy's, lengths and states against the
same sequence run in two parts."""
import numpy as np
import pytest

from oracle import selective as sel


def _differences(loss, params, eps=1e-6):
    out = {}
    for name, p in params.items():
        g = np.zeros_like(p)
        for i in np.ndindex(p.shape):
            old = p[i]
            p[i] = old + eps
            hi = loss()
            p[i] = old - eps
            lo = loss()
            p[i] = old
            g[i] = (hi - lo) / (2 * eps)
        out[name] = g
    return out


def _near(got, want):
    # central differences of a smooth function in float64: eps^2 of the third derivative, 1e-16 / eps of rounding
    assert np.abs(got - want).max() <= 1e-7 * max(1.0, np.abs(want).max())


def test_norm_backward_matches_differences():
    rng = np.random.default_rng(0)
    p = {"x": rng.standard_normal((3, 5)), "residual": rng.standard_normal((3, 5)), "weight": rng.standard_normal(5)}
    dy, dr_out = rng.standard_normal((3, 5)), rng.standard_normal((3, 5))

    def loss():
        r, y, _ = sel.norm(p["x"], p["residual"], p["weight"], 1e-3)
        return (y * dy).sum() + (r * dr_out).sum()
    want = _differences(loss, p)
    dr, dweight = sel.norm_backward(p["x"] + p["residual"], p["weight"], dy, dr_out, 1e-3)
    for got, name in ((dr, "x"), (dr, "residual"), (dweight, "weight")):
        _near(got, want[name])


@pytest.mark.parametrize("W,silu,state,lengths", [(1, True, False, None), (2, False, True, None), (4, True, True, [5, 0, 1]),
                                                  (4, True, False, [2, 5, 3]), (8, True, True, [3, 5, 1])])
def test_conv_backward_matches_differences(W, silu, state, lengths):
    rng = np.random.default_rng(W)
    t, B, C = 5, 3, 2
    p = {"x": rng.standard_normal((t, B, C)), "weight": rng.standard_normal((C, W)), "bias": rng.standard_normal(C),
         "state": rng.standard_normal((B, W - 1, C))}
    st = p["state"] if state else None
    dy, dlast = rng.standard_normal((t, B, C)), rng.standard_normal((B, W - 1, C))

    def loss():
        y, last = sel.conv(p["x"], p["weight"], p["bias"], lengths, st, silu)
        return (y * dy).sum() + (last * dlast).sum()
    want = _differences(loss, p)
    dx, dw, db, ds = sel.conv_backward(p["x"], p["weight"], p["bias"], lengths, st, silu, dy, dlast)
    _near(dx, want["x"])
    _near(dw, want["weight"])
    _near(db, want["bias"])
    if state:
        _near(ds, want["state"])


def test_conv_is_the_convolution():
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((9, 1, 1)), rng.standard_normal((1, 4))
    y, _ = sel.conv(x, w, None, None, None, False)
    assert np.allclose(y[:, 0, 0], np.convolve(x[:, 0, 0], w[0, ::-1])[:9], atol=1e-12)


@pytest.mark.parametrize("G,gate,softplus,lengths", [(1, True, True, None), (2, False, True, [4, 0]), (2, True, False, [1, 4])])
def test_scan_backward_matches_differences(G, gate, softplus, lengths):
    rng = np.random.default_rng(G)
    t, B, D, N = 4, 2, 4, 3
    n = rng.standard_normal
    p = {"u": n((t, B, D)), "delta": n((t, B, D)) if softplus else rng.uniform(0.1, 1, (t, B, D)), "A": -rng.uniform(0.1, 2, (D, N)),
         "Bm": n((t, B, G * N)), "Cm": n((t, B, G * N)), "skip": n(D), "delta_bias": n(D) * 0.1, "h0": n((B, D, N)), "z": n((t, B, D))}
    dy, dh = n((t, B, D)), n((B, D, N))
    args = lambda: (p["u"], p["delta"], p["A"], p["Bm"], p["Cm"], G, p["skip"], p["z"] if gate else None, p["delta_bias"],  # noqa: E731
                    lengths, p["h0"], softplus)

    def loss():
        y, h = sel.scan(*args())
        return (y * dy).sum() + (h * dh).sum()
    want = _differences(loss, p)
    got = sel.scan_backward(*args(), dy, dh)
    for k, name in (("du", "u"), ("ddelta", "delta"), ("dA", "A"), ("dB", "Bm"), ("dC", "Cm"), ("dskip", "skip"),
                    ("ddelta_bias", "delta_bias"), ("dh0", "h0"), ("dz", "z")):
        _near(got[k], want[name])


def test_scan_of_a_constant_decay_is_a_geometric_sum():
    t = 7
    one = np.ones((t, 1, 1))
    y, h = sel.scan(one, 0.5 * one, -np.ones((1, 1)), one, one, 1, softplus=False)
    a = np.exp(-0.5)
    want = [0.5 * (1 - a ** (s + 1)) / (1 - a) for s in range(t)]
    assert np.allclose(y[:, 0, 0], want, atol=1e-14) and np.isclose(h[0, 0, 0], want[-1], atol=1e-14)


def test_parts_of_a_sequence_give_the_whole():
    rng = np.random.default_rng(5)
    t, B, D, N, cut = 9, 2, 4, 3, 4
    n = rng.standard_normal
    u, delta, Bm, Cm, A = n((t, B, D)), n((t, B, D)), n((t, B, N)), n((t, B, N)), -rng.uniform(0.1, 2, (D, N))
    y, h = sel.scan(u, delta, A, Bm, Cm, 1)
    y1, h1 = sel.scan(u[:cut], delta[:cut], A, Bm[:cut], Cm[:cut], 1)
    y2, h2 = sel.scan(u[cut:], delta[cut:], A, Bm[cut:], Cm[cut:], 1, h0=h1)
    assert np.allclose(np.concatenate([y1, y2]), y, atol=1e-12) and np.allclose(h, h2, atol=1e-12)
    w = n((D, 4))
    y, last = sel.conv(u, w, None, None, None, True)
    y1, l1 = sel.conv(u[:cut], w, None, None, None, True)
    y2, l2 = sel.conv(u[cut:], w, None, None, l1, True)
    assert np.allclose(np.concatenate([y1, y2]), y, atol=1e-12) and np.allclose(last, l2, atol=1e-12)
    # a length is a shorter sequence
    y3, h3 = sel.scan(u, delta, A, Bm, Cm, 1, lengths=[cut, cut])
    assert np.allclose(y3[:cut], sel.scan(u[:cut], delta[:cut], A, Bm[:cut], Cm[:cut], 1)[0]) and np.allclose(h3, h1) and not y3[cut:].any()
