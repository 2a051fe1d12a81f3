"""The float64 formulas of the delta rule, the norms around a block and AdamW against differences, against each other and against hand-worked values."""
import numpy as np
import pytest

from oracle import delta as od


def _differences(f, x, at, h=1e-6):
    up, down = x.copy(), x.copy()
    up[at] += h
    down[at] -= h
    return (f(up) - f(down)) / (2 * h)


@pytest.mark.parametrize("activate,normalise,decay,lengths", [(True, True, True, None), (True, False, True, [5, 0, 1]), (False, True, True, [3, 5, 2]),
                                                              (True, True, False, None)])
def test_delta_gradients_against_differences(activate, normalise, decay, lengths):
    rng = np.random.default_rng(5)
    t, B, Hk, H, dk, dv = 5, 3, 2, 4, 3, 2
    x = {"q": rng.standard_normal((t, B, Hk * dk)), "k": rng.standard_normal((t, B, Hk * dk)) * 0.5, "v": rng.standard_normal((t, B, H * dv)),
         "a": -rng.random((t, B, H)), "b": rng.random((t, B, H)), "A": -rng.random(H), "a_bias": rng.standard_normal(H), "h0": rng.standard_normal((B, H, dk, dv))}
    if not decay:
        x.update(a=None, A=None, a_bias=None)
    dy, dh = rng.standard_normal((t, B, H * dv)), rng.standard_normal((B, H, dk, dv))

    def run(v, **more):
        return od.delta(v["q"], v["k"], v["v"], v["a"], v["b"], v["A"], v["a_bias"], Hk, H, 0.7, activate, normalise, 1e-3, lengths, v["h0"], **more)

    def loss(v):
        y, h = run(v)
        return (y * dy).sum() + (h * dh).sum()
    got = run(x, dy=dy, dh_out=dh)[2]
    names = ["q", "k", "v", "b", "h0"] + (["a"] if decay else []) + (["A", "a_bias"] if decay and activate else [])
    for n in names:
        for i in rng.integers(0, x[n].size, 12):
            at = np.unravel_index(i, x[n].shape)
            want = _differences(lambda m: loss({**x, n: m}), x[n], at)
            assert abs(got["d" + n][at] - want) <= 1e-6 * (1 + abs(want)), (n, at)


def test_delta_by_hand():
    """One head of one value: S = beta k v, then what is left of v after the state's answer, forgotten by half."""
    one = lambda *x: np.array(x, np.float64).reshape(-1, 1, 1)  # noqa: E731
    y, h = od.delta(one(1, 2), one(1, 1), one(3, 5), one(0.0, np.log(0.5)), one(0.5, 0.25), None, None, 1, 1, 1.0, False, False)
    assert np.allclose(y[:, 0, 0], [1.5, 2 * (0.75 + 0.25 * (5 - 0.75))]) and np.isclose(h[0, 0, 0, 0], 0.75 + 0.25 * 4.25)


def test_keys_written_with_beta_one_are_read_back():
    rng = np.random.default_rng(1)
    k = np.eye(4)[:, None, :]
    v = rng.standard_normal((4, 1, 3))
    _, h = od.delta(k, k, v, None, np.ones((4, 1, 1)), None, None, 1, 1, 1.0, False, True, 0.0)
    y, _ = od.delta(k, k, np.zeros_like(v), None, np.zeros((4, 1, 1)), None, None, 1, 1, 1.0, False, True, 0.0, h0=h)
    assert np.allclose(y, v)


@pytest.mark.parametrize("gate,residual,group", [(True, True, 3), (False, True, 12), (True, False, 4)])
def test_join_gradients_against_differences(gate, residual, group):
    rng = np.random.default_rng(2)
    M, W = 3, 12
    n = lambda *s: rng.standard_normal(s)  # noqa: E731
    x, z, w, r, wn = n(M, W), n(M, W) if gate else None, 1 + n(W), n(M, W) if residual else None, 1 + n(W) if residual else None
    dy, dr = n(M, W), n(M, W)

    def loss(v):
        y, out, _, _ = od.join(v["x"], v["z"], v["weight"], v["residual"], v["weight_next"], group, 0.8, 1e-3)
        return (y * dy).sum() + (0.0 if out is None else (out * dr).sum())
    v = {"x": x, "z": z, "weight": w, "residual": r, "weight_next": wn}
    total = od.join(x, z, w, r, wn, group, 0.8, 1e-3)[1]
    got = od.join_backward(x, z, w, total, wn, dy, dr, group, 0.8, 1e-3)
    got = {k: v for k, v in got.items() if not k.endswith("_terms")}
    assert set(got) == {"dx", "dweight"} | ({"dz"} if gate else set()) | ({"dresidual", "dweight_next"} if residual else set())
    for k, m in v.items():
        if m is None:
            continue
        for i in rng.integers(0, m.size, 10):
            at = np.unravel_index(i, m.shape)
            want = _differences(lambda u: loss({**v, k: u}), m, at)
            assert abs(got["d" + k][at] - want) <= 1e-6 * (1 + abs(want)), (k, at)


def test_adamw_by_hand():
    p, m, v = od.adamw([1.0], [2.0], [0.0], [0.0], 0.1, 0.9, 0.99, 0.0, 0.5, 1)
    assert np.allclose([p[0], m[0], v[0]], [1.0 * 0.95 - 0.1, 0.2, 0.04])       # the first step's size is the rate


def test_codes_of_8_bits():
    assert np.allclose(od.values8([0, 1, 127, 255, 128 + 64], [2.0], True), [0, 2.25 * 2.0 ** -15, 3.75, -3.75, -2 * 2.0 ** -7])
    assert np.allclose(od.values8([0, 1, 255], [1.0], False), [0, 1.125 * 2.0 ** -31, 1.875])
    x = np.concatenate([np.linspace(-3, 3, 500), [1e-9, -1e-9, 0.0]])
    scale, low, high = od.neighbours8(x, True)
    assert (np.abs(low) <= np.abs(x) * (1 + 1e-12)).all() and (np.abs(high) >= np.abs(x) * (1 - 1e-12)).all() and scale.size == 2
    assert (np.abs(high - low) <= np.maximum(np.abs(x) / 8, 1.125 * 2.0 ** -15 * scale.max()) * (1 + 1e-12)).all()
    _, low, high = od.neighbours8(np.array([1.0, 1e-12, 0.0]), False)
    assert low[1] > 0 and high[2] == 0
