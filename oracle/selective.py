"""The operators of a selective state space block in float64 numpy: root-mean-square norm with the residual's addition, product
of 8-bit integers with scales, short causal convolution, selective scan; forward, and backward by the formulas, one
step and one sequence at a time.  Sequences are [t, B, channels]; `lengths` gives every sequence's own number of steps."""
from __future__ import annotations

import numpy as np


def _sig(x):
    return 1.0 / (1.0 + np.exp(-x))


def _f(a):
    return None if a is None else np.asarray(a, np.float64)


# ---- norm ------------------------------------------------------------------------------------------


def norm(x, residual, weight, eps):
    """(r, y, rstd)"""
    r = _f(x) if residual is None else _f(x) + _f(residual)
    rstd = 1.0 / np.sqrt((r * r).mean(1) + eps)
    return r, r * rstd[:, None] * (1.0 if weight is None else _f(weight)), rstd


def quantised(y):
    """(scale, values the 8 bits stand for, before rounding: y / scale)"""
    scale = np.abs(y).max(1) / 127.0
    return scale, y / np.where(scale > 0, scale, 1.0)[:, None]


def norm_backward(r, weight, dy, dresidual_out, eps):
    """(dr, dweight)"""
    r, dy = _f(r), _f(dy)
    rstd = 1.0 / np.sqrt((r * r).mean(1) + eps)
    n = r * rstd[:, None]
    g = dy * (1.0 if weight is None else _f(weight))
    dr = rstd[:, None] * (g - n * (g * n).mean(1)[:, None])
    return dr + (0.0 if dresidual_out is None else _f(dresidual_out)), (dy * n).sum(0)


# ---- product ---------------------------------------------------------------------------------------


def product(a, a_scale, b, b_scale, bias):
    acc = (np.asarray(a, np.int64) @ np.asarray(b, np.int64).T).astype(np.float64)
    return acc * _f(a_scale)[:, None] * _f(b_scale) + (0.0 if bias is None else _f(bias))


# ---- convolution -----------------------------------------------------------------------------------


def _ends(lengths, t, B):
    return [t] * B if lengths is None else [min(max(int(n), 0), t) for n in lengths]


def conv(x, weight, bias, lengths, state, silu):
    """(y, the last W - 1 inputs)"""
    t, B, C = x.shape
    W = weight.shape[1]
    y, last = np.zeros((t, B, C)), np.zeros((B, W - 1, C))
    for b, n in enumerate(_ends(lengths, t, B)):
        rows = np.concatenate([np.zeros((W - 1, C)) if state is None else _f(state[b]), _f(x[:n, b])])
        for s in range(n):
            pre = (rows[s:s + W] * _f(weight).T).sum(0) + (0.0 if bias is None else _f(bias))
            y[s, b] = pre * _sig(pre) if silu else pre
        last[b] = rows[n:]
    return y, last


def conv_backward(x, weight, bias, lengths, state, silu, dy, dlast):
    """(dx, dweight, dbias, dstate)"""
    t, B, C = x.shape
    W = weight.shape[1]
    w = _f(weight)
    dx, dw, db, dstate = np.zeros((t, B, C)), np.zeros((C, W)), np.zeros(C), np.zeros((B, W - 1, C))
    for b, n in enumerate(_ends(lengths, t, B)):
        rows = np.concatenate([np.zeros((W - 1, C)) if state is None else _f(state[b]), _f(x[:n, b])])
        drows = np.zeros_like(rows)
        if dlast is not None:
            drows[n:] += _f(dlast[b])
        for s in range(n):
            d = _f(dy[s, b])
            if silu:
                pre = (rows[s:s + W] * w.T).sum(0) + (0.0 if bias is None else _f(bias))
                d = d * (_sig(pre) + pre * _sig(pre) * (1 - _sig(pre)))
            drows[s:s + W] += d * w.T
            dw += (d * rows[s:s + W]).T
            db += d
        dstate[b], dx[:n, b] = drows[:W - 1], drows[W - 1:]
    return dx, dw, db, dstate


# ---- scan ------------------------------------------------------------------------------------------


def _per_channel(m, G, D):
    """[G N] -> [D, N]"""
    return np.repeat(_f(m).reshape(G, -1), D // G, axis=0)


def scan(u, delta, A, Bm, Cm, G, skip=None, z=None, delta_bias=None, lengths=None, h0=None, softplus=True):
    """(y, h_out)"""
    return _scan(u, delta, A, Bm, Cm, G, skip, z, delta_bias, lengths, h0, softplus, None, None)[:2]


def scan_backward(u, delta, A, Bm, Cm, G, skip, z, delta_bias, lengths, h0, softplus, dy, dh_out):
    """{du, ddelta, dz, dB, dC, dA, dskip, ddelta_bias, dh0}"""
    return _scan(u, delta, A, Bm, Cm, G, skip, z, delta_bias, lengths, h0, softplus, dy, dh_out)[2]


def _scan(u, delta, A, Bm, Cm, G, skip, z, delta_bias, lengths, h0, softplus, dy, dh_out):
    t, B, D = u.shape
    A = _f(A)
    N = A.shape[1]
    sk = np.zeros(D) if skip is None else _f(skip)
    y, h_out = np.zeros((t, B, D)), np.zeros((B, D, N))
    d = {k: np.zeros((t, B, D)) for k in ("du", "ddelta", "dz")}
    d.update({k: np.zeros((t, B, G * N)) for k in ("dB", "dC")})
    d.update(dA=np.zeros((D, N)), dskip=np.zeros(D), ddelta_bias=np.zeros(D), dh0=np.zeros((B, D, N)))
    for b, n in enumerate(_ends(lengths, t, B)):
        h = [np.zeros((D, N)) if h0 is None else _f(h0[b])]
        kept = []
        for s in range(n):
            raw = _f(delta[s, b]) + (0.0 if delta_bias is None else _f(delta_bias))
            w = np.logaddexp(raw, 0.0) if softplus else raw
            us, Bs, Cs = _f(u[s, b]), _per_channel(Bm[s, b], G, D), _per_channel(Cm[s, b], G, D)
            a = np.exp(w[:, None] * A)
            h.append(a * h[-1] + (w * us)[:, None] * Bs)
            core = (h[-1] * Cs).sum(1) + sk * us
            zs = None if z is None else _f(z[s, b])
            y[s, b] = core if z is None else core * zs * _sig(zs)
            kept.append((raw, w, us, Bs, Cs, a, core, zs))
        h_out[b] = h[-1]
        if dy is None:
            continue
        g = np.zeros((D, N)) if dh_out is None else _f(dh_out[b])
        for s in reversed(range(n)):
            raw, w, us, Bs, Cs, a, core, zs = kept[s]
            gy = _f(dy[s, b])
            if z is not None:
                d["dz"][s, b] = gy * core * (_sig(zs) + zs * _sig(zs) * (1 - _sig(zs)))
                gy = gy * zs * _sig(zs)
            g = g + gy[:, None] * Cs
            d["dC"][s, b] = (gy[:, None] * h[s + 1]).reshape(G, D // G, N).sum(1).reshape(-1)
            d["dB"][s, b] = (g * (w * us)[:, None]).reshape(G, D // G, N).sum(1).reshape(-1)
            dlog, through = g * a * h[s], (g * Bs).sum(1)
            d["du"][s, b] = w * through + sk * gy
            dw = (us * through + (dlog * A).sum(1)) * (_sig(raw) if softplus else 1.0)
            d["ddelta"][s, b] = dw
            d["dA"] += dlog * w[:, None]
            d["dskip"] += gy * us
            d["ddelta_bias"] += dw
            g = g * a
        d["dh0"][b] = g
    return y, h_out, d
