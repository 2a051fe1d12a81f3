"""The gated delta rule, the norms around a block with its gate and the residual's scale, and AdamW with states in 32 or 8 bits, in float64
numpy; forward, and backward by the formulas, one step at a time.  Sequences are [t, B, channels]; `lengths` gives every sequence's own number of steps."""
from __future__ import annotations

import numpy as np


def _f(a):
    return None if a is None else np.asarray(a, np.float64)


def _sig(x):
    return 1.0 / (1.0 + np.exp(-x))


# ---- gated delta rule ------------------------------------------------------------------------------


def _unit(m, normalise, eps):
    """(rows at length one, the factors that made them so)"""
    r = 1.0 / np.sqrt((m * m).sum(-1, keepdims=True) + eps) if normalise else np.ones_like(m[..., :1])
    return m * r, r


def delta(q, k, v, a, b, A, a_bias, Hk, H, scale=1.0, activate=True, normalise=True, eps=1e-6, lengths=None, h0=None, dy=None, dh_out=None):
    """(y, h_out) or, with a dy, (y, h_out, gradients): dq, dk, dv, da, db, dA, da_bias, dh0, and the sizes of the
    terms that dq, dk, dA and da_bias are sums of."""
    q, k, v, a, b, A, a_bias, h0, dy, dh_out = (_f(x) for x in (q, k, v, a, b, A, a_bias, h0, dy, dh_out))
    t, B, _ = v.shape
    dk, dv, group = q.shape[2] // Hk, v.shape[2] // H, H // Hk
    heads = lambda m, n: m.reshape(t, B, n, -1)  # noqa: E731
    wide = lambda m: np.repeat(m, group, axis=2)  # noqa: E731
    ends = np.full(B, t) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, t)
    live = np.arange(t)[:, None] < ends
    clean = lambda m: np.where(live.reshape(t, B, *[1] * (m.ndim - 2)), m, 0.0)  # noqa: E731
    (qn, qr), (kn, kr) = (_unit(clean(heads(m, Hk)), normalise, eps) for m in (q, k))
    vs = clean(heads(v, H))
    b = clean(b)
    raw = None if a is None else clean(a) + (0.0 if a_bias is None or not activate else a_bias)
    soft = None if a is None or not activate else np.logaddexp(raw, 0.0)
    g = np.zeros((t, B, H)) if a is None else A * soft if activate else raw
    beta = _sig(b) if activate else b
    qw, kw = wide(qn) * scale, wide(kn)
    S = np.zeros((B, H, dk, dv)) if h0 is None else h0.copy()
    y, kept = np.zeros((t, B, H, dv)), []
    for s in range(t):
        on = live[s][:, None, None, None]
        moved = np.exp(g[s])[..., None, None] * S
        r = vs[s] - np.einsum("bhkv,bhk->bhv", moved, kw[s])
        new = moved + kw[s][..., None] * (beta[s][..., None] * r)[:, :, None]
        y[s] = np.where(live[s][:, None, None], np.einsum("bhkv,bhk->bhv", new, qw[s]), 0.0)
        if dy is not None:
            kept.append((moved, r, new))
        S = np.where(on, new, S)
    y = y.reshape(t, B, H * dv)
    if dy is None:
        return y, S
    d = {"dq": np.zeros((t, B, Hk, dk)), "dk": np.zeros((t, B, Hk, dk)), "dv": np.zeros((t, B, H, dv)), "db": np.zeros((t, B, H)), "dg": np.zeros((t, B, H))}
    d.update({n + "_terms": np.zeros_like(d[n]) for n in ("dq", "dk")})
    dys = clean(heads(dy, H))
    G = np.zeros_like(S) if dh_out is None else dh_out.copy()
    shared = lambda m: m.reshape(B, Hk, group, dk).sum(2)  # noqa: E731
    for s in reversed(range(t)):
        on = live[s][:, None, None, None]
        moved, r, new = kept[s]
        h = G + qw[s][..., None] * dys[s][:, :, None]
        into = np.einsum("bhkv,bhk->bhv", h, kw[s])
        dr = beta[s][..., None] * into
        back = lambda m, n, f: f * (m - n * (m * n).sum(-1, keepdims=True)) if normalise else m  # noqa: E731
        dqs = shared(np.einsum("bhkv,bhv->bhk", new, dys[s])) * scale
        dks = shared(np.einsum("bhkv,bhv->bhk", h, beta[s][..., None] * r) - np.einsum("bhkv,bhv->bhk", moved, dr))
        dmoved = h - kw[s][..., None] * dr[:, :, None]
        mask = live[s][:, None, None]
        d["dq"][s], d["dk"][s] = np.where(mask, back(dqs, qn[s], qr[s]), 0.0), np.where(mask, back(dks, kn[s], kr[s]), 0.0)
        for n, m, unit, f in (("dq", dqs, qn[s], qr[s]), ("dk", dks, kn[s], kr[s])):
            d[n + "_terms"][s] = np.where(mask, f * (np.abs(m) + np.abs(unit * (m * unit).sum(-1, keepdims=True))), 0.0)
        d["dv"][s], d["db"][s] = np.where(mask, dr, 0.0), np.where(live[s][:, None], (into * r).sum(2), 0.0)
        d["dg"][s] = np.where(live[s][:, None], (dmoved * moved).sum((2, 3)), 0.0)
        G = np.where(on, dmoved * np.exp(g[s])[..., None, None], G)
    out = {n: d[n].reshape(t, B, -1) for n in ("dq", "dk", "dv", "dq_terms", "dk_terms")}
    out["db"] = d["db"] * beta * (1.0 - beta) if activate else d["db"]
    out["dh0"] = G
    if a is not None:
        out["da"] = d["dg"] * A * _sig(raw) * live[..., None] if activate else d["dg"]
        if activate:
            out.update(dA=(d["dg"] * soft * live[..., None]).sum((0, 1)), da_bias=out["da"].sum((0, 1)), dA_terms=np.abs(d["dg"] * soft * live[..., None]).sum((0, 1)),
                       da_bias_terms=np.abs(out["da"]).sum((0, 1)))
    return y, S, out


# ---- norms around a block --------------------------------------------------------------------------


def join(x, z, weight, residual, weight_next, group, scale, eps):
    """(y, r or None, rstd, rstd_next or None)"""
    x = _f(x)
    M, W = x.shape
    rstd = 1.0 / np.sqrt((x.reshape(M, -1, group) ** 2).mean(2) + eps)
    branch = x * np.repeat(rstd, group, axis=1) * (1.0 if weight is None else _f(weight)) * (1.0 if z is None else _f(z) * _sig(_f(z)))
    if residual is None:
        return branch, None, rstd, None
    r = scale * _f(residual) + branch
    rn = 1.0 / np.sqrt((r * r).mean(1) + eps)
    return r * rn[:, None] * (1.0 if weight_next is None else _f(weight_next)), r, rstd, rn


def join_backward(x, z, weight, r, weight_next, dy, dresidual_out, group, scale, eps):
    """{dx, dz, dweight, dresidual, dweight_next}; r None: there was no residual.  And for each but the last the sizes of the terms that it is a sum of
    ("dx_terms", ...): what a norm takes away may be nearly all."""
    x, d = _f(x), _f(dy)
    M, W = x.shape
    got, size = {}, np.abs(d)
    if r is not None:
        r = _f(r)
        rn = 1.0 / np.sqrt((r * r).mean(1, keepdims=True) + eps)
        m = r * rn
        got["dweight_next"] = (d * m).sum(0)
        g = d * (1.0 if weight_next is None else _f(weight_next))
        more = 0.0 if dresidual_out is None else _f(dresidual_out)
        away = m * (g * m).mean(1, keepdims=True)
        d, size = rn * (g - away) + more, rn * (np.abs(g) + np.abs(away)) + np.abs(more)
        got.update(dresidual=scale * d, dresidual_terms=scale * size)
    rstd = np.repeat(1.0 / np.sqrt((x.reshape(M, -1, group) ** 2).mean(2) + eps), group, axis=1)
    n, w = x * rstd, np.ones(W) if weight is None else _f(weight)
    act = 1.0
    if z is not None:
        z = _f(z)
        sg = _sig(z)
        act, slope = z * sg, sg + z * sg * (1.0 - sg)
        got.update(dz=d * n * w * slope, dz_terms=size * np.abs(n * w) * (sg + np.abs(z * sg * (1.0 - sg))))
    got.update(dweight=(d * n * act).sum(0), dweight_terms=(size * np.abs(n * act)).sum(0))
    g, size = d * w * act, size * np.abs(w * act)
    mean = lambda m: np.repeat(m.reshape(M, -1, group).mean(2), group, axis=1)  # noqa: E731
    got.update(dx=rstd * (g - n * mean(g * n)), dx_terms=rstd * (size + np.abs(n) * mean(size * np.abs(n))))
    return got


# ---- AdamW -----------------------------------------------------------------------------------------

BLOCK = 256


def adamw(p, g, m, v, rate, beta1, beta2, eps, decay, step):
    """(param, m, v)"""
    p, g, m, v = (_f(x) for x in (p, g, m, v))
    m, v = beta1 * m + (1.0 - beta1) * g, beta2 * v + (1.0 - beta2) * g * g
    return p * (1.0 - rate * decay) - rate * (m / (1.0 - beta1 ** step)) / (np.sqrt(v / (1.0 - beta2 ** step)) + eps), m, v


def values8(code, scale, signed):
    """What codes of one tensor stand for."""
    code = np.asarray(code, np.int64)
    low = code & 127 if signed else code
    size = np.where(low == 0, 0.0, 2.0 ** ((low >> 3) - (15.0 if signed else 31.0)) * (1.0 + (low & 7) / 8.0))
    size = size * np.repeat(_f(scale), BLOCK)[:code.size]
    return np.where(code >= 128, -size, size) if signed else size


def neighbours8(x, signed):
    """(scales, the values below and above each x that a code can stand for)"""
    n = x.size
    blocks = np.pad(np.abs(x), (0, -n % BLOCK)).reshape(-1, BLOCK)
    scale = blocks.max(1) / 1.875
    s = np.repeat(np.where(scale > 0, scale, 1.0), BLOCK)[:n]
    codes = np.arange(128 if signed else 256)
    table = values8(codes, np.ones(2), signed)[:codes.size]
    u = np.minimum(np.abs(x) / s, table[-1])
    at = np.clip(np.searchsorted(table, u, side="right") - 1, 0, table.size - 1)
    low, high = table[at], table[np.minimum(at + (u > table[at]), table.size - 1)]
    if not signed:      # never zero unless it is
        low = np.where((u > 0) & (low == 0), high, low)
    return scale, np.sign(x) * low * s, np.sign(x) * high * s
