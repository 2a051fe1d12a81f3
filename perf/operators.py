"""Operators of a selective state space block, as cases that a timing harness can run.

Four operators stand in the block and each is reached through its own entry points: the
root-mean-square norm with the residual's addition ("norm", "norm8" with an output in 8 bits, "norm
grad"), the product of 8-bit integers with scales ("product"), the short causal convolution ("conv",
"conv grad", "conv token") and the selective scan ("scan", "scan grad", "scan token").

Sequences are time-major, [t, B, channels], as everywhere in this package.  ``own`` False computes an
operator from elementary torch operations in 32 bits; ``own`` True calls the library.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _case(name, what, **kw):
    return {"name": name, "what": what, **kw}


def listed():
    return [
        # one token of a stack as wide as the smallest named core, its norm in 8 bits for the product that follows
        _case("norm8 token", "norm8", rows=4, width=1024, dtype="bf16", residual="bf16"),
        # prompts of a core of width 4096, batch 32: rows enough to fill the chip, an 8-bit output
        _case("norm8 prompt", "norm8", rows=8192, width=4096, dtype="bf16", residual="fp32"),
        # a gradient step of the headline workload's size, forward and backward: 1000 steps x 64 sequences, residual stream in fp32
        _case("norm train", "norm grad", rows=64000, width=1024, dtype="bf16", residual="fp32"),
        # one token each for 32 sequences through four gates' worth of rows: the weights' bytes are everything
        _case("product token", "product", M=32, N=16384, K=4096, dtype="bf16", bias=False),
        # a prompt batch: a large matrix product
        _case("product prompt", "product", M=8192, N=4096, K=4096, dtype="bf16", bias=False),
        # a stack's inner layer whose sizes are a multiple of nothing, fp32 out with a bias
        _case("product ragged", "product", M=777, N=1301, K=650, dtype="fp32", bias=True),
        # a gradient step through the convolution, the inner width twice the model's
        _case("conv train", "conv grad", t=1000, B=64, C=2048, taps=4, dtype="bf16", lengths=False, state=False),
        # single tokens for a batch of running sequences
        _case("conv token", "conv token", B=256, C=2048, taps=4, dtype="bf16"),
        # one very long prompt: only a split of the time axis fills the chip
        _case("scan prompt", "scan", t=10000, B=1, D=2048, N=16, G=1, dtype="bf16", gate=True, lengths=False, state=True, stretch=0),
        # a gradient step, states kept every 64 steps
        _case("scan train", "scan grad", t=1000, B=32, D=1024, N=16, G=1, dtype="bf16", gate=True, lengths=False, state=False, stretch=64),
        # prompts of unequal lengths (none and one among them), sizes a multiple of nothing, fp32
        _case("scan ragged", "scan", t=333, B=20, D=650, N=13, G=2, dtype="fp32", gate=False, lengths=True, state=True, stretch=0),
        # single tokens for a batch of running sequences, their states in a pool
        _case("scan token", "scan token", B=256, D=2048, N=16, G=1, dtype="bf16", gate=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of all widths are round, half are whatever they are."""
    v = _log(rng, lo, hi)
    if rng.random() < 0.5:
        step = 64 if v >= 128 else 16
        v = max(step, (v + step // 2) // step * step)
    return max(lo, min(hi, v))


def _limits(case):
    w = work(case)
    if case["what"] == "product":
        return w["flops"] <= 2.8e11
    if case["what"].startswith("scan"):
        return w["flops"] <= 1.2e10 and w["bytes"] <= 1.2e9
    return w["bytes"] <= 1.2e9


def draw(rng):
    while True:
        what = rng.choice(["norm8", "norm grad", "product", "conv grad", "conv token", "scan", "scan grad", "scan token"])
        dtype = "fp32" if rng.random() < 0.3 else "bf16"
        if what.startswith("norm"):
            c = _case("", what, rows=_log(rng, 1, 64000), width=_size(rng, 64, 8192), dtype=dtype,
                      residual="fp32" if what == "norm grad" or rng.random() < 0.5 else "bf16")
        elif what == "product":
            c = _case("", what, M=_log(rng, 1, 8192), N=_size(rng, 64, 16384), K=_size(rng, 64, 4096), dtype=dtype,
                      bias=rng.random() < 0.5)
        elif what == "conv token":
            c = _case("", what, B=_log(rng, 1, 256), C=_size(rng, 64, 8192), taps=rng.randint(2, 4), dtype=dtype)
        elif what == "conv grad":
            c = _case("", what, t=_log(rng, 1, 10000), B=_log(rng, 1, 64), C=_size(rng, 64, 4096), taps=rng.randint(2, 4),
                      dtype=dtype, lengths=rng.random() < 0.4, state=rng.random() < 0.5)
        elif what == "scan token":
            G = rng.choice([1, 1, 2])
            c = _case("", what, B=_log(rng, 1, 256), D=_size(rng, 32, 4096 // G) * G, N=rng.randint(4, 32) if rng.random() < 0.5 else 16,
                      G=G, dtype=dtype, gate=rng.random() < 0.7)
        else:
            G = rng.choice([1, 1, 2])
            c = _case("", what, t=_log(rng, 1, 10000), B=_log(rng, 1, 64), D=_size(rng, 32, 4096 // G) * G,
                      N=rng.randint(4, 32) if rng.random() < 0.5 else 16, G=G, dtype=dtype, gate=rng.random() < 0.7,
                      lengths=rng.random() < 0.4, state=rng.random() < 0.5, stretch=rng.choice([16, 64, 128]) if what == "scan grad" else 0)
        del c["name"]
        if _limits(c):
            return c


# ---- inputs -------------------------------------------------------------------------------------


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 1000003 + 29)

    def normal(self, *shape, s=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.g, device="cuda") * s).to(dtype)

    def uniform(self, *shape, lo=0.0, hi=1.0):
        return lo + (hi - lo) * torch.rand(shape, generator=self.g, device="cuda")

    def whole(self, *shape):
        """8-bit values of a normal distribution whose largest is near 127, as a quantised row's are."""
        return torch.clamp(torch.round(torch.randn(shape, generator=self.g, device="cuda") * 34.0), -127, 127).to(torch.int8)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _lengths(case):
    """None, one, and everything between up to t."""
    t, B = case["t"], case["B"]
    return [t] if B == 1 else [1 if b == 1 and t > 0 else (t * b) // (B - 1) for b in range(B)]


def _inputs(case, seed):
    d, dt = _Draw(seed), DTYPES[case["dtype"]]
    what = case["what"]
    if what.startswith("norm"):
        M, W = case["rows"], case["width"]
        v = {"x": d.normal(M, W, s=0.7, dtype=dt), "residual": d.normal(M, W, s=2.0, dtype=DTYPES[case["residual"]]),
             "weight": 1.0 + d.normal(W, s=0.2)}
        if what == "norm grad":
            v["dy"] = d.normal(M, W, s=0.1, dtype=dt)
            v["dresidual"] = d.normal(M, W, s=0.1, dtype=DTYPES[case["residual"]])
        return v
    if what == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"a": d.whole(M, K), "b": d.whole(N, K), "a_scale": d.uniform(M, lo=0.01, hi=0.05),
                "b_scale": d.uniform(N, lo=0.0005, hi=0.002), "bias": d.normal(N) if case["bias"] else None}
    t, B = case.get("t", 1), case["B"]
    if what.startswith("conv"):
        C, W = case["C"], case["taps"]
        k = W ** -0.5
        v = {"x": d.normal(t, B, C, dtype=dt), "weight": d.uniform(C, W, lo=-k, hi=k), "bias": d.uniform(C, lo=-k, hi=k)}
        if what == "conv token":
            v["state"] = d.normal(B + 3, W - 1, C, dtype=dt)
            v["index"] = d.order(B + 3)[:B].to(torch.int32)
            return v
        v["state"] = d.normal(B, W - 1, C, dtype=dt) if case["state"] else None
        v["dy"] = d.normal(t, B, C, s=0.1, dtype=dt)
        v["dstate_out"] = d.normal(B, W - 1, C, s=0.1, dtype=dt) if case["state"] else None
        v["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["lengths"] else None
        return v
    D, N, G = case["D"], case["N"], case["G"]
    first = torch.exp(d.uniform(D, lo=math.log(1e-3), hi=math.log(0.1)))
    v = {"u": d.normal(t, B, D, s=0.6, dtype=dt), "delta": d.normal(t, B, D, s=0.5, dtype=dt),
         "A": -torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * torch.exp(d.normal(D, N, s=0.1)),
         "Bm": d.normal(t, B, G * N, dtype=dt), "Cm": d.normal(t, B, G * N, dtype=dt), "skip": 1.0 + d.normal(D, s=0.1),
         "delta_bias": first + torch.log(-torch.expm1(-first)), "z": d.normal(t, B, D, dtype=dt) if case["gate"] else None}
    if what == "scan token":
        v["state"] = d.normal(B + 3, D, N, s=0.3)
        v["index"] = d.order(B + 3)[:B].to(torch.int32)
        return v
    v["h0"] = d.normal(B, D, N, s=0.3) if case["state"] else None
    v["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["lengths"] else None
    if what == "scan grad":
        v["dy"] = d.normal(t, B, D, s=0.1, dtype=dt)
        v["dh_out"] = d.normal(B, D, N, s=0.1) if case["state"] else None
    return v


def _bytes(n):
    return torch.zeros(max(int(n), 256), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    return {"case": dict(case), "kept": {}, **_inputs(case, seed)}


def _kept(s, make):
    """Outputs, workspaces and descriptors that a user's program makes once and hands to every call."""
    if not s["kept"]:
        s["kept"].update(make())
    return s["kept"]


# ---- the library's calls ------------------------------------------------------------------------


def _own_norm(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]
    code = {"fp32": mb.FP32, "bf16": mb.BF16}
    like = torch.empty_like
    if c["what"] == "norm8":
        k = _kept(s, lambda: {"desc": mb.make_norm_desc(c["rows"], c["width"], code[c["dtype"]], code[c["residual"]], mb.INT8, EPS),
                              "q": torch.empty(s["x"].shape, dtype=torch.int8, device="cuda"),
                              "scale": torch.empty(c["rows"], device="cuda"), "sum": like(s["residual"]),
                              "y": torch.empty(s["x"].shape, dtype=torch.bfloat16, device="cuda")})
        mb.mebptt_norm_forward(k["desc"], s["x"], s["residual"], s["weight"], k["q"], k["scale"], k["sum"], None)
        torch.mul(k["q"], k["scale"][:, None], out=k["y"])
        return {"y": k["y"], "scale": k["scale"], "sum": k["sum"]}

    def make():
        desc = mb.make_norm_desc(c["rows"], c["width"], code[c["dtype"]], code[c["residual"]], code[c["dtype"]], EPS)
        return {"desc": desc, "y": like(s["x"]), "sum": like(s["residual"]), "rstd": torch.empty(c["rows"], device="cuda"),
                "dx": like(s["x"]), "dsum": like(s["residual"]), "dweight": like(s["weight"]),
                "ws": _bytes(mb.mebptt_norm_workspace_bytes(desc))}
    k = _kept(s, make)
    mb.mebptt_norm_forward(k["desc"], s["x"], s["residual"], s["weight"], k["y"], None, k["sum"], k["rstd"])
    mb.mebptt_norm_backward(k["desc"], k["sum"], s["weight"], k["rstd"], s["dy"], s["dresidual"], k["dx"], k["dsum"],
                            k["dweight"], k["ws"])
    return {n: k[n] for n in ("y", "sum", "dx", "dsum", "dweight")}


def _own_product(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]

    def make():
        desc = mb.make_int8_desc(c["M"], c["N"], c["K"], mb.BF16 if c["dtype"] == "bf16" else mb.FP32)
        return {"desc": desc, "out": torch.empty((c["M"], c["N"]), dtype=DTYPES[c["dtype"]], device="cuda"),
                "ws": _bytes(mb.mebptt_int8_workspace_bytes(desc))}
    k = _kept(s, make)
    mb.mebptt_int8_product(k["desc"], s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], k["out"], k["ws"])
    return {"out": k["out"]}


def _own_conv(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]

    def make():
        desc = mb.make_conv_desc(c.get("t", 1), c["B"], c["C"], c["taps"], mb.BF16 if c["dtype"] == "bf16" else mb.FP32, 1)
        k = {"desc": desc, "y": torch.empty_like(s["x"])}
        if c["what"] == "conv token":
            return {**k, "state": torch.zeros_like(s["state"])}
        state = torch.empty((c["B"], c["taps"] - 1, c["C"]), dtype=s["x"].dtype, device="cuda")
        return {**k, "state": state, "dx": torch.empty_like(s["x"]), "dweight": torch.empty_like(s["weight"]),
                "dbias": torch.empty_like(s["bias"]), "dstate": torch.empty_like(state) if c["state"] else None,
                "ws": _bytes(mb.mebptt_conv_workspace_bytes(desc))}
    k = _kept(s, make)
    if c["what"] == "conv token":
        mb.mebptt_conv_step(k["desc"], s["x"][0], s["weight"], s["bias"], s["state"], s["index"], k["y"][0], k["state"])
        return {"y": k["y"], "state": k["state"]}
    mb.mebptt_conv_forward(k["desc"], s["x"], s["weight"], s["bias"], s["lengths"], s["state"], k["y"], k["state"])
    mb.mebptt_conv_backward(k["desc"], s["x"], s["weight"], s["bias"], s["lengths"], s["state"], s["dy"], s["dstate_out"],
                            k["dx"], k["dweight"], k["dbias"], k["dstate"], k["ws"])
    return {n: k[n] for n in ("y", "state", "dx", "dweight", "dbias") + (("dstate",) if c["state"] else ())}


def _own_scan(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]
    like = torch.empty_like

    def make():
        desc = mb.make_scan_desc(c.get("t", 1), c["B"], c["D"], c["N"], c["G"], mb.BF16 if c["dtype"] == "bf16" else mb.FP32, 1,
                                 c.get("stretch", 0))
        k = {"desc": desc, "y": like(s["u"])}
        if c["what"] == "scan token":
            return {**k, "state": torch.zeros_like(s["state"])}
        k |= {"h_out": torch.empty((c["B"], c["D"], c["N"]), device="cuda"), "states": None,
              "ws": _bytes(mb.mebptt_scan_workspace_bytes(desc, c["what"] == "scan grad"))}
        if c["what"] == "scan grad":
            k |= {"states": _bytes(mb.mebptt_scan_state_bytes(desc)), "du": like(s["u"]), "ddelta": like(s["delta"]), "dA": like(s["A"]),
                  "dB": like(s["Bm"]), "dC": like(s["Cm"]), "dskip": like(s["skip"]), "ddelta_bias": like(s["delta_bias"]),
                  "dz": like(s["z"]) if c["gate"] else None, "dh0": like(s["h0"]) if c["state"] else None}
        return k
    k = _kept(s, make)
    given = (k["desc"], s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["skip"], s["z"], s["delta_bias"])
    if c["what"] == "scan token":
        mb.mebptt_scan_step(k["desc"], s["u"][0], s["delta"][0], s["A"], s["Bm"][0], s["Cm"][0], s["skip"],
                            s["z"][0] if c["gate"] else None, s["delta_bias"], s["state"], s["index"], k["y"][0], k["state"])
        return {"y": k["y"], "state": k["state"]}
    mb.mebptt_scan_forward(*given, s["lengths"], s["h0"], k["y"], k["h_out"], k["states"], k["ws"])
    if c["what"] == "scan":
        return {"y": k["y"], "h_out": k["h_out"]}
    mb.mebptt_scan_backward(*given, s["lengths"], s["h0"], s["dy"], s["dh_out"], k["states"], k["du"], k["ddelta"], k["dA"],
                            k["dB"], k["dC"], k["dskip"], k["dz"], k["ddelta_bias"], k["dh0"], k["ws"])
    names = ["y", "h_out", "du", "ddelta", "dA", "dB", "dC", "dskip", "ddelta_bias"]
    return {n: k[n] for n in names + (["dz"] if c["gate"] else []) + (["dh0"] if c["state"] else [])}


# ---- the plain forms ----------------------------------------------------------------------------


def _norm(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    r = s["x"].float() + s["residual"].float()
    rstd = torch.rsqrt((r * r).mean(1, keepdim=True) + EPS)
    n = r * rstd
    y = n * s["weight"]
    if c["what"] == "norm8":
        scale = y.abs().amax(1) / 127.0
        q = torch.round(y / torch.where(scale > 0, scale, 1.0)[:, None])
        return {"y": (q * scale[:, None]).to(torch.bfloat16), "scale": scale, "sum": r.to(s["residual"].dtype)}
    wdy = s["weight"] * s["dy"].float()
    d = rstd * (wdy - n * (wdy * n).mean(1, keepdim=True)) + s["dresidual"].float()
    return {"y": y.to(dt), "sum": r.to(s["residual"].dtype), "dx": d.to(dt), "dsum": d.to(s["residual"].dtype),
            "dweight": (s["dy"].float() * n).sum(0)}


def _product(s):
    out = (s["a"].float() @ s["b"].float().t()) * s["a_scale"][:, None] * s["b_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    return {"out": out.to(DTYPES[s["case"]["dtype"]])}


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _inside(lengths, t):
    """[t, B, 1]: whether step s is one of its sequence's own."""
    return (torch.arange(t, device="cuda")[:, None] < lengths)[:, :, None]


def _taps(x, state, W):
    """[t + W - 1, B, C]: the inputs, the state's before them."""
    before = state.float().transpose(0, 1) if state is not None else torch.zeros((W - 1,) + x.shape[1:], device="cuda")
    return torch.cat([before, x.float()])


def _last(rows, lengths, t, W):
    """The W - 1 rows before each sequence's end, [B, W - 1, C]."""
    if lengths is None:
        return rows[t:].transpose(0, 1)
    at = lengths.long()[:, None] + torch.arange(W - 1, device="cuda")
    return rows.transpose(0, 1).gather(1, at[:, :, None].expand(-1, -1, rows.shape[2]))


def _conv(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    W, w, t = c["taps"], s["weight"], s["x"].shape[0]
    if c["what"] == "conv token":
        i = s["index"].long()
        rows = torch.cat([s["state"][i].float(), s["x"][0].float()[:, None]], 1)
        pre = (rows * w.t()).sum(1) + s["bias"]
        state = torch.zeros_like(s["state"])
        state[i] = rows[:, 1:].to(dt)
        return {"y": (pre * _sigmoid(pre)).to(dt)[None], "state": state}
    rows = _taps(s["x"], s["state"], W)
    pre = s["bias"].clone()
    pre = sum((rows[j:j + t] * w[:, j] for j in range(W)), pre)
    sg = _sigmoid(pre)
    y, dpre = pre * sg, s["dy"].float() * sg * (1.0 + pre * (1.0 - sg))
    if s["lengths"] is not None:
        inside = _inside(s["lengths"], t)
        y, dpre = torch.where(inside, y, 0.0), torch.where(inside, dpre, 0.0)
    state = _last(rows, s["lengths"], t, W).to(dt)
    drows = torch.zeros_like(rows)
    dweight = torch.empty_like(w)
    for j in range(W):
        drows[j:j + t] += dpre * w[:, j]
        dweight[:, j] = (dpre * rows[j:j + t]).sum((0, 1))
    if c["state"]:
        ends = s["lengths"].long() if s["lengths"] is not None else torch.full((c["B"],), t, device="cuda")
        at = ends[None, :] + torch.arange(W - 1, device="cuda")[:, None]
        drows.scatter_add_(0, at[:, :, None].expand(-1, -1, c["C"]), s["dstate_out"].float().transpose(0, 1).contiguous())
    out = {"y": y.to(dt), "state": state, "dx": drows[W - 1:].to(dt), "dweight": dweight, "dbias": dpre.sum((0, 1))}
    if c["state"]:
        out["dstate"] = drows[:W - 1].transpose(0, 1).to(dt)
    return out


def _prefix(a, x, first):
    """h_s = a_s h_{s-1} + x_s over the first axis from h = `first`, by doubling."""
    h, k = x.clone(), 1
    if first is not None and h.shape[0]:
        h[0] += a[0] * first
    while k < h.shape[0]:
        h[k:] += a[k:] * h[:-k].clone()
        if 2 * k < h.shape[0]:
            a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return h


def _wide(m, c):
    """[.., G N] -> [.., D, N]: a channel's group."""
    G, N = c["G"], c["N"]
    return m.float().unflatten(-1, (G, N)).repeat_interleave(c["D"] // G, -2)


def _scan(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    raw = s["delta"].float() + s["delta_bias"]
    delta = torch.clamp(raw, min=0.0) + torch.log1p(torch.exp(-raw.abs()))
    u, t, A = s["u"].float(), s["u"].shape[0], s["A"]
    z = s["z"].float() if c["gate"] else None
    if c["what"] == "scan token":
        i = s["index"].long()
        h = torch.exp(delta[0][..., None] * A) * s["state"][i] + (delta * u)[0][..., None] * _wide(s["Bm"][0], c)
        y = (h * _wide(s["Cm"][0], c)).sum(-1) + s["skip"] * u[0]
        state = torch.zeros_like(s["state"])
        state[i] = h
        return {"y": (y * z[0] * _sigmoid(z[0]) if c["gate"] else y).to(dt)[None], "state": state}
    inside = None if s["lengths"] is None else _inside(s["lengths"], t)
    if inside is not None:
        delta = torch.where(inside, delta, 0.0)
    a, Bw, Cw = torch.exp(delta[..., None] * A), _wide(s["Bm"], c), _wide(s["Cm"], c)
    h = _prefix(a, (delta * u)[..., None] * Bw, s["h0"])
    core = (h * Cw).sum(-1) + s["skip"] * u
    y = core * z * _sigmoid(z) if c["gate"] else core
    if inside is not None:
        y = torch.where(inside, y, 0.0)
    h_out = h[-1] if t else s["h0"]
    if c["what"] == "scan":
        return {"y": y.to(dt), "h_out": h_out.clone()}
    dy = s["dy"].float()
    if inside is not None:
        dy = torch.where(inside, dy, 0.0)
    out = {"y": y.to(dt), "h_out": h_out.clone()}
    if c["gate"]:
        sg = _sigmoid(z)
        out["dz"] = (dy * core * sg * (1.0 + z * (1.0 - sg))).to(dt)
        dy = dy * z * sg
    per_group = lambda m: m.unflatten(-2, (c["G"], c["D"] // c["G"])).sum(-2).flatten(-2)  # noqa: E731
    out["dC"] = per_group(dy[..., None] * h).to(dt)
    # g_s = C_s dy_s + a_{s+1} g_{s+1}: the same recurrence from the last step back
    into = dy[..., None] * Cw
    if s["dh_out"] is not None:
        into[-1] += s["dh_out"]
    g = _prefix(torch.cat([torch.zeros_like(a[:1]), a[1:].flip(0)]), into.flip(0), None).flip(0)
    out["dB"] = per_group((delta * u)[..., None] * g).to(dt)
    before = torch.cat([(s["h0"] if s["h0"] is not None else torch.zeros_like(h[0]))[None], h[:-1]])
    r, p = g * a * before, (g * Bw).sum(-1)
    out["dA"] = (delta[..., None] * r).sum((0, 1))
    du = delta * p + s["skip"] * dy
    draw = (u * p + (r * A).sum(-1)) * _sigmoid(raw)
    if inside is not None:
        draw = torch.where(inside, draw, 0.0)
    out |= {"du": du.to(dt), "ddelta": draw.to(dt), "dskip": (dy * u).sum((0, 1)), "ddelta_bias": draw.sum((0, 1))}
    if c["state"]:
        out["dh0"] = g[0] * a[0]
    return out


def run(state):
    kind = state["case"]["what"].split()[0].rstrip("8")
    if own:
        return {"norm": _own_norm, "product": _own_product, "conv": _own_conv, "scan": _own_scan}[kind](state)
    return {"norm": _norm, "product": _product, "conv": _conv, "scan": _scan}[kind](state)


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    e = 4.0 if case["dtype"] == "fp32" else 2.0
    what = case["what"]
    if what.startswith("norm"):
        r = 4.0 if case["residual"] == "fp32" else 2.0
        n = float(case["rows"]) * case["width"]
        if what == "norm8":
            return {"bytes": n * (e + 2 * r + 1) + 4.0 * case["width"], "flops": 7.0 * n}
        # x, residual, dy and the sum's gradient in; y, sum, dx and the residual's gradient out
        return {"bytes": n * (4 * e + 4 * r) + 8.0 * case["width"], "flops": 16.0 * n}
    if what == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + e * M * N + 4.0 * (M + N), "flops": 2.0 * M * N * K}
    t, B = case.get("t", 1), case["B"]
    if what.startswith("conv"):
        C, W = case["C"], case["taps"]
        n = float(t) * B * C
        params = 4.0 * C * (W + 1)
        if what == "conv token":
            return {"bytes": n * e * (2 + 2 * (W - 1)) + params, "flops": n * (2 * W + 5)}
        state = e * B * C * (W - 1) * (3 if case["state"] else 1)
        return {"bytes": 4 * n * e + 2 * params + state, "flops": n * (6 * W + 14)}
    D, N, G = case["D"], case["N"], case["G"]
    n, gate = float(t) * B * D, 1 if case["gate"] else 0
    state, params = 4.0 * B * D * N, 4.0 * D * (N + 2)
    if what == "scan token":
        return {"bytes": e * n * (3 + gate) + e * 2 * B * G * N + 2 * state + params, "flops": n * (7.0 * N + 15)}
    shared = e * 2 * t * B * G * N
    given = 1 if case["state"] else 0
    if what == "scan":
        return {"bytes": e * n * (3 + gate) + shared + (1 + given) * state + params, "flops": n * (7.0 * N + 15)}
    return {"bytes": e * n * (6 + 2 * gate) + 2 * shared + (1 + 3 * given) * state + 2 * params, "flops": n * (22.0 * N + 40)}


# ---- the same in 64 bits ------------------------------------------------------------------------


def _exact_norm(case, v):
    total = v["x"].double() + v["residual"].double()
    size = torch.sqrt(total.square().mean(1, keepdim=True) + EPS)
    unit = total / size
    y = unit * v["weight"].double()
    if case["what"] == "norm8":
        return {"y": y, "scale": y.abs().max(1).values / 127, "sum": total}
    into = v["dy"].double() * v["weight"].double()
    dsum = (into - unit * (into * unit).mean(1, keepdim=True)) / size + v["dresidual"].double()
    return {"y": y, "sum": total, "dx": dsum, "dsum": dsum, "dweight": (v["dy"].double() * unit).sum(0)}


def _exact_product(case, v):
    out, b = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda"), v["b"].double()
    for i in range(0, case["M"], 1024):
        out[i:i + 1024] = v["a"][i:i + 1024].double() @ b.t()
    out *= torch.outer(v["a_scale"].double(), v["b_scale"].double())
    return {"out": out if v["bias"] is None else out + v["bias"].double()}


def _exact_conv(case, v):
    W, w, b = case["taps"], v["weight"].double(), v["bias"].double()
    if case["what"] == "conv token":
        state, y = torch.zeros_like(v["state"], dtype=torch.float64), torch.empty_like(v["x"], dtype=torch.float64)
        old = v["state"].double()[v["index"].long()]
        pre = b + v["x"][0].double() * w[:, W - 1]
        for j in range(W - 1):
            pre = pre + old[:, j] * w[:, j]
        y[0] = pre * torch.sigmoid(pre)
        state[v["index"].long()] = torch.cat([old[:, 1:], v["x"].double().transpose(0, 1)], 1)
        return {"y": y, "state": state}
    t, B, C = v["x"].shape
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    got = {"y": zeros(t, B, C), "state": zeros(B, W - 1, C), "dx": zeros(t, B, C), "dweight": zeros(C, W), "dbias": zeros(C),
           "dstate": zeros(B, W - 1, C)}
    for i in range(B):   # a sequence at a time, each of its own length
        n = _lengths(case)[i] if case["lengths"] else t
        x = torch.cat([v["state"][i].double() if case["state"] else zeros(W - 1, C), v["x"][:n, i].double()])
        pre = b.expand(n, C).clone()
        for j in range(W):
            pre += w[:, j] * x[j:j + n]
        sg = torch.sigmoid(pre)
        got["y"][:n, i] = pre * sg
        got["state"][i] = x[n:]
        dpre = v["dy"][:n, i].double() * (sg + pre * sg * (1 - sg))
        dx = torch.zeros_like(x)
        if case["state"]:
            dx[n:] += v["dstate_out"][i].double()
        for j in range(W):
            dx[j:j + n] += w[:, j] * dpre
            got["dweight"][:, j] += (dpre * x[j:j + n]).sum(0)
        got["dbias"] += dpre.sum(0)
        got["dx"][:n, i] = dx[W - 1:W - 1 + n]
        got["dstate"][i] = dx[:W - 1]
    if not case["state"]:
        del got["dstate"]
    return got


def _exact_scan(case, v):
    D, N, G = case["D"], case["N"], case["G"]
    A, skip = v["A"].double(), v["skip"].double()
    group = torch.arange(D, device="cuda") // (D // G)
    t, B = v["u"].shape[0], case["B"]

    def at(s):
        raw = v["delta"][s].double() + v["delta_bias"].double()
        delta = torch.logaddexp(raw, torch.zeros_like(raw))
        pick = lambda m: m[s].double().view(B, G, N)[:, group]  # noqa: E731
        z = v["z"][s].double() if case["gate"] else None
        return raw, delta, v["u"][s].double(), pick(v["Bm"]), pick(v["Cm"]), z

    def forward(s, h):
        raw, delta, u, Bs, Cs, z = at(s)
        new = torch.exp(delta[:, :, None] * A) * h + (delta * u)[:, :, None] * Bs
        core = torch.matmul(new[:, :, None, :], Cs[:, :, :, None])[:, :, 0, 0] + skip * u
        return new, core, (core * z * torch.sigmoid(z) if case["gate"] else core)

    if case["what"] == "scan token":
        i = v["index"].long()
        new, _, y = forward(0, v["state"].double()[i])
        state = torch.zeros_like(v["state"], dtype=torch.float64)
        state[i] = new
        return {"y": y[None], "state": state}
    live = [None] * t
    if case["lengths"]:
        ends = v["lengths"]
        live = [(ends > s)[:, None] for s in range(t)]
    h = v["h0"].double() if case["state"] else torch.zeros((B, D, N), dtype=torch.float64, device="cuda")
    back = case["what"] == "scan grad"
    if back and float(t) * B * D * N > 2.0e9:
        return None
    ys, hs, cores = torch.zeros((t, B, D), dtype=torch.float64, device="cuda"), [h], []
    for s in range(t):
        new, core, y = forward(s, h)
        h = new if live[s] is None else torch.where(live[s][:, :, None], new, h)
        ys[s] = y if live[s] is None else torch.where(live[s], y, 0.0)
        if back:
            hs.append(h)
            cores.append(core)
    if not back:
        return {"y": ys, "h_out": h}
    got = {"y": ys, "h_out": h, "dA": torch.zeros_like(A), "dskip": torch.zeros_like(skip), "ddelta_bias": torch.zeros_like(skip)}
    got |= {k: torch.zeros((t, B, D), dtype=torch.float64, device="cuda") for k in ("du", "ddelta", "dz")}
    got |= {k: torch.zeros((t, B, G * N), dtype=torch.float64, device="cuda") for k in ("dB", "dC")}
    g = v["dh_out"].double() if case["state"] else torch.zeros_like(h)
    for s in reversed(range(t)):
        raw, delta, u, Bs, Cs, z = at(s)
        dy = v["dy"][s].double()
        if live[s] is not None:
            dy, delta = torch.where(live[s], dy, 0.0), torch.where(live[s], delta, 0.0)
        if case["gate"]:
            sg = torch.sigmoid(z)
            got["dz"][s] = dy * cores[s] * (sg + z * sg * (1 - sg))
            dy = dy * z * sg
        a = torch.exp(delta[:, :, None] * A)
        g = g + dy[:, :, None] * Cs
        got["dC"][s] = (dy[:, :, None] * hs[s + 1]).view(B, G, D // G, N).sum(2).view(B, G * N)
        got["dB"][s] = ((delta * u)[:, :, None] * g).view(B, G, D // G, N).sum(2).view(B, G * N)
        dlog = g * a * hs[s]
        through = (g * Bs).sum(2)
        got["du"][s] = delta * through + skip * dy
        dd = (u * through + (dlog * A).sum(2)) * torch.sigmoid(raw)
        got["ddelta"][s] = dd if live[s] is None else torch.where(live[s], dd, 0.0)
        got["dA"] += (dlog * delta[:, :, None]).sum(0)
        got["dskip"] += (dy * u).sum(0)
        g = g * a
        hs[s + 1] = None
    got["ddelta_bias"] = got["ddelta"].sum((0, 1))
    got["dh0"] = g
    for k, there in (("dz", case["gate"]), ("dh0", case["state"])):
        if not there:
            del got[k]
    return got


def exact(case, seed):
    v = _inputs(case, seed)
    kind = case["what"].split()[0].rstrip("8")
    return {"norm": _exact_norm, "product": _exact_product, "conv": _exact_conv, "scan": _exact_scan}[kind](case, v)
