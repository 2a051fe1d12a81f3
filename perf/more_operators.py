"""Operators of a block with a matrix for a state, and of the step that trains it, as cases that a timing harness can run.

Three operators, each reached through its own entry points: the gated delta rule ("delta", "delta grad", "delta
token"), the norms behind a block and before the next one with the block's gate and the residual's scale between them
("join", "join grad"), and AdamW over many tensors at once with states in 32 or 8 bits ("adamw").

Sequences are time-major, [t, B, channels], as everywhere in this package.  ``own`` False computes an
operator from elementary torch operations in 32 bits; ``own`` True calls the library.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
EPS_HEAD = 1e-6     # of the lengths of q and k
CHUNK = 64
BLOCK = 256         # values that share a scale where an optimiser's states have 8 bits
ADAM = {"rate": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "decay": 0.1, "step": 10, "seed": 12345}


def _case(name, what, **kw):
    return {"name": name, "what": what, **kw}


def listed():
    return [
        # one very long prompt: only a split of the time axis fills the chip
        _case("delta prompt", "delta", t=10000, B=1, Hk=16, H=16, dk=128, dv=128, dtype="bf16", decay=True, normalise=True, lengths=False, state=True, stretch=0),
        # a gradient step of 1000 steps x 32 sequences
        _case("delta train", "delta grad", t=1000, B=32, Hk=8, H=8, dk=128, dv=128, dtype="bf16", decay=True, normalise=True, lengths=False, state=False, stretch=256),
        # sequences of unequal lengths (none and one among them), sizes a multiple of nothing, shared heads, fp32, trained
        _case("delta ragged", "delta grad", t=333, B=20, Hk=2, H=4, dk=50, dv=75, dtype="fp32", decay=True, normalise=True, lengths=True, state=True, stretch=128),
        # single tokens for a batch of running sequences, their states in a pool
        _case("delta token", "delta token", B=256, Hk=8, H=16, dk=128, dv=128, dtype="bf16", decay=True, normalise=True),
        # one token of four sequences: latency
        _case("delta few", "delta token", B=4, Hk=4, H=4, dk=64, dv=64, dtype="bf16", decay=True, normalise=True),
        # behind the heads of a core, 1000 steps x 32 sequences of a gradient step: a norm per head and the gate
        _case("join heads", "join grad", rows=32000, width=1024, group=128, dtype="bf16", gate=True, residual="", scale=1.0),
        # between two blocks, a gradient step of the headline workload's size: a norm, the scaled residual stream in fp32, the next norm
        _case("join train", "join grad", rows=64000, width=1024, group=1024, dtype="bf16", gate=False, residual="fp32", scale=0.8),
        # prompts of a core of width 4096, every part of it
        _case("join prompt", "join", rows=8192, width=4096, group=128, dtype="bf16", gate=True, residual="bf16", scale=1.0),
        # one token of a stack as wide as the smallest named core
        _case("join token", "join", rows=4, width=1024, group=1024, dtype="bf16", gate=False, residual="fp32", scale=1.0),
        # the weights of a core 1024 -> 4096 and many small tensors beside them, states in 32 bits, gradients clipped
        _case("adamw core", "adamw", bits=32, count=40, smallest=64, largest=67108864, grad="fp32", copy=True, clip=True),
        # the same with states in 8 bits
        _case("adamw 8 bits", "adamw", bits=8, count=40, smallest=64, largest=67108864, grad="bf16", copy=True, clip=False),
        # the weights of a small stack: many tensors with little in them
        _case("adamw small", "adamw", bits=32, count=60, smallest=33, largest=65536, grad="fp32", copy=False, clip=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, step):
    """Half of all widths are round, half are whatever they are."""
    v = _log(rng, lo, hi)
    if rng.random() < 0.5:
        v = max(step, (v + step // 2) // step * step)
    return max(lo, min(hi, v))


def _limits(case):
    w = work(case)
    if case["what"].startswith("delta"):
        chunks = -(-case.get("t", 1) // CHUNK) * case["B"] * case["H"]
        return w["flops"] <= 9.0e10 and w["bytes"] <= 7.0e8 and chunks <= 4096
    return w["bytes"] <= 1.3e9


def draw(rng):
    while True:
        what = rng.choice(["delta", "delta grad", "delta token", "join", "join grad", "adamw"])
        dtype = "fp32" if rng.random() < 0.3 else "bf16"
        if what.startswith("delta"):
            Hk = rng.randint(1, 16)
            sizes = dict(B=_log(rng, 1, 256 if what == "delta token" else 64), Hk=Hk, H=Hk * rng.choice([1, 1, 2, 3]), dk=_size(rng, 16, 128, 16), dv=_size(rng, 16, 256, 16),
                         dtype=dtype, decay=rng.random() < 0.8, normalise=rng.random() < 0.8)
            if what == "delta token":
                c = _case("", what, **sizes)
            else:
                c = _case("", what, t=_log(rng, 1, 10000), **sizes, lengths=rng.random() < 0.4, state=rng.random() < 0.5,
                          stretch=rng.choice([64, 128, 256, 512]) if what == "delta grad" else 0)
        elif what.startswith("join"):
            groups = rng.choice([1, 1, 2, 8, 16, 33])
            group = _size(rng, 16, 8192 // groups, 16)
            c = _case("", what, rows=_log(rng, 1, 64000), width=group * groups, group=group, dtype=dtype, gate=rng.random() < 0.6,
                      residual=rng.choice(["", "fp32", "bf16"]), scale=rng.choice([1.0, 0.8]))
        else:
            smallest = _log(rng, 1, 1000)
            c = _case("", what, bits=rng.choice([8, 32]), count=rng.randint(1, 300), smallest=smallest, largest=smallest * _log(rng, 2, 4000),
                      grad=rng.choice(["fp32", "bf16"]), copy=rng.random() < 0.5, clip=rng.random() < 0.5)
        del c["name"]
        if _limits(c):
            return c


# ---- inputs -------------------------------------------------------------------------------------


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 1000003 + 31)

    def normal(self, *shape, s=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.g, device="cuda") * s).to(dtype)

    def uniform(self, *shape, lo=0.0, hi=1.0):
        return lo + (hi - lo) * torch.rand(shape, generator=self.g, device="cuda")

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _lengths(case):
    """None, one, and everything between up to t."""
    t, B = case["t"], case["B"]
    return [t] if B == 1 else [1 if b == 1 and t > 0 else (t * b) // (B - 1) for b in range(B)]


def _sizes(case):
    """Values of each tensor: spread over their logarithm, the largest last."""
    n, lo, hi = case["count"], case["smallest"], case["largest"]
    return [hi if i == n - 1 else int(lo * (hi / lo) ** (0.8 * i / max(n - 1, 1))) for i in range(n)]


def _places(case):
    """(offset, values) of each tensor in one buffer, each at a whole block."""
    at, got = 0, []
    for n in _sizes(case):
        got.append((at, n))
        at += -(-n // BLOCK) * BLOCK
    return got, at


def _inside_tensors(case):
    places, total = _places(case)
    ends = torch.zeros(total // BLOCK, dtype=torch.int64)
    for at, n in places:
        ends[at // BLOCK:at // BLOCK + -(-n // BLOCK)] = at + n
    return torch.arange(total, device="cuda") < ends.cuda().repeat_interleave(BLOCK)


def _inputs(case, seed):
    d, what = _Draw(seed), case["what"]
    if what == "adamw":
        there = _inside_tensors(case)
        total = there.numel()
        size = torch.exp(d.normal(total // BLOCK, s=1.5)).repeat_interleave(BLOCK) * 1e-3
        g = torch.where(there, d.normal(total) * size, 0.0)
        v = {"p": torch.where(there, d.normal(total, s=0.02), 0.0), "g": g.to(DTYPES[case["grad"]]),
             "m": torch.where(there, (0.5 * g + 0.5 * d.normal(total) * size), 0.0),
             "v": torch.where(there, size * size * d.uniform(total, lo=0.1, hi=2.0), 0.0)}
        if case["bits"] == 8:   # states as an earlier step left them: any codes but those of "nothing" for v
            v["m"] = torch.where(there, (d.uniform(total) * 256).to(torch.int64).clamp(max=255), 0).to(torch.uint8)
            v["v"] = torch.where(there, (d.uniform(total) * 80).to(torch.int64) + 176, 0).clamp(max=255).to(torch.uint8)
            v["m_scale"], v["v_scale"] = size[::BLOCK] * 0.5, (size * size)[::BLOCK].contiguous()
        return v
    dt = DTYPES[case["dtype"]]
    if what.startswith("join"):
        M, W = case["rows"], case["width"]
        v = {"x": d.normal(M, W, s=0.7, dtype=dt), "weight": 1.0 + d.normal(W, s=0.2), "z": d.normal(M, W, dtype=dt) if case["gate"] else None}
        if case["residual"]:
            rt = DTYPES[case["residual"]]
            v |= {"residual": d.normal(M, W, s=2.0, dtype=rt), "weight_next": 1.0 + d.normal(W, s=0.2)}
        if what == "join grad":
            v["dy"] = d.normal(M, W, s=0.1, dtype=dt)
            if case["residual"]:
                v["dresidual_out"] = d.normal(M, W, s=0.1, dtype=rt)
        return v
    t, B, Hk, H, dk, dv = case.get("t", 1), case["B"], case["Hk"], case["H"], case["dk"], case["dv"]
    unit = 1.0 if case["normalise"] else dk ** -0.5
    first = torch.exp(d.uniform(H, lo=math.log(1e-3), hi=math.log(0.1)))
    v = {"q": d.normal(t, B, Hk * dk, s=unit, dtype=dt), "k": d.normal(t, B, Hk * dk, s=unit, dtype=dt), "v": d.normal(t, B, H * dv, dtype=dt),
         "b": d.normal(t, B, H, dtype=dt), "a": d.normal(t, B, H, s=0.5, dtype=dt) if case["decay"] else None,
         "A": -torch.exp(d.uniform(H, lo=0.0, hi=math.log(16.0))) if case["decay"] else None,
         "a_bias": first + torch.log(-torch.expm1(-first)) if case["decay"] else None}
    if what == "delta token":
        v["state"] = d.normal(B + 3, H, dk, dv, s=0.3)
        v["index"] = d.order(B + 3)[:B].to(torch.int32)
        return v
    v["h0"] = d.normal(B, H, dk, dv, s=0.3) if case["state"] else None
    v["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["lengths"] else None
    if what == "delta grad":
        v["dy"] = d.normal(t, B, H * dv, s=0.1, dtype=dt)
        v["dh_out"] = d.normal(B, H, dk, dv, s=0.1) if case["state"] else None
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


def _own_delta(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]
    like = torch.empty_like

    def make():
        desc = mb.make_delta_desc(c.get("t", 1), c["B"], c["Hk"], c["H"], c["dk"], c["dv"], mb.BF16 if c["dtype"] == "bf16" else mb.FP32, 1,
                                  1 if c["normalise"] else 0, c.get("stretch", 0), c["dk"] ** -0.5, EPS_HEAD)
        k = {"desc": desc, "y": like(s["v"])}
        if c["what"] == "delta token":
            return {**k, "state": torch.zeros_like(s["state"])}
        grad = c["what"] == "delta grad"
        k |= {"h_out": torch.empty((c["B"], c["H"], c["dk"], c["dv"]), device="cuda"), "states": None,
              "ws": _bytes(mb.mebptt_delta_workspace_bytes(desc, grad))}
        if grad:
            k |= {"states": _bytes(mb.mebptt_delta_state_bytes(desc)), "dq": like(s["q"]), "dk": like(s["k"]), "dv": like(s["v"]), "db": like(s["b"]),
                  "da": like(s["a"]) if c["decay"] else None, "dA": like(s["A"]) if c["decay"] else None,
                  "da_bias": like(s["a_bias"]) if c["decay"] else None, "dh0": like(s["h0"]) if c["state"] else None}
        return k
    k = _kept(s, make)
    if c["what"] == "delta token":
        mb.mebptt_delta_step(k["desc"], s["q"][0], s["k"][0], s["v"][0], s["a"][0] if c["decay"] else None, s["b"][0], s["A"], s["a_bias"],
                             s["state"], s["index"], k["y"][0], k["state"])
        return {"y": k["y"], "state": k["state"]}
    given = (k["desc"], s["q"], s["k"], s["v"], s["a"], s["b"], s["A"], s["a_bias"], s["lengths"], s["h0"])
    mb.mebptt_delta_forward(*given, k["y"], k["h_out"], k["states"], k["ws"])
    if c["what"] == "delta":
        return {"y": k["y"], "h_out": k["h_out"]}
    mb.mebptt_delta_backward(*given, s["dy"], s["dh_out"], k["states"], k["dq"], k["dk"], k["dv"], k["da"], k["db"], k["dA"], k["da_bias"],
                             k["dh0"], k["ws"])
    names = ["y", "h_out", "dq", "dk", "dv", "db"]
    return {n: k[n] for n in names + (["da", "dA", "da_bias"] if c["decay"] else []) + (["dh0"] if c["state"] else [])}


def _own_join(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]
    like = torch.empty_like
    next_ = bool(c["residual"])

    def make():
        desc = mb.make_join_desc(c["rows"], c["width"], c["group"], mb.BF16 if c["dtype"] == "bf16" else mb.FP32,
                                 mb.FP32 if c["residual"] == "fp32" else mb.BF16, c["scale"], EPS, again=next_)
        k = {"desc": desc, "y": like(s["x"]), "sum": like(s["residual"]) if next_ else None}
        if c["what"] == "join grad":
            k |= {"rstd": torch.empty((c["rows"], c["width"] // c["group"]), device="cuda"), "rstd_next": torch.empty(c["rows"], device="cuda") if next_ else None,
                  "dx": like(s["x"]), "dz": like(s["z"]) if c["gate"] else None, "dweight": like(s["weight"]),
                  "dresidual": like(s["residual"]) if next_ else None, "dweight_next": like(s["weight_next"]) if next_ else None,
                  "ws": _bytes(mb.mebptt_join_workspace_bytes(desc))}
        return k
    k = _kept(s, make)
    residual, weight_next = (s["residual"], s["weight_next"]) if next_ else (None, None)
    back = c["what"] == "join grad"
    mb.mebptt_join_forward(k["desc"], s["x"], s["z"], s["weight"], residual, weight_next, k["y"], k["sum"], k["rstd"] if back else None,
                           k["rstd_next"] if back else None)
    names = ["y"] + (["sum"] if next_ else [])
    if back:
        mb.mebptt_join_backward(k["desc"], s["x"], s["z"], s["weight"], residual, weight_next, k["rstd"], k["rstd_next"], s["dy"],
                                s["dresidual_out"] if next_ else None, k["dx"], k["dz"], k["dweight"], k["dresidual"], k["dweight_next"], k["ws"])
        names += ["dx", "dweight"] + (["dz"] if c["gate"] else []) + (["dresidual", "dweight_next"] if next_ else [])
    return {n: k[n] for n in names}


def _own_adamw(s):
    from paper_1606_03401_amd import binding as mb
    c = s["case"]
    small = c["bits"] == 8

    def make():
        places, total = _places(c)
        cut = lambda name: [s[name][at:at + n] for at, n in places]  # noqa: E731
        scales = lambda name: [s[name][at // BLOCK:at // BLOCK + -(-n // BLOCK)] for at, n in places]  # noqa: E731
        k = {"copy": torch.zeros(total, dtype=torch.bfloat16, device="cuda") if c["copy"] else None, "norm": torch.zeros(2, device="cuda")}
        tensors = mb.make_adamw_tensors(cut("p"), cut("g"), cut("m"), cut("v"), scales("m_scale") if small else None, scales("v_scale") if small else None,
                                        [k["copy"][at:at + n] for at, n in places] if c["copy"] else None)
        table = _bytes(mb.mebptt_adamw_table_bytes(tensors))
        mb.mebptt_adamw_prepare(tensors, table)
        k |= {"table": table, "tensors": tensors, "ws": _bytes(mb.mebptt_adamw_workspace_bytes(tensors)),
              "desc": mb.make_adamw_desc(ADAM["rate"], ADAM["beta1"], ADAM["beta2"], ADAM["eps"], ADAM["decay"], ADAM["step"], ADAM["seed"])}
        if small:
            k |= {"m": torch.empty(total, dtype=torch.bfloat16, device="cuda"), "v": torch.empty(total, dtype=torch.bfloat16, device="cuda")}
        return k
    k = _kept(s, make)
    if c["clip"]:
        mb.mebptt_adamw_norm(k["tensors"], k["table"], 1.0, k["norm"], k["ws"])
    mb.mebptt_adamw_step(k["desc"], k["tensors"], k["table"], k["norm"][1:] if c["clip"] else None)
    out = {"p": s["p"], "m": s["m"], "v": s["v"]}
    if small:
        mb.mebptt_adamw_unpack(s["m"], s["m_scale"], True, k["m"])
        mb.mebptt_adamw_unpack(s["v"], s["v_scale"], False, k["v"])
        out |= {"m": k["m"], "v": k["v"]}
    return out | ({"copy": k["copy"]} if c["copy"] else {}) | ({"norm": k["norm"]} if c["clip"] else {})


# ---- the plain forms ----------------------------------------------------------------------------


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-x.abs()))


def _heads(m, c, t, d):
    """[t, B, heads d] -> [chunks, B, heads, CHUNK, d] in 32 bits, zeros behind the last step."""
    n = -(-t // CHUNK)
    m = torch.nn.functional.pad(m.float(), (0, 0, 0, 0, 0, n * CHUNK - t))
    return m.view(n, CHUNK, c["B"], -1, d).permute(0, 2, 3, 1, 4)


def _flat(m, t):
    """The other way."""
    n, B, H, C, d = m.shape
    return m.permute(0, 3, 1, 2, 4).reshape(n * C, B, H * d)[:t]


def _inverse(N):
    """(I + N)^-1 of strictly lower triangular [.., CHUNK, CHUNK]: the inverses of two diagonal blocks give that of the block around them."""
    T = torch.eye(CHUNK, device=N.device).expand(N.shape).contiguous()
    size = 1
    while size < CHUNK:
        pairs = CHUNK // (2 * size)
        at = torch.arange(pairs, device=N.device)
        blocks = lambda m: m.view(*m.shape[:-2], pairs, 2, size, pairs, 2, size)[..., at, :, :, at, :, :]  # noqa: E731
        t, low = blocks(T), blocks(N)[..., 1, :, 0, :]
        new = -torch.matmul(torch.matmul(t[..., 1, :, 1, :], low), t[..., 0, :, 0, :])
        view = T.view(*T.shape[:-2], pairs, 2, size, pairs, 2, size)
        view[..., at, 1, :, at, 0, :] = new
        size *= 2
    return T


def _prefix(A, B):
    """S_c = A_c S_{c-1} + B_c over the first axis from zero, by doubling."""
    k = 1
    while k < B.shape[0]:
        B = torch.cat([B[:k], torch.matmul(A[k:], B[:-k]) + B[k:]])
        if 2 * k < B.shape[0]:
            A = torch.cat([A[:k], torch.matmul(A[k:], A[:-k])])
        k *= 2
    return B


def _unit(m, c):
    """Heads at length one, and the factors that made them so."""
    r = torch.rsqrt((m * m).sum(-1, keepdim=True) + EPS_HEAD) if c["normalise"] else torch.ones_like(m[..., :1])
    return m * r, r


def _gates(s):
    """(raw, log decay, beta)"""
    raw = s["a"].float() + s["a_bias"] if s["case"]["decay"] else torch.zeros_like(s["b"], dtype=torch.float32)
    return raw, s["A"] * _softplus(raw) if s["case"]["decay"] else raw, _sigmoid(s["b"].float())


def _delta_token(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    B, Hk, H = c["B"], c["Hk"], c["H"]
    wide = lambda m: m.repeat_interleave(H // Hk, 1)  # noqa: E731
    q, k = (wide(_unit(s[n][0].float().view(B, Hk, -1), c)[0]) for n in ("q", "k"))
    v = s["v"][0].float().view(B, H, -1)
    _, g, beta = _gates(s)
    i = s["index"].long()
    h = torch.exp(g[0])[..., None, None] * s["state"][i]
    r = v - (h * k[..., None]).sum(2)
    h = h + (beta[0][..., None] * k)[..., None] * r[:, :, None]
    y = (h * q[..., None]).sum(2) * c["dk"] ** -0.5
    state = torch.zeros_like(s["state"])
    state[i] = h
    return {"y": y.to(dt).view(1, B, -1), "state": state}


def _delta(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    if c["what"] == "delta token":
        return _delta_token(s)
    t, B, Hk, H = s["v"].shape[0], c["B"], c["Hk"], c["H"]
    n, mm, tr = -(-t // CHUNK), torch.matmul, lambda m: m.transpose(-1, -2)
    wide = lambda m: m.repeat_interleave(H // Hk, 2)  # noqa: E731
    raw, g, beta = _gates(s)
    v = s["v"]
    inside = None if s["lengths"] is None else (torch.arange(t, device="cuda")[:, None] < s["lengths"])[:, :, None]
    only = (lambda m: m) if inside is None else (lambda m: torch.where(inside, m, torch.zeros((), dtype=m.dtype, device="cuda")))
    (qn, q_r), (kn, k_r) = (_unit(_heads(only(s[m]), c, t, c["dk"]), c) for m in ("q", "k"))
    q, k = wide(qn) * c["dk"] ** -0.5, wide(kn)
    v = _heads(only(v), c, t, c["dv"])
    be, gs = _heads(only(beta), c, t, 1), _heads(only(g), c, t, 1)
    G = gs.double().cumsum(3)
    D = torch.exp((G - tr(G)).float().masked_fill(torch.ones((CHUNK, CHUNK), dtype=torch.bool, device="cuda").triu(1), -math.inf))
    ga, last = torch.exp(G.float()), torch.exp((G[..., -1:, :] - G).float())
    lower = torch.ones((CHUNK, CHUNK), device="cuda").tril(-1)
    M, P = mm(k, tr(k)) * D * lower, mm(q, tr(k)) * D
    T = _inverse(M * tr(be))
    kd, kg, qg = last * k, ga * k, ga * q
    end = ga[..., -1:, :]
    across = tr(mm(tr(mm(T, kg)), be * kd))                          # Kd^T beta T (gamma K)
    move = end * torch.eye(c["dk"], device="cuda") - across
    add = mm(tr(kd), be * mm(T, v))
    if c["state"] and n:
        add[0] += mm(move[0], s["h0"])
    S = _prefix(move, add)
    first = s["h0"] if c["state"] else torch.zeros((B, H, c["dk"], c["dv"]), device="cuda")
    S0 = torch.cat([first[None], S[:-1]])
    R = mm(T, v - mm(kg, S0))
    U = be * R
    y = only(_flat(mm(qg, S0) + mm(P, U), t))
    out = {"y": y.to(dt), "h_out": (S[-1] if n else first).clone()}
    if c["what"] == "delta":
        return out
    dy = _heads(only(s["dy"]), c, t, c["dv"])
    into, adj = mm(tr(P), dy), mm(tr(T), be * torch.eye(CHUNK, device="cuda"))
    add = mm(tr(qg), dy) - mm(tr(kg), mm(adj, into))
    if s["dh_out"] is not None:
        add[-1] += mm(tr(move[-1]), s["dh_out"])
    back = _prefix(tr(move).flip(0), add.flip(0)).flip(0)            # dS at the start of every chunk
    dS1 = torch.cat([back[1:], (s["dh_out"] if s["dh_out"] is not None else torch.zeros_like(first))[None]])
    dU = into + mm(kd, dS1)
    Z = mm(adj, dU)
    dP, E = mm(dy, tr(U)), mm(Z, tr(R)) * lower
    dM = -E * tr(be)
    F = dP * P + dM * M
    US, YS, ZS = mm(U, tr(dS1)) * last, mm(dy, tr(S0)) * ga, mm(Z, tr(S0)) * ga
    dPD, dMD = dP * D, dM * D
    dq = (mm(dPD, k) + YS) * c["dk"] ** -0.5
    dk = mm(tr(dPD), q) + mm(dMD, k) + mm(tr(dMD), k) + US - ZS
    ends = (US * k).sum(-1, keepdim=True)
    dG = F.sum(-1, keepdim=True) - F.sum(-2)[..., None] + (YS * q).sum(-1, keepdim=True) - (ZS * k).sum(-1, keepdim=True) - ends
    dG[..., -1:, :] += ends.sum(-2, keepdim=True) + end * (dS1 * S0).sum((-1, -2))[..., None, None]
    dg = _flat(dG.flip(3).cumsum(3).flip(3), t)
    dbeta = (dU * R).sum(-1, keepdim=True) - (M * E).sum(-2)[..., None]

    def heads_back(d, unit, r):
        """The gradient of a shared head, through its norm."""
        d = d.unflatten(2, (Hk, H // Hk)).sum(3)
        return only(_flat(r * (d - unit * (d * unit).sum(-1, keepdim=True)) if c["normalise"] else d, t)).to(dt)
    out |= {"dq": heads_back(dq, qn, q_r), "dk": heads_back(dk, kn, k_r), "dv": only(_flat(Z, t)).to(dt)}
    out["db"] = only(_flat(dbeta, t) * beta * (1.0 - beta)).to(dt)
    if c["decay"]:
        da = only(dg * s["A"] * _sigmoid(raw))
        out |= {"da": da.to(dt), "dA": only(dg * _softplus(raw)).sum((0, 1)), "da_bias": da.sum((0, 1))}
    if c["state"]:
        out["dh0"] = back[0].clone() if n else s["dh_out"].clone()
    return out


def _join(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    groups = lambda m: m.unflatten(1, (-1, c["group"]))  # noqa: E731
    x, w = s["x"].float(), s["weight"]
    rstd = torch.rsqrt((groups(x) ** 2).mean(2, keepdim=True) + EPS)
    n = (groups(x) * rstd).flatten(1)
    z = s["z"].float() if c["gate"] else None
    sg = _sigmoid(z) if c["gate"] else None
    a = n * w * (z * sg) if c["gate"] else n * w
    out = {}
    if c["residual"]:
        rt = DTYPES[c["residual"]]
        r = c["scale"] * s["residual"].float() + a
        out["sum"] = r.to(rt)
        y = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * s["weight_next"]
    else:
        y = a
    out["y"] = y.to(dt)
    if c["what"] == "join":
        return out
    da = s["dy"].float()
    if c["residual"]:
        rn = torch.rsqrt((r * r).mean(1, keepdim=True) + EPS)
        m = r * rn
        g = da * s["weight_next"]
        out["dweight_next"] = (da * m).sum(0)
        da = rn * (g - m * (g * m).mean(1, keepdim=True)) + s["dresidual_out"].float()
        out["dresidual"] = (c["scale"] * da).to(rt)
    act = z * sg if c["gate"] else 1.0
    if c["gate"]:
        out["dz"] = (da * n * w * sg * (1.0 + z * (1.0 - sg))).to(dt)
    out["dweight"] = (da * n * act).sum(0)
    g = da * w * act
    out["dx"] = (groups(g) - groups(n) * (groups(g) * groups(n)).mean(2, keepdim=True)).mul(rstd).flatten(1).to(dt)
    return out


def _mix(x):
    """32 bits out of 32, each of which depends on all: multiplications by odd numbers and shifts."""
    mask = 0xFFFFFFFF
    x = ((x ^ (x >> 17)) * 0x2C9277B5) & mask
    x = ((x ^ (x >> 14)) * 0x5851F42D) & mask
    return x ^ (x >> 16)


def _random(case, total):
    """What a value is rounded with: a hash of the seed, the step, its block's number over all tensors and its place there."""
    block, place = torch.arange(total // BLOCK, device="cuda"), torch.arange(BLOCK, device="cuda")
    key = _mix((ADAM["seed"] + ADAM["step"] * 0x632BE5AB + block * 0x9E3779B9) & 0xFFFFFFFF)
    return _mix((key[:, None] + place * 0x85157AF5) & 0xFFFFFFFF).flatten()


def _value8(code, scale, signed):
    """What a code stands for: 2^(e - bias) (1 + f / 8) times its block's scale, the lowest one for zero."""
    code = code.to(torch.int64)
    low = code & 127 if signed else code
    size = torch.exp2((low >> 3).to(scale.dtype) - (15 if signed else 31)) * (1.0 + (low & 7).to(scale.dtype) / 8)
    size = torch.where(low == 0, 0.0, size) * scale.repeat_interleave(BLOCK)
    return torch.where(code >= 128, -size, size) if signed else size


def _code8(x, bits16, signed):
    """(codes, scales): the two neighbours of x / scale, one of them by chance."""
    scale = x.abs().view(-1, BLOCK).amax(1) / 1.875
    u = x.abs() / torch.where(scale > 0, scale, 1.0).repeat_interleave(BLOCK)
    code = ((u.view(torch.int32).to(torch.int64) + (bits16 << 4)) >> 20) - ((112 if signed else 96) << 3)
    if signed:
        least = 1.125 * 2.0 ** -15
        code = torch.where(u < least, (u * (65536.0 / least) > bits16).to(torch.int64), code.clamp(1, 127))
        return torch.where((x < 0) & (code > 0), code + 128, code), scale
    return torch.where(u > 0, code.clamp(1, 255), 0), scale


def _adamw(s):
    c, small = s["case"], s["case"]["bits"] == 8
    g = s["g"].float()
    out = {}
    if c["clip"]:
        norm = torch.sqrt((g * g).sum())
        factor = torch.clamp(1.0 / norm, max=1.0)
        g = g * factor
        out["norm"] = torch.stack([norm, factor])
    m, v = (_value8(s["m"], s["m_scale"], True), _value8(s["v"], s["v_scale"], False)) if small else (s["m"], s["v"])
    m = ADAM["beta1"] * m + (1.0 - ADAM["beta1"]) * g
    v = ADAM["beta2"] * v + (1.0 - ADAM["beta2"]) * (g * g)
    c1, c2 = (1.0 - ADAM[b] ** ADAM["step"] for b in ("beta1", "beta2"))
    s["p"].mul_(1.0 - ADAM["rate"] * ADAM["decay"]).sub_(ADAM["rate"] * (m / c1) / (torch.sqrt(v / c2) + ADAM["eps"]))
    if small:
        h = _random(c, g.numel())
        for name, x, bits in (("m", m, h >> 16), ("v", v, h & 0xFFFF)):
            code, scale = _code8(x, bits, name == "m")
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
            out[name] = _value8(code, scale, name == "m").to(torch.bfloat16)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out |= {"m": s["m"], "v": s["v"]}
    return {**out, "p": s["p"]} | ({"copy": s["p"].to(torch.bfloat16)} if c["copy"] else {})


def run(state):
    kind = state["case"]["what"].split()[0]
    if own:
        return {"delta": _own_delta, "join": _own_join, "adamw": _own_adamw}[kind](state)
    return {"delta": _delta, "join": _join, "adamw": _adamw}[kind](state)


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    what = case["what"]
    if what == "adamw":
        n = float(sum(_sizes(case)))
        g = 4.0 if case["grad"] == "fp32" else 2.0
        states = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK + 4.0    # (8 bits: and their values in bf16)
        return {"bytes": n * (8.0 + g + states + (2.0 if case["copy"] else 0.0)), "flops": n * 14.0}
    e = 4.0 if case["dtype"] == "fp32" else 2.0
    if what.startswith("join"):
        n, back = float(case["rows"]) * case["width"], what == "join grad"
        r = {"": 0.0, "fp32": 4.0, "bf16": 2.0}[case["residual"]]
        gate = e if case["gate"] else 0.0
        # x, z, residual in, y and the sum out; back: dy and the sum's gradient in, dx, dz and the residual's gradient out
        return {"bytes": n * ((2 * e + gate + 2 * r) + (2 * e + gate + 2 * r if back else 0.0)) + 8.0 * case["width"], "flops": n * (40.0 if back else 15.0)}
    t, B, Hk, H, dk, dv = case.get("t", 1), case["B"], case["Hk"], case["H"], case["dk"], case["dv"]
    n, state = float(t) * B, 4.0 * B * H * dk * dv
    rows = e * n * (2 * Hk * dk + H * dv + H * (2 if case["decay"] else 1))
    y = e * n * H * dv
    if what == "delta token":
        return {"bytes": rows + y + 2 * state, "flops": 7.0 * n * H * dk * dv}
    given = 1 if case["state"] else 0
    if what == "delta":
        return {"bytes": rows + y + (1 + given) * state, "flops": 7.0 * n * H * dk * dv}
    return {"bytes": 2 * rows + 2 * y + (1 + 3 * given) * state, "flops": 22.0 * n * H * dk * dv}


# ---- the same in 64 bits ------------------------------------------------------------------------


def _exact_join(case, v):
    M, W, d = case["rows"], case["width"], case["group"]
    x = v["x"].double().view(M, W // d, d)
    size = torch.sqrt((x * x).sum(2, keepdim=True) / d + EPS)
    unit = (x / size).reshape(M, W)
    z = v["z"].double() if case["gate"] else None
    act = z * torch.sigmoid(z) if case["gate"] else torch.ones_like(unit)
    w = v["weight"].double()
    branch = unit * w * act
    got = {"y": branch}
    if case["residual"]:
        total = case["scale"] * v["residual"].double() + branch
        size_next = torch.sqrt((total * total).sum(1, keepdim=True) / W + EPS)
        unit_next = total / size_next
        got |= {"sum": total, "y": unit_next * v["weight_next"].double()}
    if case["what"] == "join":
        return got
    into = v["dy"].double()
    if case["residual"]:
        got["dweight_next"] = (into * unit_next).sum(0)
        into = into * v["weight_next"].double()
        into = (into - unit_next * (into * unit_next).sum(1, keepdim=True) / W) / size_next + v["dresidual_out"].double()
        got["dresidual"] = into * case["scale"]
    got["dweight"] = (into * unit * act).sum(0)
    if case["gate"]:
        sg = torch.sigmoid(z)
        got["dz"] = into * unit * w * (sg + z * sg * (1 - sg))
    into = (into * w * act).view(M, W // d, d)
    unit = unit.view(M, W // d, d)
    got["dx"] = ((into - unit * (into * unit).sum(2, keepdim=True) / d) / size).reshape(M, W)
    return got


def _exact_adamw(case, v):
    places, total = _places(case)
    got = {k: torch.zeros(total, dtype=torch.float64, device="cuda") for k in ("p", "m", "v")}
    factor = 1.0
    if case["clip"]:
        norm = torch.sqrt(v["g"].double().square().sum())
        factor = torch.clamp(1.0 / norm, max=1.0)
        got["norm"] = torch.stack([norm, factor])
    b1, b2 = ADAM["beta1"], ADAM["beta2"]
    h = _random(case, total) if case["bits"] == 8 else None
    for at, n in places:   # a tensor at a time
        g = v["g"][at:at + n].double() * factor
        if case["bits"] == 8:
            end = at + -(-n // BLOCK) * BLOCK
            m, u = (_value8(v[k][at:end], v[k + "_scale"][at // BLOCK:end // BLOCK].double(), k == "m")[:n] for k in ("m", "v"))
        else:
            m, u = v["m"][at:at + n].double(), v["v"][at:at + n].double()
        m, u = m * b1 + g * (1 - b1), u * b2 + g.square() * (1 - b2)
        p = v["p"][at:at + n].double() * (1 - ADAM["rate"] * ADAM["decay"])
        got["p"][at:at + n] = p - ADAM["rate"] * m / (1 - b1 ** ADAM["step"]) / (torch.sqrt(u / (1 - b2 ** ADAM["step"])) + ADAM["eps"])
        if case["bits"] == 8:
            m, u = (torch.nn.functional.pad(k, (0, end - at - n)) for k in (m, u))
            got["m"][at:end] = _rounded8(m, h[at:end] >> 16, True)
            got["v"][at:end] = _rounded8(u, h[at:end] & 0xFFFF, False)
        else:
            got["m"][at:at + n], got["v"][at:at + n] = m, u
    if case["copy"]:
        got["copy"] = got["p"]
    return got


def _rounded8(x, bits16, signed):
    """x rounded to a block's scale, an exponent and three bits, up where the part cut off is above what `bits16` says."""
    scale = (x.abs().view(-1, BLOCK).amax(1) / 1.875).repeat_interleave(BLOCK)
    u = x.abs() / torch.where(scale > 0, scale, 1.0)
    lowest = 2.0 ** (-15 if signed else -31)
    e = torch.floor(torch.log2(u.clamp(min=lowest)))
    step = torch.exp2(e - 3)
    units = u / step
    r = (torch.floor(units) + ((units - torch.floor(units)) + bits16.double() / 65536 >= 1)) * step
    r = torch.minimum(r, torch.full_like(r, 1.875))
    least = 1.125 * lowest
    small = torch.where(u * (65536 / least) > bits16, least, 0.0) if signed else torch.where(u > 0, least, 0.0)
    return torch.where(u < least, small, r) * scale * torch.sign(x)


def _exact_delta(case, v):
    B, Hk, H, dk, dv = case["B"], case["Hk"], case["H"], case["dk"], case["dv"]
    t = v["v"].shape[0]
    back, scale = case["what"] == "delta grad", dk ** -0.5
    if back and float(t) * B * H * dk * dv > 5.0e9:
        return None
    of = torch.arange(H, device="cuda") // (H // Hk)

    def unit(m):
        m = m.double().view(B, Hk, dk)
        return m / torch.sqrt((m * m).sum(2, keepdim=True) + EPS_HEAD) if case["normalise"] else m

    def at(i):
        raw = v["a"][i].double() + v["a_bias"].double() if case["decay"] else None
        decay = torch.exp(v["A"].double() * torch.logaddexp(raw, torch.zeros_like(raw))) if case["decay"] else torch.ones((B, H), dtype=torch.float64, device="cuda")
        return raw, decay[:, :, None, None], torch.sigmoid(v["b"][i].double())[:, :, None], unit(v["q"][i])[:, of] * scale, unit(v["k"][i])[:, of], v["v"][i].double().view(B, H, dv)

    def dot(S, x):
        return torch.matmul(x[:, :, None, :], S)[:, :, 0]

    def forward(i, S):
        _, decay, beta, q, k, val = at(i)
        S = S * decay
        r = val - dot(S, k)
        S = S + k[..., None] * (beta * r)[:, :, None]
        return S, r, dot(S, q)

    if case["what"] == "delta token":
        i = v["index"].long()
        S, _, y = forward(0, v["state"].double()[i])
        state = torch.zeros_like(v["state"], dtype=torch.float64)
        state[i] = S
        return {"y": y.view(1, B, H * dv), "state": state}
    ends = v["lengths"] if case["lengths"] else torch.full((B,), t, device="cuda")
    S = v["h0"].double() if case["state"] else torch.zeros((B, H, dk, dv), dtype=torch.float64, device="cuda")
    y, kept = torch.zeros((t, B, H * dv), dtype=torch.float64, device="cuda"), []
    for i in range(t):
        live = ends > i
        new, r, out = forward(i, S)
        if back:
            kept.append((S, r))
        S = torch.where(live[:, None, None, None], new, S) if case["lengths"] else new
        y[i] = torch.where(live[:, None], out.view(B, H * dv), 0.0)
    got = {"y": y, "h_out": S}
    if not back:
        return got
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    got |= {"dq": new(t, B, Hk * dk), "dk": new(t, B, Hk * dk), "dv": new(t, B, H * dv), "db": new(t, B, H)}
    if case["decay"]:
        got |= {"da": new(t, B, H), "dA": new(H), "da_bias": new(H)}
    g = v["dh_out"].double() if case["state"] else new(B, H, dk, dv)
    for i in reversed(range(t)):
        live = (ends > i)[:, None]
        raw, decay, beta, q, k, val = at(i)
        before, r = kept.pop()
        moved = before * decay
        dy = torch.where(live, v["dy"][i].double(), 0.0).view(B, H, dv)
        after = moved + k[..., None] * (beta * r)[:, :, None]
        dq = torch.matmul(after, dy[..., None])[..., 0] * scale
        h = g + q[..., None] * dy[:, :, None]
        into = dot(h, k)                                   # gradient of beta r
        dr = beta * into
        dk_ = torch.matmul(h, (beta * r)[..., None])[..., 0] - torch.matmul(moved, dr[..., None])[..., 0]
        dmoved = h - k[..., None] * dr[:, :, None]
        db = (into * r).sum(2) * (beta * (1 - beta))[..., 0]
        dlog = (dmoved * moved).sum((2, 3))
        mask = lambda m: torch.where(live, m.reshape(B, -1), 0.0)  # noqa: E731
        for name, d in (("q", dq), ("k", dk_)):
            d = d.view(B, Hk, H // Hk, dk).sum(2)
            m = v[name][i].double().view(B, Hk, dk)
            if case["normalise"]:
                length = torch.sqrt((m * m).sum(2, keepdim=True) + EPS_HEAD)
                d = d / length - m * (d * m).sum(2, keepdim=True) / length ** 3
            got["d" + name][i] = mask(d)
        got["dv"][i], got["db"][i] = mask(dr), mask(db)
        if case["decay"]:
            da = mask(dlog * v["A"].double() * torch.sigmoid(raw))
            got["da"][i] = da
            got["dA"] += mask(dlog * torch.logaddexp(raw, torch.zeros_like(raw))).sum(0)
            got["da_bias"] += da.sum(0)
        g = torch.where(live[:, :, None, None], dmoved * decay, g)
    if case["state"]:
        got["dh0"] = g
    return got


def exact(case, seed):
    v = _inputs(case, seed)
    kind = case["what"].split()[0]
    return {"delta": _exact_delta, "join": _exact_join, "adamw": _exact_adamw}[kind](case, v)
