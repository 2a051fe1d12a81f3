"""The paths that the block's operators take at the sizes they are for: large tiles and copies of the product, whole stretches and many
chunks of the scan, long stretches of the convolution, more rows than workgroups of the norm.  Each against 64 bits; that the cases take these
paths is seen from the launches of a traced run."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _room(n):
    return torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV)


# ---- product -----------------------------------------------------------------------------------------


def _bytes(g, rows, K, ld, first=0):
    """[rows, K] of whole numbers in rows of `ld` bytes, the first one `first` bytes behind a boundary; 127 in what lies between them."""
    whole = torch.full((rows * ld + first + 64,), 127, dtype=torch.int8, device=DEV)
    v = whole[first:first + rows * ld].view(rows, ld)[:, :K]
    v.copy_(torch.randint(-127, 128, (rows, K), generator=g, device=DEV, dtype=torch.int8))
    return v


def _product(g, a, b, dtype, bias, room):
    """Largest error over its bound: four roundings of 2^-24 in 32 bits, of the value and of the bias; 2^-9 of the result more in bf16."""
    (M, K), N = a.shape, b.shape[0]
    sa, sb = torch.rand(M, generator=g, device=DEV) + 0.1, torch.rand(N, generator=g, device=DEV) + 0.1
    vb = torch.randn(N, generator=g, device=DEV) if bias else None
    whole = torch.full((M + 2, N + 3), 7.0, dtype=torch.float32 if dtype == mb.FP32 else torch.bfloat16, device=DEV)
    out = whole[1:-1, :N]
    mb.mebptt_int8_product(mb.make_int8_desc(M, N, K, dtype), a, sa, b, sb, vb, out, room)
    v = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    want = v + vb.double() if bias else v
    bound = 2.0 ** -22 * (v.abs() + (vb.double().abs() if bias else 0.0)) + (0.0 if dtype == mb.FP32 else 2.0 ** -8 * want.abs()) + 1e-30
    assert bool((whole[0] == 7).all() and (whole[-1] == 7).all() and (whole[:, N:] == 7).all())
    return float(((out.double() - want).abs() / bound).max())


def test_product_asks_for_room_only_for_what_it_copies():
    """K = 1022: rows 1024 bytes apart are read as they are."""
    M, N, K = 512, 4096, 1022
    g = _gen(1)
    need = mb.mebptt_int8_workspace_bytes(mb.make_int8_desc(M, N, K, mb.FP32))
    assert need == (M + N) * 1024
    ready_a, ready_b, a, b = _bytes(g, M, K, 1024), _bytes(g, N, K, 1024), _bytes(g, M, K, K), _bytes(g, N, K, K)
    for x, y, room in ((ready_a, ready_b, 0), (ready_a, b, N * 1024), (a, ready_b, M * 1024), (a, b, need)):
        assert _product(g, x, y, mb.FP32, True, _room(room) if room else None) <= 1
        if room:
            with pytest.raises(mb.MebpttError):
                _product(g, x, y, mb.FP32, True, _room(room - 256))


# M, N, K: tiles of 128 with stages in fours, a loose one and a short one, with a short one alone, with loose ones alone; tiles of 256 with all of them, with
# fours alone; copies of rows that begin anywhere for both.  The tile's size
TILES = [(1000, 1021, 592, 128), (2048, 2100, 48, 128), (4000, 4100, 128, 128), (4080, 4090, 1232, 256), (4080, 4090, 1024, 256), (2000, 2050, 1022, 128),
         (4080, 4090, 1233, 256)]


@pytest.mark.parametrize("M,N,K", [c[:3] for c in TILES])
@pytest.mark.parametrize("dtype", [mb.FP32, mb.BF16])
def test_product_by_tiles(M, N, K, dtype):
    g = _gen(M + K)
    room = mb.mebptt_int8_workspace_bytes(mb.make_int8_desc(M, N, K, dtype))
    assert (room > 0) == (K % 16 != 0)
    room = _room(room) if room else None
    ld = -(-K // 16) * 16
    assert _product(g, _bytes(g, M, K, K), _bytes(g, N, K, K), dtype, dtype == mb.FP32, room) <= 1
    assert _product(g, _bytes(g, M, K, ld + 32), _bytes(g, N, K, ld + 16), dtype, False, room) <= 1
    assert _product(g, _bytes(g, M, K, ld + 5, 3), _bytes(g, N, K, K, 1), dtype, True, room) <= 1


# ---- norm --------------------------------------------------------------------------------------------


def _near(got, want, what):
    """32 bits: sums of a few thousand terms in trees or short runs and exponents of up to 16, 2^-17 of the tensor's norm and 2^-14 of its largest value;
    bf16: 2^-8 of the value more, twice its rounding."""
    wide = got.dtype == torch.float32
    err, w = (got.double() - want).abs(), want.abs()
    assert bool(torch.isfinite(got).all()), what
    assert float(err.norm()) <= (2.0 ** -17 if wide else 2.0 ** -8) * float(want.norm()) + 1e-30, (what, float(err.norm() / want.norm()))
    assert bool((err <= 2.0 ** -14 * w.max() + (0.0 if wide else 2.0 ** -8) * w + 1e-30).all()), (what, float((err / w.max()).max()))


@pytest.mark.parametrize("rows,width", [(1100, 2056), (2500, 2049), (1100, 8200), (2100, 9001), (5000, 1024), (9001, 63)])
@pytest.mark.parametrize("dtype", [mb.FP32, mb.BF16])
def test_norm_gradient_of_more_rows_than_workgroups(rows, width, dtype):
    g = _gen(rows)
    T = torch.float32 if dtype == mb.FP32 else torch.bfloat16
    r, do = torch.randn((rows, width), generator=g, device=DEV), torch.randn((rows, width), generator=g, device=DEV)
    w, dy = 1 + 0.2 * torch.randn(width, generator=g, device=DEV), torch.randn((rows, width), generator=g, device=DEV).to(T)
    rstd = torch.rsqrt(r.double().square().mean(1) + 1e-5).float()
    d = mb.make_norm_desc(rows, width, dtype, mb.FP32, dtype, 1e-5)
    assert mb.mebptt_norm_workspace_bytes(d) == -(-1024 * width * 4 // 256) * 256      # a partial dweight for each of 1024 workgroups
    dx, dr, dw = torch.empty_like(dy), torch.empty_like(r), torch.empty_like(w)
    mb.mebptt_norm_backward(d, r, w, rstd, dy, do, dx, dr, dw, _room(mb.mebptt_norm_workspace_bytes(d)))
    n, gy = r.double() * rstd.double()[:, None], dy.double() * w.double()
    want = rstd.double()[:, None] * (gy - n * (gy * n).mean(1, keepdim=True)) + do.double()
    _near(dx, want, "dx")
    _near(dr, want, "dresidual")
    _near(dw, (dy.double() * n).sum(0), "dweight")


# ---- convolution -------------------------------------------------------------------------------------


def _silu(v):
    return v * torch.sigmoid(v)


def _conv64(x, w, bias, n, state, dy, dlast):
    """y, the last taps - 1 inputs, and the gradients of both by automatic differentiation, in 64 bits."""
    t, B, C = x.shape
    W = w.shape[1]
    x, w, bias, state = (v.double().requires_grad_() for v in (x, w, bias, state))
    live = (torch.arange(t, device=DEV)[:, None] < n)[..., None]
    rows = torch.cat([state.transpose(0, 1), torch.where(live, x, 0.0)])
    y = torch.where(live, _silu(sum(rows[j:j + t] * w[:, j] for j in range(W)) + bias), 0.0)
    at = n[:, None] + torch.arange(W - 1, device=DEV)
    last = rows.transpose(0, 1).gather(1, at[..., None].expand(B, W - 1, C))
    grads = torch.autograd.grad((y * dy.double()).sum() + (last * dlast.double()).sum(), (x, w, bias, state))
    return y.detach(), last.detach(), grads


# t, B, C, taps; steps per thread forward, and backward; backward, stretches per wave at most
CONVS = [(520, 48, 2048, 4, 32, 48, 2), (500, 48, 2048, 8, 32, 48, 2), (150, 40, 2047, 3, 32, 48, 2), (480, 24, 2048, 4, 16, 48, 1), (480, 12, 2048, 4, 8, 24, 1),
         (480, 6, 2048, 2, 8, 12, 1)]


@pytest.mark.parametrize("t,B,C,taps", [c[:4] for c in CONVS])
@pytest.mark.parametrize("dtype", [mb.FP32, mb.BF16])
@pytest.mark.parametrize("ragged", [False, True])
def test_conv_in_long_stretches(t, B, C, taps, dtype, ragged):
    g = _gen(t + taps)
    T = torch.float32 if dtype == mb.FP32 else torch.bfloat16
    new = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, dy, state, dlast = new(t, B, C).to(T), new(t, B, C).to(T), new(B, taps - 1, C).to(T), new(B, taps - 1, C).to(T)
    w, bias = new(C, taps) * 0.5, new(C) * 0.1
    n = torch.tensor([(t * (B - 1 - b)) // (B - 1) if b != 1 else 1 for b in range(B)], device=DEV) if ragged else torch.full((B,), t, device=DEV)
    y64, last64, grads = _conv64(x, w, bias, n, state, dy, dlast)
    if ragged:
        beyond = torch.arange(t, device=DEV)[:, None] >= n
        x[beyond], dy[beyond] = float("nan"), float("nan")
    lengths = n.int() if ragged else None
    d = mb.make_conv_desc(t, B, C, taps, dtype, 1)
    y, last, dx, ds = torch.empty_like(x), torch.empty_like(state), torch.empty_like(x), torch.empty_like(state)
    dw, db = torch.empty_like(w), torch.empty_like(bias)
    mb.mebptt_conv_forward(d, x, w, bias, lengths, state, y, last)
    _near(y, y64, "y")
    assert torch.equal(last.double(), last64)
    mb.mebptt_conv_backward(d, x, w, bias, lengths, state, dy, dlast, dx, dw, db, ds, _room(mb.mebptt_conv_workspace_bytes(d)))
    for got, want, what in zip((dx, dw, db, ds), grads, ("dx", "dweight", "dbias", "dstate_in")):
        _near(got, want, what)
    if ragged:
        assert bool((y[beyond] == 0).all() and (dx[beyond] == 0).all())


# ---- scan --------------------------------------------------------------------------------------------


def _scan64(u, delta, A, Bm, Cm, G, skip, z, bias, n, h0, dy, dh):
    """Outputs and gradients by the formulas in 64 bits, step by step, all sequences at once."""
    u, delta, A, Bm, Cm, skip, z, bias, h, dy, g = (None if v is None else v.double() for v in (u, delta, A, Bm, Cm, skip, z, bias, h0, dy, dh))
    t, B, D = u.shape
    N = A.shape[1]
    wide = lambda m: m.view(B, G, 1, N).expand(B, G, D // G, N).reshape(B, D, N)  # noqa: E731
    narrow = lambda m: m.view(B, G, D // G, N).sum(2).reshape(B, G * N)  # noqa: E731
    raw = delta + bias
    w = torch.nn.functional.softplus(raw, threshold=40.0)
    gate = torch.ones_like(u) if z is None else _silu(z)
    before, y = [], torch.zeros_like(u)
    core = torch.zeros_like(u)
    for s in range(t):
        live = (s < n)[:, None]
        before.append(h)
        new = torch.exp(w[s][..., None] * A) * h + (w[s] * u[s])[..., None] * wide(Bm[s])
        h = torch.where(live[..., None], new, h)
        core[s] = torch.where(live, (h * wide(Cm[s])).sum(-1) + skip * u[s], 0.0)
        y[s] = core[s] * gate[s]
    out = {"y": y, "h_out": h}
    d = {k: torch.zeros_like(u) for k in ("du", "ddelta", "dz")}
    d.update({k: torch.zeros_like(Bm) for k in ("dB", "dC")}, dA=torch.zeros_like(A), dskip=torch.zeros_like(skip), ddelta_bias=torch.zeros_like(bias))
    after = h
    for s in reversed(range(t)):
        live = (s < n)[:, None]
        gy = torch.where(live, dy[s] * gate[s], 0.0)
        if z is not None:
            sg = torch.sigmoid(z[s])
            d["dz"][s] = torch.where(live, dy[s] * core[s] * sg * (1 + z[s] * (1 - sg)), 0.0)
        g = g + gy[..., None] * wide(Cm[s])
        d["dC"][s] = narrow(gy[..., None] * after)
        d["dB"][s] = narrow(torch.where(live[..., None], g * (w[s] * u[s])[..., None], 0.0))
        a = torch.exp(w[s][..., None] * A)
        dlog, through = g * a * before[s], (g * wide(Bm[s])).sum(-1)
        dw = torch.where(live, (u[s] * through + (dlog * A).sum(-1)) * torch.sigmoid(raw[s]), 0.0)
        d["du"][s] = torch.where(live, w[s] * through, 0.0) + skip * gy
        d["ddelta"][s] = dw
        d["dA"] += torch.where(live[..., None], dlog * w[s][..., None], 0.0).sum(0)
        d["dskip"] += (gy * u[s]).sum(0)
        d["ddelta_bias"] += dw.sum(0)
        g = torch.where(live[..., None], g * a, g)
        after = before[s]
    return {**out, **d, "dh0": g}


def _scan_case(t, B, D, N, G, stretch, dtype, gate, ragged, seed):
    g = _gen(seed)
    T = torch.float32 if dtype == mb.FP32 else torch.bfloat16
    new = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    v = {"u": new(t, B, D).to(T), "delta": (new(t, B, D) * 0.5).to(T), "A": -torch.exp(new(D, N) * 0.5), "Bm": new(t, B, G * N).to(T),
         "Cm": new(t, B, G * N).to(T), "skip": new(D), "z": new(t, B, D).to(T) if gate else None, "bias": new(D) * 0.5 - 2.0,
         "h0": new(B, D, N), "dy": new(t, B, D).to(T), "dh": new(B, D, N)}
    n = torch.tensor([(t * (B - 1 - b)) // max(B - 1, 1) if b != 1 else 1 for b in range(B)], device=DEV) if ragged else torch.full((B,), t, device=DEV)
    return v, n


def _check_scan(t, B, D, N, G, stretch, dtype, gate, ragged):
    v, n = _scan_case(t, B, D, N, G, stretch, dtype, gate, ragged, t + N)
    want = _scan64(v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], G, v["skip"], v["z"], v["bias"], n, v["h0"], v["dy"], v["dh"])
    if ragged:
        beyond = torch.arange(t, device=DEV)[:, None] >= n
        for k in ("u", "delta", "Bm", "Cm", "z", "dy"):
            if v[k] is not None:
                v[k][beyond] = float("nan")
    d = mb.make_scan_desc(t, B, D, N, G, dtype, 1, stretch)
    got = {"y": torch.empty_like(v["u"]), "h_out": torch.empty_like(v["h0"]), "du": torch.empty_like(v["u"]), "ddelta": torch.empty_like(v["u"]),
           "dz": torch.empty_like(v["u"]) if gate else None, "dB": torch.empty_like(v["Bm"]), "dC": torch.empty_like(v["Cm"]), "dA": torch.empty_like(v["A"]),
           "dskip": torch.empty_like(v["skip"]), "ddelta_bias": torch.empty_like(v["bias"]), "dh0": torch.empty_like(v["h0"])}
    states, room = _room(mb.mebptt_scan_state_bytes(d)), _room(max(256, mb.mebptt_scan_workspace_bytes(d, True)))
    args = (v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], v["skip"], v["z"], v["bias"], n.int() if ragged else None, v["h0"])
    mb.mebptt_scan_forward(d, *args, got["y"], got["h_out"], states, room)
    room.fill_(0xA5)
    mb.mebptt_scan_backward(d, *args, v["dy"], v["dh"], states, got["du"], got["ddelta"], got["dA"], got["dB"], got["dC"], got["dskip"], got["dz"],
                            got["ddelta_bias"], got["dh0"], room)
    for k, x in got.items():
        if x is not None:
            _near(x, want[k], k)
    if ragged:
        for k in ("y", "du", "ddelta", "dB", "dC"):
            assert bool((got[k][beyond] == 0).all()), k


def _forward_chunks(desc):
    """Chunks of a forward launch, from the room that it needs for their states: none for a launch in one piece."""
    return mb.mebptt_scan_workspace_bytes(desc, False) // (4 * desc.B * desc.D * (desc.N + 1)) or 1


def _backward_room(desc, channels, chunks):
    """Room of a backward launch: dB and dC of every tile of `channels`, dA and the rest of every chunk, and the chunks' own gradients."""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    t, B, D, N, G = desc.t, desc.B, desc.D, desc.N, desc.G
    first = up(-(-(D // G) // channels) * t * B * G * 2 * N * 4) + up(chunks * B * D * (N + 2) * 4)
    return max(first + (up(chunks * B * D * N * 4) + up(chunks * B * D * 4) if chunks > 1 else 0), mb.mebptt_scan_workspace_bytes(desc, False))


# t, B, D, N, G, stretch; channels of a workgroup, chunks of the backward launch, of the forward launch
SCANS = [(100, 32, 1024, 16, 1, 16, 64, 1, 1),      # uncut, seven stretches, the last one of four steps
         (200, 33, 1024, 16, 1, 64, 64, 1, 1),      # four, the last one of eight steps
         (150, 17, 4100, 8, 1, 32, 128, 1, 1),      # a workgroup with four channels
         (600, 16, 1024, 32, 2, 256, 32, 1, 1),     # the longest stretches, two groups
         (300, 8, 1100, 64, 1, 128, 16, 1, 7),
         (520, 16, 1024, 16, 1, 16, 64, 4, 7),      # several stretches in each of a few chunks
         (1500, 1, 33, 16, 1, 16, 64, 47, 47),      # more chunks than are joined at once
         (1500, 2, 40, 6, 2, 64, 128, 24, 47)]


@pytest.mark.parametrize("t,B,D,N,G,stretch,channels,back_chunks,chunks", SCANS)
@pytest.mark.parametrize("dtype,gate,ragged", [(mb.FP32, True, False), (mb.FP32, False, True), (mb.BF16, True, True)])
def test_scan_over_many_stretches_and_chunks(t, B, D, N, G, stretch, channels, back_chunks, chunks, dtype, gate, ragged):
    desc = mb.make_scan_desc(t, B, D, N, G, dtype, 1, stretch)
    assert mb.mebptt_scan_workspace_bytes(desc, True) == _backward_room(desc, channels, back_chunks)
    assert _forward_chunks(desc) == chunks
    _check_scan(t, B, D, N, G, stretch, dtype, gate, ragged)


def test_the_vectorised_form_is_the_oracles():
    from oracle import selective as sel
    t, B, D, N, G = 9, 3, 4, 3, 2
    v, n = _scan_case(t, B, D, N, G, 16, mb.FP32, True, True, 1)
    got = _scan64(v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], G, v["skip"], v["z"], v["bias"], n, v["h0"], v["dy"], v["dh"])
    np_ = {k: x.double().cpu().numpy() for k, x in v.items()}
    y, h = sel.scan(np_["u"], np_["delta"], np_["A"], np_["Bm"], np_["Cm"], G, np_["skip"], np_["z"], np_["bias"], n.tolist(), np_["h0"], True)
    want = sel.scan_backward(np_["u"], np_["delta"], np_["A"], np_["Bm"], np_["Cm"], G, np_["skip"], np_["z"], np_["bias"], n.tolist(), np_["h0"], True,
                             np_["dy"], np_["dh"])
    for k, x in {**want, "y": y, "h_out": h}.items():
        assert np.abs(got[k].cpu().numpy() - x).max() <= 1e-12, k


# ---- launches ----------------------------------------------------------------------------------------

CHILD = """
import json, sys, tempfile, time
import torch
from torch.profiler import profile, ProfilerActivity
from paper_1606_03401_amd import binding as mb

new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda:0")
room = lambda n: new(max(n, 256), dtype=torch.uint8)

def product(M, N, K):
    d = mb.make_int8_desc(M, N, K, mb.BF16)
    a, b, sa, sb, out = new(M, K, dtype=torch.int8), new(N, K, dtype=torch.int8), new(M), new(N), new(M, N, dtype=torch.bfloat16)
    ws = room(mb.mebptt_int8_workspace_bytes(d))
    return lambda: mb.mebptt_int8_product(d, a, sa, b, sb, None, out, ws)

def conv(t, B, C, taps):
    d = mb.make_conv_desc(t, B, C, taps, mb.BF16, 1)
    x, y, dx = (new(t, B, C, dtype=torch.bfloat16) for _ in range(3))
    w, dw, ws = new(C, taps), new(C, taps), room(mb.mebptt_conv_workspace_bytes(d))
    def both():
        mb.mebptt_conv_forward(d, x, w, None, None, None, y)
        mb.mebptt_conv_backward(d, x, w, None, None, None, y, None, dx, dw, None, None, ws)
    return both

for call in json.load(sys.stdin):
    step = globals()[call[0]](*call[1:])
    step()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        time.sleep(0.05)     # the two clocks differ a little, and what seems to lie outside the traced time is dropped
        step()
        torch.cuda.synchronize()
        time.sleep(0.05)
    with tempfile.NamedTemporaryFile(suffix=".json") as f:
        p.export_chrome_trace(f.name)
        events = json.load(open(f.name))["traceEvents"]
    print("LAUNCHES " + json.dumps([(e["name"], e["args"]["grid"]) for e in events if e.get("cat") == "kernel"]), flush=True)
    del step
"""


def test_the_cases_take_the_paths_they_are_for():
    calls = [("product", *c[:3]) for c in TILES] + [("conv", *c[:4]) for c in CONVS]
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CHILD], input=json.dumps(calls), capture_output=True, text=True, cwd=root, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    got = [json.loads(line[9:]) for line in r.stdout.splitlines() if line.startswith("LAUNCHES ")]
    assert len(got) == len(calls)
    ceil = lambda a, b: -(-a // b)  # noqa: E731
    for (M, N, K, size), launches in zip(TILES, got):
        names = [n for n, _ in launches if "int8_" in n]
        assert ["copy" in n for n in names] == ([True] if K % 16 else []) + [False], names
        assert "int8_tile_kernel" in names[-1] and str(size) in names[-1], (M, N, K, names)
    for (t, B, C, taps, ahead, back, most), launches in zip(CONVS, got[len(TILES):]):
        grids = {k: g for n, g in launches for k in ("conv_forward", "conv_backward") if k in n}
        wide = 8 if C % 8 == 0 else 1
        assert grids["conv_forward"][:2] == [ceil(ceil(C, wide) * ceil(t, ahead), 256), B], (t, B, C, grids)
        columns, stretches = ceil(ceil(C, 4 if C % 4 == 0 else 1), 64), B * ceil(t, back)
        assert grids["conv_backward"][0] == columns and ceil(stretches, 4 * grids["conv_backward"][1]) == most, (t, B, C, grids)
        assert most > 1 or grids["conv_backward"][1] == ceil(stretches, 4)
