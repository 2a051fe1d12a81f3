"""The block's operators at the ends of the number ranges: scales whose product leaves fp32's range, infinities next to places that a launch only
fills up, rows that vanish."""
import numpy as np
import pytest
import torch

from oracle import selective as sel
from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


# ---- product -----------------------------------------------------------------------------------------

# K below 16; by rows; tiles of 128; tiles of 256, each with remainders
SHAPES = [(70, 33, 8), (5, 40, 200), (1000, 1021, 512), (4080, 4090, 1232)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("bias", [False, True])
def test_product_of_scales_from_both_ends_of_the_range(M, N, K, bias):
    """Scales around 1 for half of the rows and columns, 2^-75 or 2^70 for others, subnormal and zero ones, a row of zeros.  An output has four
    roundings, of the sum, of the scales' product, of theirs and of the bias' addition: 2^-22 of the value and of the bias; below the
    normal numbers half of the smallest one and as much again."""
    g = _gen(M)
    a = torch.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=torch.int8)
    b = torch.randint(-127, 128, (N, K), generator=g, device=DEV, dtype=torch.int8)
    a[1] = 0
    sa = torch.rand(M, generator=g, device=DEV) + 0.5
    sb = torch.rand(N, generator=g, device=DEV) + 0.5
    for s in (sa, sb):
        s[0::8] *= 2.0 ** -75
        s[1::8] *= 2.0 ** 70
        s[2::16] *= 2.0 ** -140
        s[10::16] = 0.0
    vb = torch.randn(N, generator=g, device=DEV) if bias else None
    out = torch.empty((M, N), device=DEV)
    d = mb.make_int8_desc(M, N, K, mb.FP32)
    mb.mebptt_int8_product(d, a, sa, b, sb, vb, out)
    v = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    want = v + vb.double() if bias else v
    inf = want.abs() > 3.4e38
    assert torch.equal(out[inf], want[inf].float())
    err = (out.double() - want).abs()
    assert bool((err <= 2.0 ** -22 * (v.abs() + (vb.double().abs() if bias else 0.0)) + 2.0 ** -149)[~inf].all())
    assert torch.equal(out[1], vb if bias else torch.zeros_like(out[1]))


# ---- convolution -------------------------------------------------------------------------------------


@pytest.mark.parametrize("C", [64, 63])
@pytest.mark.parametrize("t,lengths", [(9, None), (48, None), (16, [16, 9, 1]), (50, [50, 23, 1])])
def test_conv_gradient_next_to_an_infinite_last_input(C, t, lengths):
    """Linear taps: an infinity in a sequence's last step meets the last tap only; the other taps' gradients do not know it."""
    B, W = 3, 4
    rng = np.random.default_rng(t)
    x, dy = rng.standard_normal((t, B, C)), rng.standard_normal((t, B, C))
    w = rng.standard_normal((C, W))
    n = [t] * B if lengths is None else lengths
    up = lambda a, dtype=torch.float32: torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)  # noqa: E731
    x, dy, w = (up(a).double().cpu().numpy() for a in (x, dy, w))
    finite = x.copy()
    for b in range(B):
        x[n[b] - 1, b], finite[n[b] - 1, b] = np.inf, 0.0
    d = mb.make_conv_desc(t, B, C, W, mb.FP32, 0)
    dx, dw, db = torch.empty((t, B, C), device=DEV), torch.empty((C, W), device=DEV), torch.empty(C, device=DEV)
    ws = torch.empty(mb.mebptt_conv_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    mb.mebptt_conv_backward(d, up(x), up(w), None, None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV), None, up(dy), None,
                            dx, dw, db, None, ws)
    want_dx, want_dw, want_db, _ = sel.conv_backward(finite, w, None, lengths, None, False, dy, None)
    # sums of at most 150 products in 32 bits
    assert np.abs(dw.cpu().numpy()[:, :W - 1] - want_dw[:, :W - 1]).max() <= 2.0 ** -24 * 150 * (np.abs(dy).max() * np.abs(finite).max())
    assert not np.isfinite(dw.cpu().numpy()[:, W - 1]).any()
    assert np.abs(dx.cpu().numpy() - want_dx).max() <= 2.0 ** -24 * 8 * W * (np.abs(dy).max() * np.abs(w).max())
    assert np.abs(db.cpu().numpy() - want_db).max() <= 2.0 ** -24 * 150 * np.abs(dy).max() * 2


# ---- norm --------------------------------------------------------------------------------------------


@pytest.mark.parametrize("width", [8, 63, 1024, 2056, 9000])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_to_8_bits_of_rows_of_zeros_without_an_eps(width, residual):
    rows = 5
    g = _gen(width)
    x = torch.randn((rows, width), generator=g, device=DEV)
    res = torch.randn((rows, width), generator=g, device=DEV) if residual else None
    x[[1, 3]] = 0.0 if not residual else -res[[1, 3]]
    d = mb.make_norm_desc(rows, width, mb.FP32, mb.FP32, mb.INT8, 0.0)
    y, scale = torch.full((rows, width), 7, dtype=torch.int8, device=DEV), torch.full((rows,), 7.0, device=DEV)
    mb.mebptt_norm_forward(d, x, res, None, y, scale)
    assert bool((scale[[1, 3]] == 0).all()) and bool((y[[1, 3]] == 0).all())
    # the others: a row's largest value is 127 steps
    assert bool((y[[0, 2, 4]].abs().amax(1) == 127).all())
    r = x.double() if res is None else (x + res).double()
    top = (r * torch.rsqrt(r.square().mean(1, keepdim=True))).abs().amax(1)
    assert bool((scale[[0, 2, 4]].double() * 127 / top[[0, 2, 4]] - 1).abs().max() < 2.0 ** -18)
