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
