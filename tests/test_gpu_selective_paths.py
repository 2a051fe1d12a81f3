"""The paths that the block's operators take at the sizes they are for: large tiles and copies of the product, whole stretches and many
chunks of the scan, long stretches of the convolution, more rows than workgroups of the norm.  Each against 64 bits."""
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
