"""What is not finite in one group of columns stays in it: gradients of the norms around a block, where groups are no power of two of vectors, so that some of the lanes that
share a group have nothing of it.  Equal bits, as the other groups' values are computed the same way."""
import pytest
import torch
from placed import NAN
from test_gpu_join import CODE, _Call

from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("x_dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("width,group", [(72, 24), (256, 32), (81, 27), (120, 40), (4320, 1440), (3, 1), (9000, 3000)])
def test_gradients_of_other_groups(width, group, gate, x_dtype, layout):
    c = _Call(4, width, group, x_dtype, "fp32", layout, gate=gate, residual=False)
    names = ["y", "dx", "dw"] + (["dz"] if gate else [])
    c.forward()
    c.backward()
    want = {n: getattr(c, n).clone() for n in names}
    assert all(bool(x.isfinite().all()) for x in want.values())
    c.x[2, group // 2] = NAN
    c.forward()
    c.backward()
    for n in names:
        got = getattr(c, n)
        assert torch.equal(got[..., group:], want[n][..., group:]), n
        if n != "dw":
            assert torch.equal(got[[0, 1, 3]], want[n][[0, 1, 3]]), n
            assert bool(got[2, :group].isnan().any()), n
    assert c.m.clean()


def test_a_group_of_zeros_without_an_eps():
    """Its own results are 0 times infinity, those of the others are not touched."""
    c = _Call(3, 72, 24, "fp32", "fp32", residual=False)
    c.x[1, :24] = 0.0
    c.desc = mb.make_join_desc(3, 72, 24, CODE["fp32"], CODE["fp32"], c.scale, 0.0)
    c.forward()
    c.backward()
    for x in (c.y, c.dx, c.dz):
        assert bool(x[1, :24].isnan().all()) and bool(x[1, 24:].isfinite().all()) and bool(x[[0, 2]].isfinite().all())
