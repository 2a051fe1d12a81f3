"""The gated delta rule on rows that are no whole vectors, of so many sequences that a step of all of them, as copied rows, is over 2^32 bytes / 63 long: offsets from a chunk's first step to its
last one have 32 bits.  Sequences are independent of each other, so that a few of them at a time give the same bits."""
import pytest
import torch
from placed import DEV, NAN, room

from paper_1606_03401_amd import binding as mb

pytestmark = pytest.mark.gpu


def _run(desc_of, given, A, bias, out, dy, at):
    """Forward and backward of the sequences `at`."""
    q, k, v, a, b = (x[:, at] for x in given)
    y, dq, dk, dv, da, db = (x[:, at] for x in out)
    desc = desc_of(q.shape[1])
    states, ws = room(mb.mebptt_delta_state_bytes(desc)), room(mb.mebptt_delta_workspace_bytes(desc, True))
    mb.mebptt_delta_forward(desc, q, k, v, a, b, A, bias, None, None, y, None, states, ws)
    mb.mebptt_delta_backward(desc, q, k, v, a, b, A, bias, None, None, dy[:, at], None, states, dq, dk, dv, da, db, None, None, None, ws)


@pytest.mark.parametrize("dtype,code,H", [(torch.float32, mb.FP32, 32), (torch.bfloat16, mb.BF16, 64)])
def test_many_sequences_of_copied_rows(dtype, code, H):
    t, B, Hk, dk, dv, few = 64, 4096, 1, 10, 130, 512
    assert B * H * (132 if code == mb.FP32 else 136) * 63 * dtype.itemsize > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(6)

    def made(channels, s=1.0):      # the batch outermost
        m = torch.empty((B, t, channels), dtype=dtype, device=DEV)
        for i in range(0, B, few):
            m[i:i + few] = torch.randn((few, t, channels), generator=g, device=DEV) * s
        return m.transpose(0, 1)
    given = [made(c) for c in (Hk * dk, Hk * dk, H * dv, H, H)]
    dy, A, bias = made(H * dv, 0.1), -torch.rand(H, generator=g, device=DEV) - 0.1, torch.randn(H, generator=g, device=DEV) - 3
    empty = lambda n: [torch.full((n, t, c), NAN, dtype=dtype, device=DEV).transpose(0, 1) for c in (H * dv, Hk * dk, Hk * dk, H * dv, H, H)]  # noqa: E731
    desc_of = lambda n: mb.make_delta_desc(t, n, Hk, H, dk, dv, code, 1, 1, 64, dk ** -0.5)  # noqa: E731
    out = empty(B)
    _run(desc_of, given, A, bias, out, dy, slice(0, B))
    for i in range(0, B, few):
        at = slice(i, i + few)
        want = empty(few)
        _run(desc_of, [x[:, at] for x in given], A, bias, want, dy[:, at], slice(0, few))
        for x, w in zip(out, want):
            assert bool(w.isfinite().all()) and torch.equal(x[:, at], w), i
