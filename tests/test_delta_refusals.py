"""What the delta rule, the norms around a block and AdamW refuse, and the room that they ask for.  No GPU: a refused call enqueues nothing, and pointers are
not looked into before the arguments are right."""
import ctypes as C

import pytest

from paper_1606_03401_amd import binding as mb

P = 1 << 20      # an address that nobody reads
GOOD = dict(t=100, B=2, Hk=1, H=2, dk=16, dv=24, dtype=mb.BF16, activate=1, normalise=1, stretch=64, scale=1.0, eps=1e-6)


def _desc(**kw):
    return mb.make_delta_desc(**{**GOOD, **kw})


def _seq(channels, B=2, data=P):
    return mb.mebptt_seq(data, B * channels, channels)


def _inputs(**kw):
    v = dict(q=_seq(16), k=_seq(16), v=_seq(48), a=_seq(2), b=_seq(2), A=P, a_bias=P, lengths=None, h0=None)
    v.update(kw)
    return mb.mebptt_delta_inputs(*v.values())


def _grads(**kw):
    v = dict(dq=_seq(16), dk=_seq(16), dv=_seq(48), db=_seq(2), da=_seq(2), dA=P, da_bias=P, dh0=None)
    v.update(kw)
    return mb.mebptt_delta_grads(*v.values())


def _forward(desc=None, y=None, states=None, states_bytes=0, ws=P, ws_bytes=1 << 40, **kw):
    d = desc or _desc()
    return mb.lib().mebptt_delta_forward(C.byref(d), C.byref(_inputs(**kw)), y or _seq(48), None, states, states_bytes, ws, ws_bytes, None)


def _backward(desc=None, grads=None, states=P, states_bytes=1 << 40, ws=P, ws_bytes=1 << 40, dy=None, **kw):
    d = desc or _desc()
    return mb.lib().mebptt_delta_backward(C.byref(d), C.byref(_inputs(**kw)), dy or _seq(48), None, states, states_bytes, C.byref(grads or _grads()), ws, ws_bytes, None)


BAD = [dict(t=-1), dict(t=(1 << 30) + 1), dict(B=-1), dict(B=65536), dict(Hk=0), dict(H=0), dict(Hk=2, H=3), dict(H=1025), dict(B=65535, H=128), dict(dk=0), dict(dk=129),
       dict(dv=0), dict(dv=257), dict(dtype=mb.INT8), dict(dtype=7), dict(eps=-1.0), dict(eps=float("nan"))]


@pytest.mark.parametrize("kw", BAD)
def test_delta_descriptors_that_no_call_accepts(kw):
    d = _desc(**kw)
    assert mb.mebptt_delta_workspace_bytes(d, False) == 0 and mb.mebptt_delta_workspace_bytes(d, True) == 0 and mb.mebptt_delta_state_bytes(d) == 0
    assert _forward(d) == mb.EINVAL and _backward(d) == mb.EINVAL
    assert mb.lib().mebptt_delta_step(C.byref(d), C.byref(_inputs()), P, 2, None, _seq(48), P, None) == mb.EINVAL


@pytest.mark.parametrize("stretch", [0, -64, 63, 65, 96, (1 << 20) + 64])
def test_stretches(stretch):
    d = _desc(stretch=stretch)
    assert mb.mebptt_delta_state_bytes(d) == 0 and mb.mebptt_delta_workspace_bytes(d, True) == 0 and mb.mebptt_delta_workspace_bytes(d, False) > 0
    assert _forward(d, states=P, states_bytes=1 << 40) == mb.EINVAL and _backward(d) == mb.EINVAL


def test_delta_arguments():
    assert mb.lib().mebptt_delta_forward(None, C.byref(_inputs()), _seq(48), None, None, 0, P, 1 << 40, None) == mb.EINVAL
    d = _desc()
    assert mb.lib().mebptt_delta_forward(C.byref(d), None, _seq(48), None, None, 0, P, 1 << 40, None) == mb.EINVAL
    for n, c in (("q", 16), ("k", 16), ("v", 48), ("b", 2)):
        assert _forward(**{n: _seq(c, data=None)}) == mb.EINVAL and n in mb.mebptt_last_error()
    assert _forward(A=None) == mb.EINVAL and "A" in mb.mebptt_last_error()
    assert _forward(y=_seq(48, data=None)) == mb.EINVAL
    for bad in ((-32, 16), ((1 << 23) + 1, 16)):
        assert _forward(q=mb.mebptt_seq(P, *bad)) == mb.EINVAL and "stride_t" in mb.mebptt_last_error()
        assert _forward(a=mb.mebptt_seq(P, *bad)) == mb.EINVAL
        assert _backward(dy=mb.mebptt_seq(P, *bad)) == mb.EINVAL and _backward(grads=_grads(dq=mb.mebptt_seq(P, *bad))) == mb.EINVAL
    for bad in ((48, 48), (96, 47), (0, 48), (47, 4800)):
        assert _forward(y=mb.mebptt_seq(P, *bad)) == mb.EINVAL and "overlap" in mb.mebptt_last_error()
    for n in ("dq", "dk", "dv", "db", "da"):
        assert _backward(grads=_grads(**{n: mb.mebptt_seq(None, 96, 48)})) == mb.EINVAL and n in mb.mebptt_last_error()
    assert _backward(states=None) == mb.EINVAL
    assert mb.lib().mebptt_delta_backward(C.byref(d), C.byref(_inputs()), _seq(48), None, P, 1 << 40, None, P, 1 << 40, None) == mb.EINVAL
    step = lambda t=1, pool=P, slots=2, y=None: mb.lib().mebptt_delta_step(  # noqa: E731
        C.byref(_desc(t=t)), C.byref(_inputs()), pool, slots, None, y or _seq(48), P, None)
    assert step(t=2) == mb.EINVAL and step(pool=None) == mb.EINVAL and step(slots=-1) == mb.EINVAL and step(y=mb.mebptt_seq(P, 0, 47)) == mb.EINVAL


def test_delta_room():
    d = _desc()
    need, back, states = mb.mebptt_delta_workspace_bytes(d, False), mb.mebptt_delta_workspace_bytes(d, True), mb.mebptt_delta_state_bytes(d)
    assert back >= need > 0 and states == 2 * 2 * 2 * 16 * 24 * 4
    assert _forward(ws_bytes=need - 1) == mb.EWORKSPACE and _forward(ws=P + 128) == mb.EWORKSPACE and _forward(ws=None) == mb.EWORKSPACE
    assert _forward(states=P, states_bytes=states - 1) == mb.EWORKSPACE and _forward(states=P + 4, states_bytes=1 << 40) == mb.EWORKSPACE
    assert _backward(ws_bytes=back - 1) == mb.EWORKSPACE and _backward(states_bytes=states - 1) == mb.EWORKSPACE
    # the backward pass's room goes with the stretch, a forward pass's does not with t beyond what it takes at a time
    size = lambda t, stretch, B=64: mb.mebptt_delta_workspace_bytes(_desc(t=t, stretch=stretch, B=B, Hk=8, H=8, dk=128, dv=128), True)  # noqa: E731
    assert size(10000, 64) < size(10000, 256) < size(10000, 1024)
    f = lambda t: mb.mebptt_delta_workspace_bytes(_desc(t=t, B=64, Hk=8, H=8, dk=128, dv=128), False)  # noqa: E731
    assert f(100000) == f(10000)


# ---- join ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(width=0), dict(width=16385, group=16385), dict(group=0), dict(group=5), dict(width=8192, group=1), dict(x_dtype=mb.INT8),
                                dict(residual_dtype=mb.INT8), dict(eps=-1.0)])
def test_join_descriptors_that_no_call_accepts(kw):
    d = mb.make_join_desc(**{**dict(rows=4, width=64, group=16, x_dtype=mb.BF16, residual_dtype=mb.FP32, scale=1.0, eps=1e-5), **kw})
    assert mb.mebptt_join_workspace_bytes(d) == 0
    assert mb.lib().mebptt_join_forward(C.byref(d), P, 1 << 20, None, 0, None, None, 0, None, P, 1 << 20, None, 0, None, None, None) == mb.EINVAL


def test_every_width_has_a_shape():
    """Widths and groups of every kind within the limits are taken: the next refusal is the missing pointer."""
    for width, group in ((1, 1), (4096, 1), (16384, 4), (16384, 8), (16384, 16384), (16380, 9 * 4), (16371, 17 * 9), (16383, 16383), (16384, 4096), (12, 3), (8191, 8191), (16368, 11)):
        if width % group:
            continue
        d = mb.make_join_desc(4, width, group, mb.BF16, mb.FP32)
        assert mb.mebptt_join_workspace_bytes(d) > 0
        assert mb.lib().mebptt_join_forward(C.byref(d), None, width, None, 0, None, None, 0, None, None, width, None, 0, None, None, None) == mb.EINVAL
        assert "required" in mb.mebptt_last_error()


def test_join_arguments():
    d = mb.make_join_desc(4, 64, 16, mb.BF16, mb.FP32)
    f = lambda x=P, ldx=64, z=None, ldz=0, res=None, ldr=0, wn=None, y=P, ldy=64, out=None, ldo=0, rn=None: mb.lib().mebptt_join_forward(  # noqa: E731
        C.byref(d), x, ldx, z, ldz, None, res, ldr, wn, y, ldy, out, ldo, None, rn, None)
    for kw in (dict(x=None), dict(y=None), dict(ldx=63), dict(ldy=63), dict(z=P, ldz=63), dict(res=P, ldr=63), dict(res=P, ldr=64, out=P, ldo=63), dict(wn=P), dict(out=P, ldo=64),
               dict(rn=P)):
        assert f(**kw) == mb.EINVAL, kw

    def b(x=P, z=None, r=None, wn=None, rstd=P, rn=None, dy=P, do=None, dx=P, dz=None, dw=None, dr=None, dwn=None, ws=P, n=1 << 30, ld=64):
        return mb.lib().mebptt_join_backward(C.byref(d), x, ld, z, 64, None, r, 64, wn, rstd, rn, dy, 64, do, 64, dx, 64, dz, 64, dw, dr, 64, dwn, ws, n, None)
    for kw in (dict(x=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(z=P), dict(dz=P), dict(wn=P), dict(rn=P), dict(do=P), dict(dr=P), dict(dwn=P), dict(r=P), dict(ld=63)):
        assert b(**kw) == mb.EINVAL, kw
    need = mb.mebptt_join_workspace_bytes(d)
    assert need >= 2 * 64 * 4
    assert b(dw=P, ws=None) == mb.EWORKSPACE and b(dw=P, n=need - 1) == mb.EWORKSPACE and b(dw=P, ws=P + 8) == mb.EWORKSPACE


# ---- AdamW -----------------------------------------------------------------------------------------


def _tensors(*changes):
    t = [dict(param=P, grad=P, m=P, v=P, m_scale=None, v_scale=None, copy=None, n=1000, grad_dtype=mb.FP32, state_dtype=mb.FP32, flags=0, reserved=0) for _ in changes]
    for x, c in zip(t, changes):
        x.update(c)
    return (mb.mebptt_adamw_tensor * len(t))(*[mb.mebptt_adamw_tensor(*x.values()) for x in t])


def _prepare(*changes):
    return mb.lib().mebptt_adamw_prepare(_tensors(*changes), len(changes), P, 1 << 40, None)


def test_adamw_tensors():
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(grad_dtype=mb.INT8), dict(state_dtype=mb.BF16), dict(state_dtype=mb.INT8), dict(flags=2),
                dict(reserved=1), dict(n=-1), dict(n=(1 << 40) + 1)):
        assert _prepare({}, bad) == mb.EINVAL, bad
    lib = mb.lib()
    assert lib.mebptt_adamw_prepare(None, 1, P, 1 << 40, None) == mb.EINVAL and lib.mebptt_adamw_prepare(_tensors({}), -1, P, 1 << 40, None) == mb.EINVAL
    assert lib.mebptt_adamw_prepare(_tensors({}), 65537, P, 1 << 40, None) == mb.EINVAL
    assert lib.mebptt_adamw_table_bytes(_tensors(dict(n=-1)), 1) == 0 and lib.mebptt_adamw_workspace_bytes(_tensors(dict(n=-1)), 1) == 0
    many = _tensors(*[dict(n=1 << 40)] * 5)
    assert lib.mebptt_adamw_table_bytes(many, 5) == 0
    need = lib.mebptt_adamw_table_bytes(_tensors({}, {}), 2)
    assert need > 0
    for table, n in ((None, need), (P, need - 256), (P + 16, need)):
        assert lib.mebptt_adamw_prepare(_tensors({}, {}), 2, table, n, None) == mb.EWORKSPACE


def test_adamw_steps():
    t, lib = _tensors({}), mb.lib()
    need = lib.mebptt_adamw_table_bytes(t, 1)
    good = dict(rate=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=0.0, step=1)
    step = lambda table=P, n=need, step=None, **kw: lib.mebptt_adamw_step(  # noqa: E731
        C.byref(mb.make_adamw_desc(**{**good, **kw})), t, 1, table, n, None, None, step, None)
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-9)):
        assert step(**kw) == mb.EINVAL, kw
    d = mb.make_adamw_desc(**{**good, "step": 0})
    assert lib.mebptt_adamw_step(C.byref(d), t, 1, P, need, None, None, None, None) == mb.EINVAL
    assert lib.mebptt_adamw_step(None, t, 1, P, need, None, None, None, None) == mb.EINVAL
    assert step(table=None) == mb.EWORKSPACE and step(n=need - 1) == mb.EWORKSPACE
    norm = lambda limit=1.0, out=P, ws=P, n=1 << 20: lib.mebptt_adamw_norm(t, 1, P, need, limit, out, ws, n, None)  # noqa: E731
    assert norm(limit=0.0) == mb.EINVAL and norm(limit=float("nan")) == mb.EINVAL and norm(out=None) == mb.EINVAL
    assert norm(ws=None) == mb.EWORKSPACE and norm(n=8) == mb.EWORKSPACE
    unpack = lambda n=10, codes=P, dtype=mb.FP32: lib.mebptt_adamw_unpack(codes, P, n, 1, P, dtype, None)  # noqa: E731
    assert unpack(n=-1) == mb.EINVAL and unpack(codes=None) == mb.EINVAL and unpack(dtype=mb.INT8) == mb.EINVAL


def test_join_flags_that_mean_nothing():
    for field, value in (("again", 2), ("again", -1), ("reserved", 1)):
        d = mb.make_join_desc(4, 64, 16, mb.BF16, mb.FP32)
        assert mb.mebptt_join_workspace_bytes(d) > 0
        setattr(d, field, value)
        assert mb.mebptt_join_workspace_bytes(d) == 0
        assert mb.lib().mebptt_join_forward(C.byref(d), P, 64, None, 0, None, None, 0, None, P, 64, None, 0, None, None, None) == mb.EINVAL
