"""Refusals of the linear attention's calls: on the host, before any HIP call."""
import ctypes as C

import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3
BIG = 1 << 40
MB = 1 << 20


def shape(prec=0, T=4, E=3, heads=2, dk=16, dv=32, **strides):
    s = P.LinattnShape()
    s.prec, s.T, s.E, s.heads, s.dk, s.dv, s.scale = prec, T, E, heads, dk, dv, 1.0
    for n in ("q", "k", "gq", "gk"):
        setattr(s, n, P.LinattnStrides(E * heads * dk, heads * dk, dk))
    for n in ("v", "o", "gv"):
        setattr(s, n, P.LinattnStrides(E * heads * dv, heads * dv, dv))
    s.done_t, s.done_e = E, 1
    for n, v in strides.items():
        setattr(s, n, P.LinattnStrides(*v) if isinstance(v, tuple) else v)
    return s


def fwd(s, q=1 * MB, k=2 * MB, v=3 * MB, a=4 * MB, d=5 * MB, s0=6 * MB, o=7 * MB, s_out=8 * MB, ws=9 * MB, wsb=BIG):
    return P.lib.impala_linattn_fwd(C.byref(s) if s else None, q, k, v, a, d, s0, o, s_out, ws, wsb, None)


def bwd(s, do=1 * MB, q=2 * MB, k=3 * MB, v=4 * MB, a=5 * MB, d=6 * MB, s0=7 * MB, ds=8 * MB, dq=9 * MB, dk=10 * MB,
        dv=11 * MB, ds0=12 * MB, ws=13 * MB, wsb=BIG):
    return P.lib.impala_linattn_bwd(C.byref(s) if s else None, do, q, k, v, a, d, s0, ds, dq, dk, dv, ds0, ws, wsb, None)


def step(s, q=1 * MB, k=2 * MB, v=3 * MB, a=4 * MB, d=5 * MB, s0=6 * MB, o=7 * MB, s_out=8 * MB):
    return P.lib.impala_linattn_step(C.byref(s) if s else None, q, k, v, a, d, s0, o, s_out, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_shapes(call):
    assert call(None) == EINVAL
    for bad in (dict(prec=2), dict(T=-1), dict(E=-1), dict(heads=0), dict(dk=0), dict(dv=0)):
        assert call(shape(**bad)) == EINVAL, bad
        assert P.impala_linattn_workspace_bytes(shape(**bad)) == 0
    for bad in (dict(dk=129), dict(dv=129), dict(E=1 << 21, heads=2), dict(T=(1 << 30) + 1)):
        assert call(shape(**bad)) == EUNSUPPORTED, bad
    assert call(shape(E=0)) == 0


def test_null_arguments():
    for n in ("q", "k", "v", "a", "o"):
        assert fwd(shape(), **{n: None}) == EINVAL, n
    for n in ("do", "q", "k", "v", "a", "dq", "dk", "dv"):
        assert bwd(shape(), **{n: None}) == EINVAL, n
    assert step(shape(T=1), s_out=None) == EINVAL
    assert step(shape(T=2)) == EINVAL and step(shape(T=0)) == EINVAL


def test_strides_of_outputs():
    """Every axis has to step over what the smaller strides span; inputs may do as they like, but not go back."""
    for bad in (dict(o=(0, 64, 32)), dict(o=(192, 0, 32)), dict(o=(192, 64, 31)), dict(o=(191, 64, 32)), dict(o=(192, 63, 32))):
        assert fwd(shape(**bad)) == EINVAL, bad
        assert b"one place" in P.lib.impala_last_error()
    for n in ("gq", "gk", "gv"):
        assert bwd(shape(**{n: (1000, 100, 0)})) == EINVAL
    for n in ("q", "k", "v"):
        assert fwd(shape(**{n: (-96, 32, 16)})) == EINVAL
        assert b"negative" in P.lib.impala_last_error()
    assert fwd(shape(done_t=-1)) == EINVAL
    assert fwd(shape(o=(1 << 60, 64, 32))) == EINVAL and b"far" in P.lib.impala_last_error()
    for n in ("q", "k", "v", "o"):   # bf16 addresses are even, float32 ones multiples of four
        assert fwd(shape(), **{n: MB * 20 + 1}) == EINVAL
        assert fwd(shape(prec=1), **{n: MB * 20 + 2}) == EINVAL
    assert fwd(shape(), s_out=MB * 20 + 2) == EINVAL


def test_overlaps():
    """o with an input, elements between each other's only with the same strides; states as whole ranges."""
    es = 2
    n = 4 * 3 * 2 * 32 * es
    for at in (3 * MB, 3 * MB + n - es, 3 * MB - n + es):
        assert fwd(shape(), o=at) == EINVAL, at
        assert b"overlap" in P.lib.impala_last_error()
    # one buffer [T, E, 4, heads, 32] of q, k, v and o; each two of them
    packed = dict(dk=32, **{x: (3 * 256, 256, 32) for x in ("q", "k", "v", "o", "gq", "gk", "gv")})
    at = lambda i: MB + i * 64 * es   # noqa: E731
    for i in range(4):
        for j in range(4):
            args = dict(q=at(i), k=2 * MB, v=at(j), o=at(i))
            assert fwd(shape(**packed), **args) == EINVAL
    for off in (es, 31 * es, 32 * es, 63 * es):          # another head, or rows that share elements
        assert fwd(shape(**packed), q=at(0), k=at(1), v=at(2), o=at(0) + off) == EINVAL, off
    assert fwd(shape(**packed), q=at(0), k=at(1), v=at(2), o=at(0) + 256 * es) == EINVAL   # the next env's q
    assert fwd(shape(**packed), q=at(0), k=at(1), v=at(2), o=at(3) + 1) == EINVAL
    other = dict(packed, o=(3 * 512, 512, 32))
    assert fwd(shape(**other), q=at(0), k=at(1), v=at(2), o=at(3)) == EINVAL
    state = 3 * 2 * 16 * 32 * 4
    for s_out in (6 * MB + 4, 6 * MB + state - 4, 6 * MB - state + 4, 7 * MB, 3 * MB, 4 * MB, 5 * MB):
        assert fwd(shape(), s_out=s_out) == EINVAL, s_out
    for name in ("dq", "dk", "dv", "ds0"):
        for other in ("do", "q", "k", "v", "a", "d", "s0", "ds", "dq", "dk", "dv", "ds0"):
            if other != name:
                where = dict(zip(("do", "q", "k", "v", "a", "d", "s0", "ds", "dq", "dk", "dv", "ds0"), range(1, 13)))[other]
                assert bwd(shape(), **{name: where * MB}) == EINVAL, (name, other)


def test_workspace():
    need = P.impala_linattn_workspace_bytes(shape(T=1 << 14, E=1, heads=1, dk=128, dv=128), 1)
    s = shape(T=1 << 14, E=1, heads=1, dk=128, dv=128)
    far = {n: (i + 1) << 30 for i, n in enumerate(("do", "q", "k", "v", "a", "d", "s0", "ds", "dq", "dk", "dv", "ds0", "ws"))}
    if need:
        assert bwd(s, **far, wsb=need - 1) == EWORKSPACE
        assert bwd(s, **{**far, "ws": None}, wsb=0) == EINVAL
        assert bwd(s, **{**far, "ws": far["ws"] + 8}) == EINVAL


def test_binding_checks_tensors():
    q = torch.zeros(4, 3, 2, 16, dtype=torch.bfloat16)
    v = torch.zeros(4, 3, 2, 32, dtype=torch.bfloat16)
    s = P.linattn_shape(q, q, v, v, torch.zeros(4, 3, dtype=torch.uint8), 0.5)
    assert (s.T, s.E, s.heads, s.dk, s.dv, s.prec, s.scale) == (4, 3, 2, 16, 32, 0, 0.5)
    assert (s.q.t, s.q.e, s.q.h, s.o.t, s.done_t, s.done_e) == (96, 32, 16, 192, 3, 1)
    for bad in ((q, v, v, v, None), (q, q.float(), v, v, None), (q[0], q, v, v, None), (q, q, v, v[:, :2], None),
                (q, q, v.transpose(2, 3).contiguous().transpose(2, 3), v, None), (q.half(), q, v, v, None),
                (q, q, v, v, torch.zeros(4, 3)), (q, q, v, v, torch.zeros(3, 4, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            P.linattn_shape(*bad)
    with pytest.raises(ValueError):
        P.linattn_shape(q, q, v, v, None, 1.0, dq=v)
