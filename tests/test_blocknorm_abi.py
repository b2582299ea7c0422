"""Refusals of the block norms' and the many-tensor clip's calls: on the host, before any HIP call."""
import ctypes as C

import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3
BIG = 1 << 40
MB = 1 << 20
lib = P.lib


def shape(prec=0, n=6, C_=64, groups=1, norm=1, norm2=2, act=0, eps=1e-5, **ld):
    return P.blocknorm_shape(prec, n, C_, groups, norm, norm2, act, eps, **ld)


F_ARGS = ("h", "gamma", "beta", "gate", "rscale", "res", "out", "gamma2", "beta2", "out2")
B_ARGS = ("dout", "dout2", "h", "gamma", "beta", "gate", "rscale", "out", "gamma2", "dh", "dgamma", "dbeta", "dgate",
          "drscale", "dres", "dgamma2", "dbeta2")


def fwd(s, **args):
    a = {n: (i + 1) * MB for i, n in enumerate(F_ARGS)}
    a.update(args)
    return lib.impala_blocknorm_fwd(C.byref(s) if s else None, *(a[n] for n in F_ARGS), None)


def bwd(s, ws=64 * MB, wsb=BIG, **args):
    a = {n: (i + 1) * MB for i, n in enumerate(B_ARGS)}
    a.update(args)
    return lib.impala_blocknorm_bwd(C.byref(s) if s else None, *(a[n] for n in B_ARGS), ws, wsb, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_shapes(call):
    assert call(None) == EINVAL
    for bad in (dict(prec=2), dict(n=-1), dict(C_=0), dict(groups=0), dict(groups=5), dict(norm=3), dict(norm=-1),
                dict(norm2=3), dict(act=3), dict(act=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(shape(**bad)) == EINVAL, bad
        assert P.impala_blocknorm_bwd_workspace_bytes(shape(**bad)) == 0
    assert call(shape(C_=8193)) == EUNSUPPORTED
    assert call(shape(groups=4)) == EUNSUPPORTED     # with a second norm
    for ld in ("ld_h", "ld_gate", "ld_out"):
        assert call(shape(**{ld: 63})) == EINVAL
        assert b"row stride" in lib.impala_last_error()


def test_null_arguments():
    assert fwd(shape(), h=None) == EINVAL and fwd(shape(), out=None) == EINVAL
    for bad in (dict(h=None), dict(dh=None), dict(out=None), dict(dout=None, dout2=None), dict(gate=None), dict(ws=None),
                dict(dout2=None)):
        assert bwd(shape(), **bad) == EINVAL, bad
    assert fwd(shape(n=0), h=None, out=None) == 0


def test_overlaps():
    n = 6 * 64 * 2
    for k in ("h", "gate", "res"):
        at = (F_ARGS.index(k) + 1) * MB
        for out in (at + 2, at + n - 2, at - n + 2):
            assert fwd(shape(), out=out) == EINVAL
            assert b"overlap" in lib.impala_last_error()
        assert fwd(shape(ld_out=72), out=at) == EINVAL     # itself, but with another stride
    assert fwd(shape(), out=10 * MB) == EINVAL             # out and out2
    for k in ("gamma", "beta", "rscale", "gamma2", "beta2"):
        assert fwd(shape(), out=(F_ARGS.index(k) + 1) * MB + 4) == EINVAL
    outs = ("dh", "dgate", "dres", "dgamma", "dbeta", "drscale", "dgamma2", "dbeta2")
    for o in outs:
        for other in outs + ("gamma", "beta", "rscale", "gamma2"):
            if o != other:
                assert bwd(shape(prec=1), **{o: (B_ARGS.index(other) + 1) * MB + 8}) == EINVAL, (o, other)
    for k in ("h", "out"):
        assert fwd(shape(), **{k: 20 * MB + 1}) == EINVAL
        assert fwd(shape(prec=1), **{k: 20 * MB + 2}) == EINVAL
    assert fwd(shape(), gamma=20 * MB + 2) == EINVAL


def test_workspace():
    need = P.impala_blocknorm_bwd_workspace_bytes(shape())
    assert need > 0 and bwd(shape(), wsb=need - 1) == EWORKSPACE
    assert bwd(shape(), ws=64 * MB + 8) == EINVAL
    with pytest.raises(ValueError):
        P.blocknorm_shape(0, 1, 8, ld_x=9)


def test_binding_checks_rows():
    t = torch.zeros(6, 80)[:, :64]
    s = P.blocknorm_shape(P.PREC_FP32, 6, 64)
    with pytest.raises(ValueError):
        P.impala_blocknorm_fwd(s, t, None, None, None, None, None, torch.zeros(6, 64), stream=torch.Stream(device="cpu"))


def clip(entries, limit=0.5, stats=None, ws=1 << 30, wsb=BIG, n=None):
    t = (P.GradTensor * max(1, len(entries)))(*(P.GradTensor(*e) for e in entries))
    return lib.grad_clip(t, len(entries) if n is None else n, limit, stats, ws, wsb, None)


def test_clip_refusals():
    one = (MB, 2 * MB, 1000, 1, 1)
    assert clip([one], n=-1) == EINVAL and clip([one], n=65537) == EINVAL
    assert lib.grad_clip(None, 1, 0.5, None, 1 << 30, BIG, None) == EINVAL
    for bad in ((None, 2 * MB, 10, 1, 1), (MB, 2 * MB, -1, 1, 1), (MB, 2 * MB, 10, 2, 1), (MB, 2 * MB, 10, 1, -1),
                (MB + 2, 2 * MB, 10, 1, 1), (MB, 2 * MB + 2, 10, 1, 1), (MB + 1, None, 10, 0, 0), (MB, MB, 10, 0, 1),
                (MB, MB, 10, 1, 0), (MB, MB + 4, 10, 1, 1), (MB + 4, MB, 10, 1, 1), (MB, 2 * MB, (1 << 40) + 1, 1, 1)):
        assert clip([bad]) == EINVAL, bad
    # a dst on another's src or dst, also in part; the same src twice is fine up to the workspace
    for other in ((2 * MB, 3 * MB, 10, 1, 1), (4 * MB, 2 * MB, 10, 1, 1), (4 * MB, 2 * MB + 3996, 10, 1, 1),
                  (4 * MB, MB + 400, 10, 1, 1), (MB, MB, 1000, 1, 1)):
        assert clip([one, other]) == EINVAL, other
        assert b"overlaps" in lib.impala_last_error()
    assert clip([one, (MB, 3 * MB, 1000, 1, 1)], wsb=0) == EWORKSPACE
    assert clip([(MB, MB, 1000, 1, 1)], wsb=8) == EWORKSPACE
    assert clip([one], ws=None) == EINVAL and clip([one], ws=(1 << 30) + 4) == EINVAL
    t = P.grad_tensors([(torch.zeros(3), None)])
    assert P.grad_clip_workspace_bytes(t) > 0
    for bad in ((torch.zeros(3), torch.zeros(4)), (torch.zeros(3).double(), None), (torch.zeros(3), torch.zeros(3).half()),
                (torch.zeros(3, 3).t(), None)):
        with pytest.raises(ValueError):
            P.grad_tensors([bad])
