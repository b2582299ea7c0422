"""Refusals of the group norm and orthogonalised-update calls: on the host, before any HIP call."""
import pytest

P = pytest.importorskip("paper_2310_00036_amd")

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3
BIG = 1 << 40


def test_groupnorm_refusals():
    lib = P.lib

    def fwd(prec=0, n=2, H=9, W=9, C_=32, groups=4, x=1 << 20, eps=1e-5, act=1, y=1 << 30, ws=1, wsb=BIG):
        return lib.impala_groupnorm_fwd(prec, n, H, W, C_, groups, x, None, None, eps, act, y, None, None, ws, wsb, None)

    def bwd(prec=0, n=2, C_=32, groups=4, dy=1 << 20, x=1 << 25, mean=16, rstd=16, act=1, dx=1 << 30, ws=1, wsb=BIG):
        return lib.impala_groupnorm_bwd(prec, n, 9, 9, C_, groups, dy, x, None, None, mean, rstd, act, dx, None, None, ws,
                                        wsb, None)

    for bad in (dict(prec=2), dict(n=-1), dict(H=0), dict(W=0), dict(groups=0), dict(groups=5), dict(C_=0), dict(act=3),
                dict(act=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(y=None), dict(H=5000, W=5000)):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(C_=1028) == EUNSUPPORTED
    # ranges that overlap in part: 2 x 9 x 9 x 32 bf16 are 10368 bytes
    assert fwd(y=(1 << 20) + 10366) == EINVAL and fwd(y=(1 << 20) - 10366) == EINVAL
    assert b"overlap" in lib.impala_last_error()
    need = P.impala_groupnorm_fwd_workspace_bytes(P.PREC_BF16, 2, 200, 200, 64, 4)
    assert need > 0 and fwd(H=200, W=200, C_=64, wsb=need - 1) == EWORKSPACE
    assert fwd(H=200, W=200, C_=64, ws=None, wsb=0) == EINVAL
    assert fwd(n=0, x=None, y=None, ws=None, wsb=0) == 0
    for bad in (dict(prec=-1), dict(groups=3), dict(act=7), dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None),
                dict(dx=None), dict(ws=None), dict(dx=1 << 25), dict(dx=(1 << 25) + 64), dict(dx=(1 << 20) + 64)):
        assert bwd(**bad) == EINVAL, bad
    need = P.impala_groupnorm_bwd_workspace_bytes(P.PREC_BF16, 2, 9, 9, 32, 4)
    assert need > 0 and bwd(wsb=need - 1) == EWORKSPACE
    assert bwd(C_=2048, groups=1) == EUNSUPPORTED
    assert P.impala_groupnorm_fwd_workspace_bytes(P.PREC_BF16, 2, 9, 9, 32, 5) == 0
    assert P.impala_groupnorm_bwd_workspace_bytes(P.PREC_BF16, 2, 9, 9, 2000, 5) == 0
