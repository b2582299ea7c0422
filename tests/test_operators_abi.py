"""Refusals of the group norm and orthogonalised-update calls: on the host, before any HIP call."""
import ctypes as C

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
    # a launch of 2^32 threads
    assert fwd(n=1 << 24, H=1, W=1, C_=8) == EUNSUPPORTED and fwd(n=1 << 13, H=4096, W=4096, C_=64) == EUNSUPPORTED
    assert fwd(n=(1 << 24) - 1, H=1, W=1, C_=8, x=None) == EINVAL
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


def test_orthogonalize_refusals():
    lib = P.lib

    def orth(prec=1, b=2, r=40, c=30, x=1 << 20, steps=5, co=None, eps=1e-7, y=1 << 30, ws=1, wsb=BIG):
        return lib.muon_orthogonalize(prec, b, r, c, x, steps, co, eps, y, ws, wsb, None)

    for bad in (dict(prec=2), dict(b=-1), dict(r=0), dict(c=0), dict(steps=0), dict(steps=17), dict(eps=-1.0),
                dict(eps=float("nan")), dict(x=None), dict(y=None), dict(ws=None), dict(y=(1 << 20) + 4)):
        assert orth(**bad) == EINVAL, bad
    assert b"overlap" in lib.impala_last_error()
    for bad in (dict(r=1 << 15, c=1 << 15), dict(r=20000, c=20000), dict(b=1 << 20, r=1000, c=1000),
                dict(r=1, c=1 << 28), dict(r=1 << 22, c=3), dict(b=(1 << 21) + 1, r=1, c=1), dict(b=1 << 17, r=400, c=200)):
        assert orth(**bad) == EUNSUPPORTED, bad
    grow = (C.c_float * 15)(*([5.0, 5.0, 5.0] * 5))
    assert orth(co=grow) == EUNSUPPORTED and b"grow" in lib.impala_last_error()
    nan = (C.c_float * 15)(*([float("nan")] * 15))
    assert orth(co=nan) == EUNSUPPORTED
    assert P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 1 << 21, 3, 5, 5) > 0
    assert P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 1, 1, 1 << 21, 5) > 0
    assert P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 1, 1 << 14, 1 << 14, 5) > 0
    need = P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 2, 40, 30, 5)
    assert need > 0 and orth(wsb=need - 1) == EWORKSPACE
    assert orth(b=0, x=None, y=None, ws=None, wsb=0) == 0
    assert P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 2, 0, 30, 5) == 0
    assert P.muon_orthogonalize_workspace_bytes(P.PREC_FP32, 1, 1 << 15, 1 << 15, 5) == 0


def test_muon_step_refusals():
    lib = P.lib
    good = [(0, 10, 10), (100, 20, 5), (300, 7, 100)]

    def step(n=1000, mats=good, cfg=None, p=1, g=1, m=1, v=1, t=1, ws=1, wsb=BIG):
        mm = P.muon_matrices(mats)
        return lib.muon_step(n, mm, len(mm), C.byref(cfg if cfg is not None else P.muon_cfg(lr=0.02)), p, g, m, v, t,
                             None, ws, wsb, None)

    for bad in (dict(n=-1), dict(mats=[(0, 10, 10), (99, 2, 2)]), dict(mats=[(100, 2, 2), (0, 10, 11)]),
                dict(mats=[(-1, 2, 2)]), dict(mats=[(998, 2, 2)]), dict(mats=[(0, 0, 5)]), dict(mats=[(0, 5, -1)]),
                dict(mats=[(k, 1, 1) for k in range(513)]), dict(mats=[(2000, 1, 1)]), dict(t=0), dict(p=None),
                dict(g=None), dict(m=None), dict(v=None), dict(ws=None)):
        assert step(**bad) == EINVAL, bad
    # 32-bit offsets in a matrix's planes; the threads of a launch
    assert step(n=1 << 28, mats=[(0, 1, 1 << 28)]) == EINVAL
    assert step(n=64 << 28, mats=[(k << 28, 1 << 14, 1 << 14) for k in range(64)]) == EINVAL
    assert b"too large" in lib.impala_last_error()
    for kw in (dict(lr=-1.0), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-1.0), dict(steps=0),
               dict(steps=17), dict(scale=2), dict(eps=-1.0), dict(adam_lr=-1.0), dict(beta1=1.0), dict(beta2=1.5),
               dict(adam_eps=-1.0), dict(lr=float("nan"))):
        assert step(cfg=P.muon_cfg(**{"lr": 0.02, **kw})) == EINVAL, kw
    assert step(cfg=P.muon_cfg(lr=0.02, coeffs=[(9.0, 9.0, 9.0)] * 5)) == EUNSUPPORTED
    bad = P.muon_cfg(lr=0.02)
    bad.nesterov = 2
    assert step(cfg=bad) == EINVAL
    mm, cfg = P.muon_matrices(good), P.muon_cfg(lr=0.02)
    need = P.muon_workspace_bytes(1000, mm, cfg)
    assert need > 0 and step(wsb=need - 1) == EWORKSPACE
    assert lib.muon_step(1000, None, 1, C.byref(cfg), 1, 1, 1, 1, 1, None, 1, BIG, None) == EINVAL
    assert lib.muon_step(1000, mm, 3, None, 1, 1, 1, 1, 1, None, 1, BIG, None) == EINVAL
    assert step(n=0, mats=[], p=None, g=None, m=None, v=None, ws=None, wsb=0) == 0
    with pytest.raises(ValueError):
        P.muon_cfg(lr=0.02, coeffs=[(1.0, 2.0)] * 5)


def test_net_matrices_and_learner_cfg():
    from synth import NetShape, WORKLOADS
    for net in (NetShape(), NetShape(ch=(32, 64, 64), hidden=512)):
        lay = {name: (off, shape) for name, shape, off in P.impala_param_layout(net)}
        mats = {m.offset: (m.rows, m.cols) for m in P.muon_net_matrices(net)}
        want = {off: (9 * s[2], s[3]) if len(s) == 4 else (s[0], s[1]) for name, (off, s) in lay.items()
                if len(s) == 4 or name == "dense.w"}
        assert mats == want and len(mats) == 16
    wl = WORKLOADS[0].replace(optimizer="muon")
    cfg = P.learner_cfg(wl, P.PREC_BF16)
    adam = P.learner_workspace_bytes(wl.net, P.learner_cfg(WORKLOADS[0], P.PREC_BF16))
    assert P.learner_workspace_bytes(wl.net, cfg) > adam
    for field, v in (("muon_steps", 0), ("muon_momentum", 1.0), ("muon_lr", -1.0), ("muon_scale", 5),
                     ("muon_nesterov", 3), ("muon_eps", -1.0), ("optimizer", 3)):
        bad = P.learner_cfg(wl, P.PREC_BF16)
        setattr(bad, field, v)
        assert P.learner_workspace_bytes(wl.net, bad) == 0, field
