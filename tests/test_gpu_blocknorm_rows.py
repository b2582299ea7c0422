"""Block norms where a workgroup's row slots run empty or go round several times: eps = 0, many rows, in place."""
import pytest
import torch

from tests import memory_ref as ref
from tests.test_gpu_blocknorm import DEV, NAMES, TERMS, TYPES, dev, make, shape_of

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu


def forward(x, ty, groups, kinds, eps, two=True, over=None):
    a = {k: dev(v) for k, v in x.items()}
    out, out2 = torch.full_like(a["h"], 9.0), torch.full_like(a["h"], 9.0) if two else None
    if over:
        out = a[over[0]]
        out2 = a[over[1]] if two else None
    P.impala_blocknorm_fwd(shape_of(x, ty, groups, *kinds, eps), a["h"], a["gamma"], a["beta"], a["gate"], a["rscale"],
                           a["res"], out, a["gamma2"], a["beta2"], out2)
    return out, out2


def backward(x, ty, groups, kinds, eps, over=None):
    a = {k: dev(v) for k, v in x.items()}
    n, C = x["h"].shape
    o = {k: torch.full((n, C) if k in ("dh", "dgate", "dres") else (C,), 9.0, device=DEV,
                       dtype=TYPES[ty] if k in ("dh", "dgate", "dres") else torch.float32) for k in NAMES}
    if x["dout2"] is None:
        o["dgamma2"] = o["dbeta2"] = None
    for k, name in (over or {}).items():
        o[k] = a[name]
    s = shape_of(x, ty, groups, *kinds, eps)
    ws = torch.full((P.impala_blocknorm_bwd_workspace_bytes(s),), 255, dtype=torch.uint8, device=DEV)
    P.impala_blocknorm_bwd(s, a["dout"], a["dout2"], a["h"], a["gamma"], a["beta"], a["gate"], a["rscale"], a["out"],
                           a["gamma2"], *(o[k] for k in NAMES), ws)
    return o


def check(x, ty, groups, kinds, eps, out, grads):
    norm, norm2, act = kinds
    want, mag = ref.blocknorm(x["h"], x["gamma"], x["beta"], x["gate"], x["rscale"], x["res"], groups, norm, act, eps)
    ref.assert_close("out", out[0], want, mag, TERMS, False, ty == "bf16")
    if out[1] is not None:
        want, mag = ref.blocknorm_second(out[0].cpu(), x["gamma2"], x["beta2"], norm2, eps)
        ref.assert_close("out2", out[1], want, mag, TERMS, False, ty == "bf16")
    want = ref.blocknorm_grads(x["dout"], x["dout2"], x["h"], x["gamma"], x["beta"], x["gate"], x["rscale"], x["out"],
                               x["gamma2"], groups, norm, norm2, act, eps)
    for k, g in grads.items():
        if g is not None:
            rows = k in ("dh", "dgate", "dres")
            ref.assert_close(k, g, *want[k], TERMS + (0 if rows else x["h"].shape[0]), False, ty == "bf16" and rows)


KINDS = [(P.NORM_LAYER, P.NORM_RMS, P.GATE_SILU), (P.NORM_RMS, P.NORM_LAYER, P.GATE_SIGMOID),
         (P.NORM_NONE, P.NORM_RMS, P.GATE_LINEAR), (P.NORM_RMS, P.NORM_NONE, P.GATE_SILU)]


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("n,C,groups", [(1, 256, 1), (37, 256, 1), (100, 256, 1), (5, 24, 1), (3, 1100, 1), (2, 4100, 1),
                                        (37, 60, 5), (1, 40, 2)])
def test_eps_of_zero(n, C, groups, ty):
    """No row is constant, so every statistic is finite, whatever slots behind the last row hold."""
    for i, kinds in enumerate(KINDS):
        x = make(n, C, ty, seed=i)
        if groups > 1:
            x["dout2"] = None
        check(x, ty, groups, kinds, 0.0, forward(x, ty, groups, kinds, 0.0, groups == 1), backward(x, ty, groups, kinds, 0.0))


# Workgroups are at most 1024 forward and 512 backward: here each goes round several times, some without a last row.
MANY = [(9001, 256, 1), (2100, 1531, 1), (1100, 4100, 1), (90001, 24, 3), (3000, 2048, 2)]


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("n,C,groups", MANY)
def test_more_rows_than_places(n, C, groups, ty):
    for i, kinds in enumerate(KINDS[:2]):
        x = make(n, C, ty, seed=i)
        if groups > 1:
            x["dout2"] = None
        check(x, ty, groups, kinds, 1e-5, forward(x, ty, groups, kinds, 1e-5, groups == 1), backward(x, ty, groups, kinds, 1e-5))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("n,C,groups", MANY)
def test_more_rows_than_places_in_place(n, C, groups, ty):
    """An output on an input, the next rows of which may be on their way: the bits of outputs of their own."""
    kinds, two = KINDS[0], groups == 1
    x = make(n, C, ty, seed=7)
    if not two:
        x["dout2"] = None
    want, grads = forward(x, ty, groups, kinds, 1e-5, two), backward(x, ty, groups, kinds, 1e-5)
    for over in (("h", "gate"), ("res", "h"), ("gate", "res")):
        got = forward(x, ty, groups, kinds, 1e-5, two, over)
        assert torch.equal(got[0], want[0]) and (not two or torch.equal(got[1], want[1])), over
    for over in (dict(dh="h", dgate="gate", dres="dout"), dict(dh="gate", dgate="dout", dres="h"),
                 dict(dh="out", dgate="h", dres="gate") if two else dict(dh="dout")):
        got = backward(x, ty, groups, kinds, 1e-5, over)
        assert all(torch.equal(got[k], g) for k, g in grads.items() if g is not None), over


@pytest.mark.parametrize("size", [1e-17, 1e-18, 3e-19, 1e-19, 3e-20, 1e-20])
def test_rows_whose_squares_are_denormal(size):
    """eps = 0 and float32 rows down to 1e-20. A square and the sum it goes into are off by half of 2^-149 each, the mean by
    as much again, so the mean square ms is off by at most 3 2^-150 and its root by 1.5 2^-150 / ms of itself."""
    n, C = 9, 200
    x = make(n, C, "f32")
    h = (torch.randn(n, C, generator=torch.Generator().manual_seed(1)) * size)
    d = h.double()
    ms = d.square().mean(-1, keepdim=True)
    rel = TERMS * 2.0 ** -24 + 1.5 * 2.0 ** -150 / ms
    assert rel.max() < 1e-4
    s = P.blocknorm_shape(P.PREC_FP32, n, C, norm=P.NORM_RMS, eps=0.0)
    out = torch.empty(n, C, device=DEV)
    P.impala_blocknorm_fwd(s, dev(h), None, None, None, None, None, out)
    want = d / ms.sqrt()
    assert ((out.double().cpu() - want).abs() <= rel * want.abs()).all()
    # dh = r (g - xh <g xh>): r and each xh off by rel, in up to four places a term
    g = x["dout"]
    dh, ws = torch.empty_like(out), torch.empty(P.impala_blocknorm_bwd_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    P.impala_blocknorm_bwd(s, dev(g), None, dev(h), None, None, None, None, None, None, dh, *[None] * 7, ws)
    g, r = g.double(), 1 / ms.sqrt()
    want_dh = r * (g - want * (g * want).mean(-1, keepdim=True))
    mag = r * (g.abs() + want.abs() * (g * want).abs().mean(-1, keepdim=True))
    assert ((dh.double().cpu() - want_dh).abs() <= 4 * rel * mag).all()
