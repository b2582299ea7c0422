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
