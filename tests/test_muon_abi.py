"""Coefficients and shapes that the orthogonalised-update calls refuse, on the host, before any HIP call."""
import ctypes as C

import pytest

P = pytest.importorskip("paper_2310_00036_amd")

EWORKSPACE, EUNSUPPORTED = -2, -3


def _orth(prec, co, r=200, c=100):
    """The status with a workspace of no bytes: EWORKSPACE says that everything before it was accepted."""
    rows = (C.c_float * (3 * len(co)))(*[v for row in co for v in row])
    return P.lib.muon_orthogonalize(prec, 2, r, c, 1 << 20, len(co), rows, 1e-7, 1 << 30, 1, 0, None)


def _step(co):
    cfg, mats = P.muon_cfg(lr=0.02, steps=len(co), coeffs=co), P.muon_matrices([(0, 200, 100)])
    return P.lib.muon_step(20000, mats, 1, C.byref(cfg), 1, 1, 1, 1, 1, None, 1, 0, None)


# polynomials that are constants: (a, 0, 0) multiplies X by a
SMALL, LARGE = (1e-8, 0.0, 0.0), (9e14, 0.0, 0.0)


def test_coefficients_are_checked_in_the_segments_that_run():
    """Five steps run as 2, 2, 1 in float32 and as 3, 2 in bf16. The product of the polynomials passes 10^15 in the
    third and fourth step, which share a segment in float32 only; the singular values stay below 10 throughout."""
    co = [SMALL, SMALL, LARGE, (100.0, 0.0, 0.0), (1.0, 0.0, 0.0)]
    assert _orth(P.PREC_FP32, co) == EUNSUPPORTED and b"grow" in P.lib.impala_last_error()
    for sides in ((40, 30), (1, 5), (3000, 2000)):
        assert _orth(P.PREC_FP32, co, *sides) == EUNSUPPORTED, sides


def test_accepted_coefficients_stay_accepted():
    quintic = (3.4445, -4.775, 2.0315)
    for prec in (P.PREC_FP32, P.PREC_BF16):
        for steps in range(1, 17):
            assert _orth(prec, [quintic] * steps) == EWORKSPACE, (prec, steps)
        for co in ([quintic, (3.0, -3.2, 1.2), (2.5, -2.2, 0.7), (1.875, -1.25, 0.375)], [(1.5, -0.5, 0.0)] * 9,
                   [(2.0, 0.0, 0.0)], [(1.0, 0.0, 0.0)] * 16):
            assert _orth(prec, co) == EWORKSPACE, co
            assert _step(co) == EWORKSPACE, co


def test_coefficients_that_shrink_a_matrix_below_what_its_planes_hold():
    """The first two steps of a segment multiply by 10^-8 each, the third by 9 x 10^14: under the scale of the third's
    polynomial, 2^-35, the second's is 0 in f16, and so would be the result, whose exact value is 0.09 X."""
    one = (1.0, 0.0, 0.0)
    for co in ([SMALL, SMALL, LARGE], [SMALL, SMALL, LARGE, (100.0, 0.0, 0.0), one], [SMALL, one], [one, SMALL, one, one],
               [(0.0, 0.0, 0.0)] * 5):
        assert _orth(P.PREC_BF16, co) == EUNSUPPORTED, co
        assert _orth(P.PREC_FP32, co) == EUNSUPPORTED, co
        assert _step(co) == EUNSUPPORTED, co
    # after a polynomial of zeros the scales followed from nothing: the factors of the next ones were infinite
    zeros = [(6.78e13, -244.5, -1.25e-4), (-9.87e14, 1e-5, -3.6e16), (0.0, -1e-18, 0.0), (5e12, 0.0, -3.7e5)]
    assert _orth(P.PREC_FP32, [(0.0, 0.0, 0.0)] + zeros) == EUNSUPPORTED
    tenth = (0.1, 0.0, 0.0)
    for co in ([tenth] * 2, [tenth] * 3, [(0.0, 1.0, 0.0)],
               [(3.0, 1e-9, 0.0)] * 2, [(8.287, -23.596, 17.301), (4.107, -2.948, 0.545)]):
        for prec in (P.PREC_FP32, P.PREC_BF16):
            assert _orth(prec, co) == EWORKSPACE, co


def test_the_workspace_query_refuses_the_coefficients_that_the_step_refuses():
    mats = P.muon_matrices([(0, 200, 100)])
    for co in ([(9.0, 9.0, 9.0)] * 5, [SMALL, SMALL, LARGE, (100.0, 0.0, 0.0), (1.0, 0.0, 0.0)]):
        assert _step(co) == EUNSUPPORTED
        assert P.muon_workspace_bytes(20000, mats, P.muon_cfg(lr=0.02, steps=5, coeffs=co)) == 0, co
        assert b"grow" in P.lib.impala_last_error()
    assert P.muon_workspace_bytes(20000, mats, P.muon_cfg(lr=0.02, steps=1, coeffs=[(1.5, -0.5, 0.0)])) > 0
