"""How near the exact result the orthogonalised updates come, and that they repeat it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import gpu_util as G  # noqa: E402
from tests.test_gpu_muon import PREC, WORST, _close, _gauss, _gradient, _orth, ns  # noqa: E402

P = pytest.importorskip("paper_2310_00036_amd")


@PREC
def test_coefficients_that_shrink_as_far_as_is_allowed(prec):
    """Constant polynomials down to 2^-10 of the next one's: X times a power of two, within the bound of other
    coefficients."""
    x = G.q(_gauss(31, 2, 70, 400), prec)
    for co in ([(0.1, 0.0, 0.0)] * 3, [(2.0 ** -6, 0.0, 0.0), (2.0 ** 4, 0.0, 0.0)],
               [(2.0 ** -4, 0.0, 0.0), (2.0 ** -2, 0.0, 0.0), (2.0 ** 4, 0.0, 0.0)], [(0.0, 1.0, 0.0)],
               [(2.0 ** -6, 0.0, 0.0), (1.5, -0.5, 0.0), (1.5, -0.5, 0.0)]):
        _close(_orth(prec, x, len(co), co), ns(x, len(co), co), prec, WORST[prec], co)


# Gradient-like matrices in float32, five default steps in segments of 2, 2 and 1. An operand's pair of f16 numbers
# is off by at most 2^-23 of its element, uniformly (2^-23 / sqrt 3 rms), so a product of two by 2^-23 x 0.82, and the
# dropped lo lo product, 2^-11 / sqrt 3 squared, adds 2^-23 x 0.67: A is off by 2^-23 x 1.05 of its norm. A second step
# of a segment multiplies that by a^2 = 11.9 where singular values are small, and P by |b| / a = 1.4: 2.1e-6 of the
# result, 2.9e-6 for two segments of two, independent of each other. Float32 sums of hundreds to thousands of products
# are off by as much as a float32 evaluation's, 1e-6 to 2e-6. Added: 5e-6. A segment of three multiplies by 11.9 once more: 7e-6 to 17e-6 on the first of these.
F32_GRADIENT = 5e-6
# against a float32 evaluation: two bits fewer an operand
F32_RATIO = 4
GRADIENTS = [(6, 512, 128), (6, 64, 576), (6, 160, 100), (4, 128, 600), (1, 3872, 256), (2, 256, 1024), (2, 300, 300),
             (1, 2000, 500)]


def _strong(seed, b, r, c):
    """Eight strong directions over noise of about their norm."""
    rng = np.random.default_rng(seed)
    k = min(8, r, c)
    return 1e-3 * ((rng.standard_normal((b, r, k)) * 0.6 ** np.arange(k)) @ rng.standard_normal((b, k, c))
                   + rng.standard_normal((b, r, c)))


def _float32_steps(x):
    x = np.asarray(x, np.float32)
    tall = x.shape[-2] > x.shape[-1]
    X = np.ascontiguousarray(np.swapaxes(x, -1, -2)) if tall else x
    X = X / np.sqrt((X.astype(np.float64) ** 2).sum((-1, -2), keepdims=True)).astype(np.float32)
    a, b, c = (np.float32(v) for v in (3.4445, -4.7750, 2.0315))
    for _ in range(5):
        A = X @ np.swapaxes(X, -1, -2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return np.swapaxes(X, -1, -2) if tall else X


def _near(got, x, what):
    want, plain = ns(x), _float32_steps(x)
    for k in range(len(want)):
        e, f = G.rel_l2(got[k], want[k]), G.rel_l2(plain[k], want[k])
        print(what, x.shape, k, "error %.2e, float32 evaluation %.2e" % (e, f))
        assert e <= F32_GRADIENT, (what, k, e)
        assert e <= F32_RATIO * f, (what, k, e, f)


SHAPES = pytest.mark.parametrize("shape", GRADIENTS, ids=lambda s: "x".join(map(str, s)))


@SHAPES
@pytest.mark.parametrize("make", [_gradient, _strong])
def test_float32_orthogonalisation_of_gradients(make, shape):
    x = G.q(make(41, *shape), G.FP32)
    _near(_orth(G.FP32, x), x, "orthogonalize")


@SHAPES
@pytest.mark.parametrize("make", [_gradient, _strong])
def test_float32_updates_of_the_step(make, shape):
    """muon_step from zero parameters and momentum: p = -lr O(g), so the update's own error is seen."""
    t = G.torch()
    b, r, c = shape
    x = G.q(make(42, *shape), G.FP32)
    n = x.size
    p, m, v = (t.zeros(n, device="cuda:0") for _ in range(3))
    mats = P.muon_matrices([(k * r * c, r, c) for k in range(b)])
    cfg = P.muon_cfg(lr=0.5, momentum=0.5, nesterov=False)   # u = g / 2, exactly
    ws = G.ws_bytes(P.muon_workspace_bytes(n, mats, cfg))
    P.muon_step(n, mats, cfg, p, G.dev_f32(x), m, v, 1, None, ws)
    G.sync()
    scale = np.float64(np.float32(max(1.0, c / r) ** 0.5))
    _near(G.host(p).reshape(x.shape) / (-0.5 * scale), x, "step")


@pytest.mark.parametrize("shape", [(1, 7744, 512), (1, 4096, 4096), (2, 1001, 1531), (1, 3872, 256)],
                         ids=lambda s: "x".join(map(str, s)))
@PREC
def test_large_matrices_repeat_bit_for_bit(prec, shape):
    """The same call again, in another workspace with other contents."""
    x = G.q(_strong(43, *shape), prec)
    want = _orth(prec, x)
    t = G.torch()
    for k in range(3):
        t.empty(1 << 20 << k, dtype=t.uint8, device="cuda:0")   # (the next workspace lies elsewhere)
        assert np.array_equal(_orth(prec, x), want), k


@pytest.mark.parametrize("shape", [(1, 3872, 256), (24, 200, 260), (24, 100, 160), (6, 400, 1200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_float32_chains_lose_no_more_than_a_float32_evaluation(shape):
    """Over matrices of less than 512 on the smaller side, whose chains sum the small cross products of their f16 pairs
    apart: the mean error is at most 1.25 times a float32 evaluation's. The pairs' own rounding, 2^-23 x 1.05 of an A
    against float32's 2^-24 / sqrt 3 and its sums' roundings, is below that evaluation's error from 100 terms a sum on;
    what is left is the matrix cores' cutting, once per 32 terms. With all products in one sum it is 1.3 to 1.5."""
    x = G.q(_strong(44, *shape), G.FP32)
    want, plain, got = ns(x), _float32_steps(x), _orth(G.FP32, x)
    e = np.mean([G.rel_l2(g, w) for g, w in zip(got, want)])
    f = np.mean([G.rel_l2(p, w) for p, w in zip(plain, want)])
    print(shape, "error %.2e, float32 evaluation %.2e: %.2f" % (e, f, e / f))
    assert e <= 1.25 * f
