"""How near the exact result the orthogonalised updates come, and that they repeat it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import gpu_util as G  # noqa: E402
from tests.test_gpu_muon import PREC, WORST, _close, _gauss, _orth, ns  # noqa: E402

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
