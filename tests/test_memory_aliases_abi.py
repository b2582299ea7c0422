"""Which arrays the memory core's calls take as each other: on the host, before any HIP call."""
import pytest
import torch

from tests.test_blocknorm_abi import B_ARGS, F_ARGS, MB
from tests.test_blocknorm_abi import bwd as bn_bwd
from tests.test_blocknorm_abi import fwd as bn_fwd
from tests.test_blocknorm_abi import lib
from tests.test_blocknorm_abi import shape as bn_shape
from tests.test_linattn_abi import bwd as la_bwd
from tests.test_linattn_abi import fwd as la_fwd
from tests.test_linattn_abi import shape as la_shape

EINVAL = -1


@pytest.mark.parametrize("n", [1, 2])
def test_a_row_is_not_a_vector_over_the_channels(n):
    """One float32 row has a vector's size: it is refused in its place like several rows."""
    s = bn_shape(prec=1, n=n)
    for out in ("out", "out2"):
        for k in ("gamma", "beta", "rscale", "gamma2", "beta2"):
            assert bn_fwd(s, **{out: (F_ARGS.index(k) + 1) * MB}) == EINVAL, (out, k)
            assert b"overlap" in lib.impala_last_error()
    vectors = ("gamma", "beta", "rscale", "gamma2")
    rows = ("dout", "dout2", "h", "gate", "out")
    for o, others in [(o, vectors) for o in ("dh", "dgate", "dres")] + [
            (o, vectors + rows) for o in ("dgamma", "dbeta", "drscale", "dgamma2", "dbeta2")]:
        for k in others:
            assert bn_bwd(s, **{o: (B_ARGS.index(k) + 1) * MB}) == EINVAL, (o, k)
            assert b"overlap" in lib.impala_last_error()


def fused(T, E, H, dk, dv, order="ehx"):
    """Strides and element offsets of parts [.., H, dk] x 3 and [.., H, dv] x 3 in one row of a buffer [T, E, row]."""
    widths = dict(gq=dk, q=dk, k=dk, gk=dk, gv=dv, v=dv, o=dv)
    row, at, strides = 0, {}, {}
    for n in ("q", "gq", "k", "gk", "v", "gv", "o"):
        at[n] = row
        row += H * widths[n]
    for n, w in widths.items():
        strides[n] = (E * row, row, w) if order == "ehx" else (row, T * row, w)
    return at, strides


@pytest.mark.parametrize("order", ["ehx", "thx"])
@pytest.mark.parametrize("T,E,H,dk,dv", [(4, 3, 2, 16, 32), (5, 2, 3, 7, 9), (1, 4, 2, 8, 24), (3, 1, 1, 8, 16), (2, 2, 4, 128, 64)])
def test_parts_of_one_buffer_with_other_widths(T, E, H, dk, dv, order):
    """q, k of one width and v, o of another side by side, gradients too: no element is in two of them, so none is refused for
    an overlap; a part that reaches into the next one is."""
    at, strides = fused(T, E, H, dk, dv, order)
    s = la_shape(T=T, E=E, heads=H, dk=dk, dv=dv, **strides)
    p = {n: 64 * MB + 2 * a for n, a in at.items()}
    f = dict(q=p["q"], k=p["k"], v=p["v"], o=p["o"])
    b = dict(do=p["o"], q=p["q"], k=p["k"], v=p["v"], dq=p["gq"], dk=p["gk"], dv=p["gv"])
    if not torch.cuda.is_available():   # without a device the calls get to their launches and no further
        for call, args in ((la_fwd, f), (la_bwd, b)):
            assert call(s, **args) != EINVAL, lib.impala_last_error()
    for name, other in (("o", "v"), ("o", "q")):
        for off in (2, -2):
            assert la_fwd(s, **{**f, name: p[other] + off}) == EINVAL
            assert b"overlap" in lib.impala_last_error()
    for name, other in (("dq", "v"), ("dv", "k"), ("dv", "gk"), ("dk", "gv"), ("dk", "o"), ("dq", "gv")):
        for off in (0, 2):
            assert la_bwd(s, **{**b, name: p[other] + off}) == EINVAL, (name, other, off)
            assert b"overlap" in lib.impala_last_error()
