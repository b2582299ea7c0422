"""Which arrays the memory core's calls take as each other: on the host, before any HIP call."""
import pytest

from tests.test_blocknorm_abi import B_ARGS, F_ARGS, MB
from tests.test_blocknorm_abi import bwd as bn_bwd
from tests.test_blocknorm_abi import fwd as bn_fwd
from tests.test_blocknorm_abi import lib
from tests.test_blocknorm_abi import shape as bn_shape

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
