"""Sizes that the group norm calls refuse, on the host, before any HIP call."""
import pytest

P = pytest.importorskip("paper_2310_00036_amd")

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3


def _fwd(prec, n, H, W, C_, x=1 << 20, y=1 << 50, ws=1, wsb=0):
    """No bytes of workspace: EWORKSPACE says that the sizes were accepted."""
    return P.lib.impala_groupnorm_fwd(prec, n, H, W, C_, 1, x, None, None, 1e-5, 0, y, None, None, ws, wsb, None)


def _bwd(prec, n, H, W, C_):
    return P.lib.impala_groupnorm_bwd(prec, n, H, W, C_, 1, 1 << 50, 1 << 20, None, None, 16, 16, 0, 1 << 50, None, None, 1,
                                      0, None)


@pytest.mark.parametrize("prec", [P.PREC_BF16, P.PREC_FP32])
def test_launches_of_2_to_the_32_threads_at_every_width(prec):
    """A frame of 4096 x 4096 pixels of 513 to 1024 channels is 2^21 chunks of 1024 threads, 2^31 in all: one is
    accepted, two are a launch of 2^32 threads. With 512 channels it is half of that."""
    for C_, most in ((1024, 1), (1000, 1), (513, 1), (512, 3), (64, 31)):
        for call, query in ((_fwd, P.impala_groupnorm_fwd_workspace_bytes), (_bwd, P.impala_groupnorm_bwd_workspace_bytes)):
            assert call(prec, most, 4096, 4096, C_) == EWORKSPACE and query(prec, most, 4096, 4096, C_, 1) > 0, C_
            for n in (most + 1, 64, 1 << 20):
                assert call(prec, n, 4096, 4096, C_) == EUNSUPPORTED and query(prec, n, 4096, 4096, C_, 1) == 0, (C_, n)
