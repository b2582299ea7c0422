"""Group norm's forward without a workspace where a frame fits one workgroup."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import gpu_util as G  # noqa: E402

P = pytest.importorskip("paper_2310_00036_amd")


@pytest.mark.parametrize("prec,dims", [(G.BF16, (3, 42, 42, 16)), (G.FP32, (3, 42, 42, 16)), (G.BF16, (2, 42, 42, 32)),
                                       (G.BF16, (2, 64, 128, 8)), (G.FP32, (2, 8, 8, 32))],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else ("bf16" if v == G.BF16 else "fp32"))
def test_frames_of_one_workgroup_need_none(prec, dims):
    t = G.torch()
    n, H, W, C = dims
    size = n * H * W * C
    xs = G.q(np.random.default_rng(1).standard_normal(size), prec)
    dt = t.bfloat16 if prec == G.BF16 else t.float32
    x = G.dev_act(xs, prec).reshape(-1)
    outs = []
    for ws in (G.ws_bytes(max(P.impala_groupnorm_fwd_workspace_bytes(prec, n, H, W, C, 4), 16)), None):
        y = t.full((size,), 7.0, dtype=dt, device="cuda:0")
        P.impala_groupnorm_fwd(prec, n, H, W, C, 4, x, None, None, 1e-5, P.ACT_RELU, y, ws=ws)
        G.sync()
        outs.append(y)
    assert t.equal(outs[0], outs[1]) and not bool((outs[0] == 7.0).any())


def test_one_channel_columns_of_the_same_frame_do():
    """42 x 42 x 16 at an odd address goes one channel a thread, in chunks."""
    t = G.torch()
    n, H, W, C = 2, 42, 42, 16
    size = n * H * W * C
    x = t.randn(size + 1, device="cuda:0")
    y = t.empty(size + 1, device="cuda:0")
    with pytest.raises(P.LibraryError):
        P.impala_groupnorm_fwd(G.FP32, n, H, W, C, 4, x[1:], None, None, 1e-5, P.ACT_NONE, y[1:])
    with pytest.raises(P.LibraryError):
        P.impala_groupnorm_fwd(G.FP32, n, H, W, C, 4, x[:-1], None, None, 1e-5, P.ACT_NONE, y[1:])
    P.impala_groupnorm_fwd(G.FP32, n, H, W, C, 4, x[:-1], None, None, 1e-5, P.ACT_NONE, y[:-1])
    G.sync()
