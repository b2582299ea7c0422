"""Every launch of the memory core's operators is in an open profile."""
import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def keys(call):
    P.impala_profile_begin()
    try:
        call()
    finally:
        table = P.impala_profile_end()
    return {k.split("/")[0]: n for k, _, n in table}


def test_launches_are_recorded():
    n, c = 50, 64
    r, v = torch.randn(n, c, device=DEV), torch.ones(c, device=DEV)
    s = P.blocknorm_shape(P.PREC_FP32, n, c, norm2=P.NORM_LAYER)
    ws = torch.empty(P.impala_blocknorm_bwd_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    out, dh, dg = torch.empty_like(r), torch.empty_like(r), torch.empty_like(v)
    assert keys(lambda: P.impala_blocknorm_fwd(s, r, v, None, None, None, None, out)) == {"blocknorm_fwd": 1}
    bwd = lambda dg: P.impala_blocknorm_bwd(s, r, None, r, v, None, None, None, None, None, dh, dg, None, None, None, None,  # noqa: E731
                                            None, None, ws)
    assert keys(lambda: bwd(dg)) == {"blocknorm_bwd": 1, "blocknorm_params": 1}

    T, E, H, d = 5, 2, 3, 16
    q, a = torch.randn(T, E, H, d, device=DEV), torch.zeros(H, device=DEV)
    st, st2 = torch.randn(E, H, d, d, device=DEV), torch.empty(E, H, d, d, device=DEV)
    for t in (0, 1, T):
        x, o = q[:t], torch.empty_like(q[:t])
        f = P.linattn_shape(x, x, x, o)
        want = {"linattn_state": 1} if t == 0 else {"linattn": 1}
        assert keys(lambda: P.impala_linattn_fwd(f, x, x, x, a, None, st, o, st2)) == want, t
        b = P.linattn_shape(x, x, x, o, None, 1.0, x, x, x)
        g = [torch.empty_like(x) for _ in range(3)]
        assert keys(lambda: P.impala_linattn_bwd(b, o, x, x, x, a, None, st, st, *g, st2)) == want, t
    tensors = P.grad_tensors([(r, r)])
    assert keys(lambda: P.grad_clip(tensors, 1.0, None, torch.empty(P.grad_clip_workspace_bytes(tensors), dtype=torch.uint8,
                                                                    device=DEV))) == {"grad_clip": 1}
