"""Linear attention on arrays that lie in larger ones: the bits of contiguous arrays, and nothing written beside the outputs."""
import pytest
import torch

from tests.test_gpu_linattn import DEV, TYPES, backward, dev, forward, make, workspace

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu


def same_bits(x, part, scale, want, grads):
    """Forward and backward on the given views, against results of contiguous arrays."""
    for n in ("q", "k", "v", "do"):
        part[n].copy_(dev(x[n]))
    a, d, s0, ds = dev(x["a"]), dev(x["d"]), dev(x["s0"]), dev(x["ds"])
    s_out, ds0 = torch.empty_like(s0), torch.empty_like(s0)
    q, k, v, do, o, dq, dk, dv = (part[n] for n in ("q", "k", "v", "do", "o", "dq", "dk", "dv"))
    shape = P.linattn_shape(q, k, v, o, d, scale)
    P.impala_linattn_fwd(shape, q, k, v, a, d, s0, o, s_out, workspace(shape))
    assert torch.equal(o, want[0]) and torch.equal(s_out, want[1])
    shape = P.linattn_shape(q, k, v, do, d, scale, dq, dk, dv)
    P.impala_linattn_bwd(shape, do, q, k, v, a, d, s0, ds, dq, dk, dv, ds0, workspace(shape, 1))
    assert all(torch.equal(g, w) for g, w in zip((dq, dk, dv, ds0), grads))
    for n in ("q", "k", "v", "do"):
        assert torch.equal(part[n], dev(x[n])), n


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,H,dk,dv", [(70, 3, 2, 32, 64), (9, 2, 3, 7, 20), (130, 2, 2, 64, 24), (2, 5, 1, 128, 96)])
def test_one_buffer_of_parts_with_other_widths(T, E, H, dk, dv, ty):
    """Everything with an element a row side by side in [T, E, row], and env-major."""
    x = make(T, E, H, dk, dv, ty, "few", seed=T)
    want, grads = forward(x, 0.5), backward(x, 0.5)
    names = (("q", dk), ("dq", dk), ("v", dv), ("dk", dk), ("dv", dv), ("k", dk), ("o", dv), ("do", dv))
    row = sum(H * w for _, w in names)
    for major in (False, True):
        buf = torch.full((E, T, row + 3) if major else (T, E, row + 3), 7.0, dtype=TYPES[ty], device=DEV)
        view = buf.transpose(0, 1) if major else buf
        part, at = {}, 0
        for n, w in names:
            part[n] = view[..., at:at + H * w].unflatten(-1, (H, w))
            at += H * w
        same_bits(x, part, 0.5, want, grads)
        assert (buf[..., row:] == 7).all()
