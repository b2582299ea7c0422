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


# Steps of a rollout's rows in bytes: buffer resources reach 2^25, rows further apart go by their addresses.
STEPS = [2 ** 24 - 8, 2 ** 24, 2 ** 25, 2 ** 25 + 4, 2 ** 25 + 2]


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("T,dk,dv", [(65, 32, 128), (130, 64, 64), (3, 128, 31)])
def test_steps_far_apart(T, dk, dv, ty):
    E, H, es = 2, 2, 2 if ty == "bf16" else 4
    x = make(T, E, H, dk, dv, ty, "few", seed=T)
    want, grads = forward(x, 0.5), backward(x, 0.5)
    flat = torch.empty((T - 1) * (STEPS[-2] // es) + 8192, dtype=TYPES[ty], device=DEV)
    for step in STEPS:
        if step % es:
            continue
        part = {}
        for i, (n, d) in enumerate((("q", dk), ("k", dk), ("v", dv), ("do", dv), ("o", dv), ("dq", dk), ("dk", dk), ("dv", dv))):
            part[n] = flat.as_strided((T, E, H, d), (step // es, H * d, d, 1), 1024 * i)
        same_bits(x, part, 0.5, want, grads)


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 5, 33, 71, 127])
def test_rows_at_any_address(d, ty):
    """Odd widths side by side, each row at its own alignment; what lies between stays."""
    T, E, H = 70, 2, 3
    x = make(T, E, H, d, d, ty, "few", seed=d)
    want, grads = forward(x, 0.5), backward(x, 0.5)
    row = 8 * H * (d + 1) + 1
    buf = torch.full((T, E, row), 7.0, dtype=TYPES[ty], device=DEV)
    part = {n: buf[..., i * H * (d + 1):(i + 1) * H * (d + 1)].unflatten(-1, (H, d + 1))[..., :d]
            for i, n in enumerate(("q", "dq", "k", "dk", "v", "dv", "do", "o"))}
    same_bits(x, part, 0.5, want, grads)
    gaps = buf[..., :-1].unflatten(-1, (8 * H, d + 1))[..., d]
    assert (gaps == 7).all() and (buf[..., -1] == 7).all()


@pytest.mark.parametrize("ty", ["bf16", "f32"])
def test_the_step_stride_of_one_step_is_not_used(ty):
    """Axes of one element have no stride: whatever it says, also where its bytes would come round in 64 bits."""
    x = make(1, 3, 2, 16, 8, ty, "few")
    want, grads = forward(x, 0.5), backward(x, 0.5)
    q, k, v, do, a, d, s0, ds = (dev(x[n]) for n in ("q", "k", "v", "do", "a", "d", "s0", "ds"))
    for step in (0, -1, 1 << 62, (1 << 62) + 16, -(1 << 63)):
        o, dq, dk, dv = (torch.empty_like(t) for t in (v, q, k, v))
        s_out, ds0 = torch.empty_like(s0), torch.empty_like(s0)
        shape = P.linattn_shape(q, k, v, o, d, 0.5, dq, dk, dv)
        for n in ("q", "k", "v", "o", "gq", "gk", "gv"):
            getattr(shape, n).t = step
        shape.done_t = step
        P.impala_linattn_fwd(shape, q, k, v, a, d, s0, o, s_out)
        P.impala_linattn_bwd(shape, do, q, k, v, a, d, s0, ds, dq, dk, dv, ds0)
        assert torch.equal(o, want[0]) and torch.equal(s_out, want[1]), step
        assert all(torch.equal(g, w) for g, w in zip((dq, dk, dv, ds0), grads)), step
