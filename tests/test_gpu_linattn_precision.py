"""Linear attention in bf16 where a sum's terms cancel: outputs and gradients are sums of at least 24 bits, rounded once."""
import pytest
import torch

from tests import memory_ref as ref
from tests.test_gpu_linattn import backward, forward, magnitudes, make

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -14   # what is left of two cancelling terms, of their size: 2^-17 of the terms would be 1/8 of it


def close(x, scale, s0):
    """All outputs against 64 bits: roundings of 2^-24 of the magnitudes a term, and the bf16 output's own."""
    st = x["s0"] if s0 else None
    args = [x[n] for n in ("do", "q", "k", "v")]
    mags = magnitudes(x, "do", "q", "k", "v")
    T, _, _, dk = x["q"].shape
    terms = T + max(dk, x["v"].shape[3]) + 16
    o, s = ref.linattn(*args[1:], x["a"], x["d"], st, scale)
    om, sm = ref.linattn(*mags[1:], x["a"], x["d"], st.abs() if s0 else None, scale)
    got = forward(x, scale, s0=s0)
    ref.assert_close("o", got[0], o, om, terms, False, True)
    ref.assert_close("s_out", got[1], s, sm, terms, False)
    want = ref.linattn_grads(*args, x["a"], x["d"], st, x["ds"] if s0 else None, scale)
    mag = ref.linattn_grads(*mags, x["a"], x["d"], st.abs() if s0 else None, x["ds"].abs() if s0 else None, scale)
    for name, g, w, m in zip(("dq", "dk", "dv"), backward(x, scale, s0=s0, ds=s0), want, mag):
        ref.assert_close(name, g, w, m, terms, False, True)


@pytest.mark.parametrize("seed", range(4))
def test_steps_that_cancel(seed):
    """Every second step takes the one before back, but for a decay near one."""
    T, E, H, d = 8, 64, 2, 4
    x = make(T, E, H, d, d, "bf16", "none", seed=seed)
    for n in ("q", "k", "v", "do"):
        x[n][1::2] = x[n][::2]
    x["v"][1::2] *= -1     # o: k v^T and -k v^T
    x["do"][1::2] *= -1    # dk, dv: q do^T and -q do^T
    x["a"] = torch.full((H,), -NEAR)
    close(x, 0.5, False)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("T", [2, 6])
def test_state_whose_numbers_cancel(T, seed):
    """Neighbouring rows and columns of the states are nearly the same, those of q, v and d_o each other's negatives; the
    steps' own contributions are small."""
    E, H, d = 64, 2, 4
    x = make(T, E, H, d, d, "bf16", "none", seed=seed)
    for n in ("q", "k", "v", "do"):
        x[n][..., 1::2] = -x[n][..., ::2]
    for n in ("k", "do"):
        x[n] *= NEAR
    for n in ("s0", "ds"):
        s = x[n]
        x[n] = s[..., ::2, ::2].repeat_interleave(2, -1).repeat_interleave(2, -2) * (1 + NEAR * s)
    x["a"] = torch.full((H,), -0.1)
    close(x, 1.0, True)
