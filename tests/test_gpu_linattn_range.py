"""Linear attention at the ends of the numbers' range: states that grow until they overflow, infinite states."""
import pytest
import torch

from tests import memory_ref as ref
from tests.test_gpu_linattn import backward, check_forward, forward, magnitudes, make

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
BIG = 3.4028235e38


def compare(name, got, want, mag, terms, bf16):
    """Close where all that is summed is well inside the range, not finite where the result is well outside it."""
    inside, outside = mag < BIG / 64, want.abs() > BIG * 2
    got = got.cpu()
    rel = terms * 2.0 ** -24
    tol = rel * mag + (2.0 ** -8 * (want.abs() + rel * mag) if bf16 else 0)
    assert ((got.double() - want).abs() <= tol + 1e-37)[inside].all(), name
    assert not torch.isfinite(got[outside]).any(), name
    return int(inside.sum()), int(outside.sum())


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("log_decay", [0.02, 0.5, 1.38])
@pytest.mark.parametrize("T", [40, 64, 200, 900])
def test_states_that_grow(T, log_decay, ty):
    """A head that grows beside one that does not, with episodes that end in time and one that does not."""
    E, H, d = 3, 2, 24
    x = make(T, E, H, d, d, ty, "none", seed=T)
    x["a"] = torch.tensor([log_decay, -0.1])
    x["d"][::min(30, int(20 / log_decay)), 0] = 1   # env 0: short episodes, always finite
    x["d"][T // 2, 1] = 1
    terms = T + d + 16
    o, s = ref.linattn(x["q"], x["k"], x["v"], x["a"], x["d"], x["s0"], 0.3)
    om, sm = ref.linattn(*magnitudes(x, "q", "k", "v"), x["a"], x["d"], x["s0"].abs(), 0.3)
    got = forward(x, 0.3)
    n = [compare("o", got[0], o, om, terms, ty == "bf16"), compare("s_out", got[1], s, sm, terms, False)]
    args = ("do", "q", "k", "v")
    want = ref.linattn_grads(*(x[k] for k in args), x["a"], x["d"], x["s0"], x["ds"], 0.3)
    mag = ref.linattn_grads(*magnitudes(x, *args), x["a"], x["d"], x["s0"].abs(), x["ds"].abs(), 0.3)
    for name, g, w, m in zip(("dq", "dk", "dv", "ds0"), backward(x, 0.3), want, mag):
        n.append(compare(name, g, w, m, terms, ty == "bf16" and name != "ds0"))
    assert all(a > 0 for a, _ in n)
    if T * log_decay > 200:
        assert n[0][1] > 0
    kept = x["a"] < 0   # the other head is as it is alone
    y = {k: (v[:, :, kept] if k in ("q", "k", "v", "do") else v[:, kept] if k in ("s0", "ds") else v) for k, v in x.items()}
    y["a"] = x["a"][kept]
    check_forward(y, ty, 0.3, (got[0][:, :, kept], got[1][:, kept]))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 64, 100, 900])
def test_an_infinite_state(T, ty):
    """One number of s0 and of ds_out is infinite in env 0: it stays so, its column's outputs (and its row's and column's
    gradients) are not finite up to the episode's end, and nothing else differs."""
    E, H, d = 2, 2, 20
    x = make(T, E, H, d, d, ty, "none", seed=T)
    end = T // 2
    if end:
        x["d"][end, 0] = 1
    clean, clean_g = forward(x, 0.5), backward(x, 0.5)
    x["s0"][0, 1, 7, 4] = float("inf")
    x["ds"][0, 0, 3, 9] = -float("inf")
    o, s = (t.cpu() for t in forward(x, 0.5))
    hi = end if end else T
    hit = torch.zeros(T, E, H, d, dtype=torch.bool)
    hit[:hi, 0, 1, 4] = True
    assert not torch.isfinite(o[hit]).any() and torch.equal(o[~hit], clean[0].cpu()[~hit])
    at = torch.zeros(E, H, d, d, dtype=torch.bool)
    at[0, 1, 7, 4] = not end
    assert torch.isposinf(s[at]).all() and torch.equal(s[~at], clean[1].cpu()[~at])
    dq, dk, dv, ds0 = (t.cpu() for t in backward(x, 0.5))
    hit.zero_()
    hit[:hi, 0, 1, 7] = True
    assert not torch.isfinite(dq[hit]).any() and torch.equal(dq[~hit], clean_g[0].cpu()[~hit])
    for g, w, i in ((dk, clean_g[1], 3), (dv, clean_g[2], 9)):
        hit.zero_()
        hit[end:, 0, 0, i] = True
        assert not torch.isfinite(g[hit]).any() and torch.equal(g[~hit], w.cpu()[~hit])
    at.zero_()
    at[0, 0, 3, 9] = not end
    assert torch.isneginf(ds0[at]).all() and torch.equal(ds0[~at], clean_g[3].cpu()[~at])
