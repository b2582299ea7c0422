"""The oracle's Muon update against singular value decompositions, and its place in the learner."""
import numpy as np
import pytest

from oracle import learner, optim
from synth import NetShape, Workload, draw_params, draw_rollout


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6), (1, 7), (7, 1)])
def test_orthogonalize_maps_the_singular_values(shape):
    """u s v^T becomes u f(s / ||s||) v^T with f the polynomial s (a + b s^2 + c s^4) five times over."""
    x = np.random.default_rng(1).standard_normal(shape)
    u, s, vt = np.linalg.svd(x, full_matrices=False)
    f = s / np.sqrt((s * s).sum())
    a, b, c = optim.QUINTIC
    for _ in range(5):
        f = f * (a + b * f ** 2 + c * f ** 4)
    np.testing.assert_allclose(optim.orthogonalize(x), (u * f) @ vt, rtol=0, atol=1e-13)
    # below eps the division is by eps: one step from tiny singular values is a times them
    tiny = 1e-9 * x
    np.testing.assert_allclose(optim.orthogonalize(tiny, 1, 1.0), a * tiny, rtol=1e-12)


def test_muon_on_matrices_and_on_the_rest():
    rng = np.random.default_rng(2)
    p, g, m, v = (rng.standard_normal(40) for _ in range(4))
    v = v * v
    kw = dict(adam_lr=0.25, beta1=0.5, beta2=0.75, adam_eps=0.125)
    p1, m1, v1 = optim.muon(p, g, m, v, 3, [(4, 3, 8)], 0.5, 0.75, 0.125, True, 5, 0, **kw)
    pa, ma, va = optim.adam(p, g, m, v, 3, 0.25, 0.5, 0.75, 0.125)
    at = np.r_[4:28]
    rest = np.r_[0:4, 28:40]
    assert np.array_equal(p1[rest], pa[rest]) and np.array_equal(m1[rest], ma[rest]) and np.array_equal(v1[rest], va[rest])
    assert np.array_equal(v1[at], v[at])
    np.testing.assert_allclose(m1[at], 0.75 * m[at] + 0.25 * g[at], rtol=1e-15)
    u = 0.75 * m1[at] + 0.25 * g[at]
    want = p[at] * (1 - 0.0625) - 0.5 * np.sqrt(8 / 3) * optim.orthogonalize(u.reshape(3, 8)).ravel()
    np.testing.assert_allclose(p1[at], want, rtol=1e-14)
    # without Nesterov's look ahead the momentum itself; the other scale
    p2, _, _ = optim.muon(p, g, m, v, 3, [(4, 3, 8)], 0.5, 0.75, 0.0, False, 5, 1, **kw)
    want = p[at] - 0.5 * 0.2 * np.sqrt(8) * optim.orthogonalize(m1[at].reshape(3, 8)).ravel()
    np.testing.assert_allclose(p2[at], want, rtol=1e-13)


def test_the_learner_runs_the_workloads_optimiser():
    wl = Workload("o", "ppo", T=2, E=2, net=NetShape(in_h=12, in_w=12, ch=(4, 4, 8), hidden=8, num_actions=3))
    params = draw_params(wl.net, 0)
    raw = draw_rollout(wl)
    ro = learner.behaviour_rollout(wl, params, raw)
    zero = np.zeros_like(params, dtype=np.float64)

    def step(**kw):
        return learner.ppo_learner_step(wl.net, wl.replace(**kw), ro, params, zero, zero, 0, raw["perm"])

    adam, muon = step(), step(optimizer="muon", muon_momentum=0.9)
    covered = np.zeros(params.size, bool)
    for off, r, c in learner.weight_matrices(wl.net):
        covered[off:off + r * c] = True
        u = (muon[0] - params)[off:off + r * c].reshape(r, c) / (-0.02 * np.sqrt(max(1.0, c / r)))
        np.testing.assert_allclose(u, optim.orthogonalize(adam[1][off:off + r * c].reshape(r, c)), rtol=0, atol=1e-9)
    assert 0 < covered.sum() < params.size
    assert np.array_equal(adam[0][~covered], muon[0][~covered])
    np.testing.assert_allclose(muon[1], adam[1], rtol=1e-12)   # 1 - momentum = 1 - beta1 here
    assert not np.allclose(adam[0][covered], muon[0][covered])
    with pytest.raises(ValueError):
        step(optimizer="sgd")
