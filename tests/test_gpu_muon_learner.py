"""Learning phases with the Muon optimiser at hyperparameters of the workload's own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import gpu_util as G  # noqa: E402

P = pytest.importorskip("paper_2310_00036_amd")
from paper_2310_00036_amd import pipeline as PL  # noqa: E402
from synth import NetShape, Workload, draw_params  # noqa: E402

OWN = dict(optimizer="muon", muon_lr=0.01, muon_momentum=0.9, muon_weight_decay=0.1, muon_nesterov=0, muon_steps=4,
           muon_scale=1, muon_eps=1e-6)
CFG = dict(lr=0.01, momentum=0.9, weight_decay=0.1, nesterov=False, steps=4, scale=P.MUON_SCALE_RMS, eps=1e-6)


@pytest.mark.parametrize("prec", [G.BF16, G.FP32], ids=["bf16", "fp32"])
def test_a_workloads_hyperparameters_are_the_steps(prec):
    """One update of a learner is the layers' gradient and muon_step at the workload's hyperparameters, bit for bit."""
    from tests.test_gpu_network import _c1_like_inputs, _gpu_rollout, _learner_gpu
    torch = G.torch()
    wl, params, ro, perm = _c1_like_inputs(wid=0)
    wl = wl.replace(epochs=1, num_minibatches=1, **OWN)
    got = _learner_gpu(wl, prec, params, ro, perm)
    d = _gpu_rollout(ro, wl)
    T, E, A, mb, net = wl.T, wl.E, wl.net.num_actions, wl.mb, wl.net
    adv = torch.empty((T, E), dtype=torch.float32, device="cuda:0")
    ret = torch.empty_like(adv)
    P.gae_advantages(T, E, d["rewards"], d["values"], d["dones"], d["next_value"], d["next_done"], wl.gamma, wl.lam, adv,
                     ret)
    p = G.dev_f32(params)
    m, v, grads = torch.zeros_like(p), torch.zeros_like(p), torch.empty_like(p)
    ws = G.ws_bytes(P.impala_workspace_bytes(net, mb, prec, 1))
    logits = torch.empty((mb, A), dtype=torch.float32, device="cuda:0")
    value = torch.empty(mb, dtype=torch.float32, device="cuda:0")
    dz, dv = torch.empty_like(logits), torch.empty_like(value)
    stats = torch.zeros((1, 8), dtype=torch.float32, device="cuda:0")
    rows = G.dev_i32(perm)[0].contiguous()
    rl = rows.long()
    P.impala_cnn_fwd(net, prec, p, d["obs"], rows, mb, ws, 1, logits, value)
    P.ppo_loss_grad(mb, A, logits, value, d["actions"][rl].contiguous(), d["logp"][rl].contiguous(),
                    adv.view(-1)[rl].contiguous(), ret.view(-1)[rl].contiguous(), 1, wl.clip_eps, wl.vf_coef, wl.ent_coef,
                    dz, dv, stats[0])
    P.impala_cnn_bwd(net, prec, p, d["obs"], rows, mb, ws, dz, dv, grads)
    mats = P.muon_net_matrices(net)
    cfg = P.muon_cfg(adam_lr=wl.lr, beta1=wl.beta1, beta2=wl.beta2, adam_eps=wl.adam_eps, max_grad_norm=wl.max_grad_norm,
                     **CFG)
    P.muon_step(p.numel(), mats, cfg, p, grads, m, v, 1, stats[0, 6:], G.ws_bytes(P.muon_workspace_bytes(p.numel(), mats, cfg)))
    G.sync()
    assert torch.equal(got[0], p) and torch.equal(got[1], m) and torch.equal(got[2], v) and torch.equal(got[4], stats)
    default = _learner_gpu(wl.replace(muon_lr=0.02), prec, params, ro, perm)
    assert not torch.equal(default[0], got[0]) and torch.equal(default[1], got[1])


def test_pipeline_trains_at_the_workloads_hyperparameters():
    """The actor-learner pipeline on two streams equals its one-thread replay, and not the one at other settings."""
    torch = G.torch()
    wl = Workload("pipe_muon", "ppo", T=8, E=4, net=NetShape(num_actions=6), epochs=2, num_minibatches=2, seed=3, **OWN)

    def agent(w):
        return PL.LibraryAgent(w, P.PREC_BF16, draw_params(w.net, w.seed))

    p_ref, ref = PL.run_sequential(agent(wl), wl, 4, seed=9)
    p, rec = PL.run_pipeline(agent(wl), wl, 4, seed=9, learner_delay=lambda k: 0.02)
    assert rec.rollouts == ref.rollouts and torch.equal(p, p_ref) and np.isfinite(np.concatenate(rec.stats)).all()
    other = wl.replace(muon_lr=0.02)
    assert not torch.equal(PL.run_sequential(agent(other), other, 4, seed=9)[0], p_ref)


@pytest.mark.parametrize("kw", [dict(optimizer="muon"), OWN], ids=["defaults", "own"])
def test_learner_step_against_the_oracle(kw):
    """One float32 update on certified frames. The momentum against the oracle's at its gradient's tolerance; the
    parameters against the oracle's update from the learner's own gradient (an orthogonalisation turns a gradient's
    rounding into up to 485 times as much where singular values are small, and a few frames' gradient has many of
    those). Per matrix the update is off by the iteration's 2^-14 and the parameters' rounding."""
    from oracle import learner as olearner, optim
    from tests.test_gpu_network import FP32_TOL, _certified_rollout, _learner_gpu, _oracle_learner
    wl = Workload("muon_certified", "ppo", T=2, E=1, net=NetShape(num_actions=6), max_grad_norm=0.0).replace(**kw)
    params = draw_params(wl.net, 5)
    wl, raw, ro = _certified_rollout(wl, params)
    want, _ = _oracle_learner(wl, params, ro, raw["perm"], G.FP32)
    got = _learner_gpu(wl, G.FP32, params, ro, raw["perm"])
    p, m, v = (G.host(t) for t in got[:3])
    assert G.rel_l2(m, want[1]) <= FP32_TOL and G.rel_l2(v, want[2]) <= 2 * FP32_TOL
    f32 = lambda a: np.float64(np.float32(a))  # noqa: E731
    mats = olearner.weight_matrices(wl.net)
    g = m / (1 - f32(wl.beta1))
    for off, r, c in mats:
        g[off:off + r * c] = m[off:off + r * c] / (1 - f32(wl.muon_momentum))
    p0 = params.astype(np.float64)
    zero = np.zeros_like(p0)
    pw, _, _ = optim.muon(p0, g, zero, zero, 1, mats, f32(wl.muon_lr), f32(wl.muon_momentum), f32(wl.muon_weight_decay),
                          bool(wl.muon_nesterov), wl.muon_steps, wl.muon_scale, f32(wl.muon_eps), f32(wl.lr), f32(wl.beta1),
                          f32(wl.beta2), f32(wl.adam_eps))
    for off, r, c in mats:
        at = slice(off, off + r * c)
        bound = 2.0 ** -14 * np.linalg.norm(pw[at] - p0[at] * (1 - f32(wl.muon_lr) * f32(wl.muon_weight_decay))) \
            + 2.0 ** -22 * np.linalg.norm(p0[at])
        err = np.linalg.norm(p[at] - pw[at])
        print((r, c), "error %.2e of a bound of %.2e" % (err, bound))
        assert err <= bound, (off, r, c, err, bound)
    rest = np.ones(p0.size, bool)
    for off, r, c in mats:
        rest[off:off + r * c] = False
    assert G.rel_l2((p - p0)[rest], (pw - p0)[rest]) <= 1e-4
