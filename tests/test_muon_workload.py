"""The Muon optimiser's hyperparameters of a workload reach the learner's configuration."""
import pytest

from synth import WORKLOADS, Workload

P = pytest.importorskip("paper_2310_00036_amd")

VALUES = dict(muon_lr=0.0625, muon_momentum=0.875, muon_weight_decay=0.25, muon_eps=0.5, muon_nesterov=0, muon_steps=3,
              muon_scale=P.MUON_SCALE_RMS)


def test_every_hyperparameter_of_a_workload_is_the_learners():
    wl = WORKLOADS[0].replace(optimizer="muon", **VALUES)
    cfg = P.learner_cfg(wl, P.PREC_BF16)
    assert cfg.optimizer == P.LEARNER_OPT_MUON
    assert {k: getattr(cfg, k) for k in VALUES} == VALUES
    assert P.learner_workspace_bytes(wl.net, cfg) > 0
    # ... and of one that names none of them, the defaults of muon_cfg
    base, m = P.learner_cfg(Workload("w", "ppo", T=8, E=4, optimizer="muon"), P.PREC_BF16), P.muon_cfg(lr=0.02)
    for k in VALUES:
        assert getattr(base, k) == getattr(m, k[len("muon_"):]), k


def test_a_bad_hyperparameter_is_refused():
    for bad in (dict(muon_steps=0), dict(muon_momentum=1.0), dict(muon_lr=-1.0), dict(muon_scale=2), dict(muon_nesterov=2)):
        wl = WORKLOADS[0].replace(optimizer="muon", **bad)
        assert P.learner_workspace_bytes(wl.net, P.learner_cfg(wl, P.PREC_BF16)) == 0, bad
