"""The memory core's operators together, as a policy uses them: a block of norms, projections, linear attention with a gate,
trained over a rollout with episode starts, clipped and stepped, and run step by step by the actor."""
import math

import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, E, H, D, C = 70, 3, 2, 24, 48
SCALE = D ** -0.5
NAMES = ("wq", "wk", "wv", "wg", "wo", "gamma0", "gamma1", "gamma2", "gamma3", "rscale")
# Twelve stages, each off by at most 2 sqrt(terms) 2^-24 of its terms' magnitude (up to 300 terms), which is some ten times
# what is left of them: 12 * 2 * 17.4 * 6e-8 * 10 = 2.5e-4 at worst, were all of them to add up.
TOL = 2.5e-4


def params(g, dtype=torch.float32):
    p = {n: torch.randn(C, H * D, generator=g) * C ** -0.5 for n in ("wq", "wk", "wv", "wg")}
    p["wo"] = torch.randn(H * D, C, generator=g) * (H * D) ** -0.5
    p.update(gamma0=1 + 0.2 * torch.randn(C, generator=g), gamma1=1 + 0.2 * torch.randn(H * D, generator=g),
             gamma2=1 + 0.2 * torch.randn(C, generator=g), gamma3=1 + 0.2 * torch.randn(C, generator=g),
             rscale=0.5 + 0.1 * torch.randn(C, generator=g))
    return {n: t.to(dtype) for n, t in p.items()}


def rms(x, gamma):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gamma


def plain(x, p, a, dones, s):
    """(out, its next norm, the state) in 64 bits, for autograd."""
    h = rms(x, p["gamma0"])
    q, k, v, gate = ((h @ p[w]).reshape(*x.shape[:2], H, D) for w in ("wq", "wk", "wv", "wg"))
    keep = torch.exp(a)[None, :, None, None]
    os = []
    for t in range(x.shape[0]):
        s = torch.where(dones[t].bool()[:, None, None, None], torch.zeros_like(s), keep * s)
        s = s + k[t][..., :, None] * v[t][..., None, :]
        os.append(SCALE * (q[t][..., :, None] * s).sum(-2))
    o = torch.stack(os)
    var, mean = torch.var_mean(o, -1, unbiased=False, keepdim=True)
    u = (o - mean) / torch.sqrt(var + 1e-5) * p["gamma1"].reshape(H, D) * (gate * torch.sigmoid(gate))
    y = u.reshape(*x.shape[:2], H * D) @ p["wo"]
    out = x + p["rscale"] * rms(y, p["gamma2"])
    return out, rms(out, p["gamma3"]), s


class Core:
    """The same in float32 through the library's calls; the projections' products are torch's."""

    def __init__(self, p, a):
        self.p, self.a = p, a

    def forward(self, x, dones, s0, step=False):
        p, n = self.p, x.shape[0] * x.shape[1]
        k = self.kept = dict(x=x, dones=dones, s0=s0, h=torch.empty_like(x))
        P.impala_blocknorm_fwd(self.pre(n), x, p["gamma0"], None, None, None, None, k["h"])
        for w in ("q", "k", "v", "g"):
            k[w] = (k["h"] @ p["w" + w]).reshape(*x.shape[:2], H, D)
        k["o"], k["s"] = torch.empty_like(k["v"]), torch.empty_like(s0)
        shape = P.linattn_shape(k["q"], k["k"], k["v"], k["o"], dones, SCALE)
        args = (shape, k["q"], k["k"], k["v"], self.a, dones, s0, k["o"], k["s"])
        P.impala_linattn_step(*args) if step else P.impala_linattn_fwd(*args, self.ws(shape))
        k["u"] = torch.empty_like(k["o"])
        P.impala_blocknorm_fwd(self.heads(n), k["o"], p["gamma1"], None, k["g"], None, None, k["u"])
        k["y"] = k["u"].reshape(*x.shape[:2], H * D) @ p["wo"]
        k["out"], k["next"] = torch.empty_like(x), torch.empty_like(x)
        P.impala_blocknorm_fwd(self.post(n), k["y"], p["gamma2"], None, None, p["rscale"], x, k["out"], p["gamma3"], None,
                               k["next"])
        return k["out"], k["next"], k["s"]

    def backward(self, dout, dnext, ds):
        p, k = self.p, self.kept
        n = dout.shape[0] * dout.shape[1]
        g = {name: torch.empty_like(t) for name, t in p.items()}
        dy, dx = torch.empty_like(k["y"]), torch.empty_like(k["x"])
        post = self.post(n)
        P.impala_blocknorm_bwd(post, dout, dnext, k["y"], p["gamma2"], None, None, p["rscale"], k["out"], p["gamma3"], dy,
                               g["gamma2"], None, None, g["rscale"], dx, g["gamma3"], None, self.bws(post))
        flat = lambda t: t.reshape(n, -1)   # noqa: E731
        g["wo"] = flat(k["u"]).t() @ flat(dy)
        du = (dy @ p["wo"].t()).reshape(k["u"].shape)
        do, dg = torch.empty_like(k["o"]), torch.empty_like(k["g"])
        heads = self.heads(n)
        P.impala_blocknorm_bwd(heads, du, None, k["o"], p["gamma1"], None, k["g"], None, None, None, do, g["gamma1"], None, dg,
                               None, None, None, None, self.bws(heads))
        d = {w: torch.empty_like(k[w]) for w in "qkv"}
        ds0 = torch.empty_like(k["s0"])
        shape = P.linattn_shape(k["q"], k["k"], k["v"], do, k["dones"], SCALE, d["q"], d["k"], d["v"])
        P.impala_linattn_bwd(shape, do, k["q"], k["k"], k["v"], self.a, k["dones"], k["s0"], ds, d["q"], d["k"], d["v"], ds0,
                             self.ws(shape, 1))
        d["g"] = dg
        dh = sum(flat(d[w]) @ p["w" + w].t() for w in "qkvg")
        for w in "qkvg":
            g["w" + w] = flat(k["h"]).t() @ flat(d[w])
        pre, back = self.pre(n), torch.empty_like(dx)
        P.impala_blocknorm_bwd(pre, dh, None, k["x"], p["gamma0"], None, None, None, None, None, back, g["gamma0"], None, None,
                               None, None, None, None, self.bws(pre))
        return g, dx + back, ds0

    @staticmethod
    def pre(n):
        return P.blocknorm_shape(P.PREC_FP32, n, C, norm=P.NORM_RMS)

    @staticmethod
    def heads(n):
        return P.blocknorm_shape(P.PREC_FP32, n, H * D, groups=H, norm=P.NORM_LAYER, gate_act=P.GATE_SILU)

    @staticmethod
    def post(n):
        return P.blocknorm_shape(P.PREC_FP32, n, C, norm=P.NORM_RMS, norm2=P.NORM_RMS)

    @staticmethod
    def ws(shape, backward=0):
        return torch.empty(max(1, P.impala_linattn_workspace_bytes(shape, backward)), dtype=torch.uint8, device=DEV)

    @staticmethod
    def bws(shape):
        return torch.empty(P.impala_blocknorm_bwd_workspace_bytes(shape), dtype=torch.uint8, device=DEV)


def close(name, got, want):
    got, want = got.detach().double().cpu(), want.detach()
    assert float((got - want).norm()) <= TOL * float(want.norm()), (name, float((got - want).norm() / want.norm()))


def test_a_block_is_trained_clipped_and_stepped():
    g = torch.Generator().manual_seed(1)
    p = params(g)
    a = torch.log1p(-torch.tensor([0.25, 0.01]))
    x, dout, dnext = (torch.randn(T, E, C, generator=g) for _ in range(3))
    s0, ds = torch.randn(E, H, D, D, generator=g), torch.randn(E, H, D, D, generator=g)
    dones = (torch.rand(T, E, generator=g) < 0.05).to(torch.uint8)

    ref = {n: t.double().requires_grad_() for n, t in p.items()}
    xd, sd = x.double().requires_grad_(), s0.double().requires_grad_()
    want = plain(xd, ref, a.double(), dones, sd)
    loss = (want[0] * dout).sum() + (want[1] * dnext).sum() + (want[2] * ds).sum()
    grads = torch.autograd.grad(loss, [xd, sd] + [ref[n] for n in NAMES])

    dev = {n: t.to(DEV) for n, t in p.items()}
    core = Core(dev, a.to(DEV))
    got = core.forward(x.to(DEV), dones.to(DEV), s0.to(DEV))
    for name, o, w in zip(("out", "next", "state"), got, want):
        close(name, o, w)
    pg, dx, ds0 = core.backward(dout.to(DEV), dnext.to(DEV), ds.to(DEV))
    close("dx", dx, grads[0])
    close("ds0", ds0, grads[1])
    for n, w in zip(NAMES, grads[2:]):
        close(n, pg[n], w)

    # the clip over all parameters' gradients into one buffer, and one Adam step on theirs
    sizes = [p[n].numel() for n in NAMES]
    flat, step_p = torch.empty(sum(sizes), device=DEV), torch.cat([dev[n].reshape(-1) for n in NAMES])
    t = P.grad_tensors([(pg[n].reshape(-1), d) for n, d in zip(NAMES, flat.split(sizes))])
    stats = torch.empty(2, device=DEV)
    P.grad_clip(t, 0.5, stats, torch.empty(P.grad_clip_workspace_bytes(t), dtype=torch.uint8, device=DEV))
    norm = math.sqrt(sum(float(w.square().sum()) for w in grads[2:]))
    assert norm > 0.5 and abs(float(stats[0]) / norm - 1) <= TOL and float(stats[1]) == 0
    wflat = torch.cat([w.reshape(-1) for w in grads[2:]]) * (0.5 / norm)
    close("clipped", flat, wflat)
    m, v = torch.zeros_like(flat), torch.zeros_like(flat)
    P.adam_step(flat.numel(), step_p, flat, m, v, 1, 1e-3, 0.9, 0.999, 1e-5, 0.0, None,
                torch.empty(P.adam_workspace_bytes(flat.numel()), dtype=torch.uint8, device=DEV))
    close("m", m, 0.1 * wflat)


def test_the_actor_steps_through_what_the_learner_sees():
    g = torch.Generator().manual_seed(2)
    dev = {n: t.to(DEV) for n, t in params(g).items()}
    core = Core(dev, torch.log1p(-torch.tensor([0.25, 0.01])).to(DEV))
    x = torch.randn(T, E, C, generator=g).to(DEV)
    dones = (torch.rand(T, E, generator=g) < 0.05).to(torch.uint8).to(DEV)
    state = torch.randn(E, H, D, D, generator=g).to(DEV)
    out, nxt, last = core.forward(x, dones, state)
    outs, nexts = [], []
    for t in range(T):
        o, y, state = core.forward(x[t:t + 1], dones[t:t + 1], state, step=True)
        outs.append(o)
        nexts.append(y)
    close("out", torch.cat(outs), out.double().cpu())
    close("next", torch.cat(nexts), nxt.double().cpu())
    close("state", state, last.double().cpu())
