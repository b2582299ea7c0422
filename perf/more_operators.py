"""The memory core's operators as cases to time and compare.

Kinds of case, each one call through the package's public entry points:

la_fwd   impala_linattn_fwd: linear attention with a decay per head over a rollout, episode starts clear its state
la_bwd   impala_linattn_bwd: its gradients for queries, keys, values and the state before the rollout
la_step  impala_linattn_step: one step of it for each env, from state to state (the actor's form)
bn_fwd   impala_blocknorm_fwd: a block's norm, gate, scale and residual sum, and the next block's norm of that sum
bn_bwd   impala_blocknorm_bwd: its gradients
clip     grad_clip: the global norm over many gradient tensors, and their clipped values in one flat buffer

With `own` false the operators are computed from elementary torch operations in 32 bits (64 for powers of the decay
and for sums over rows or tensors).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
CHUNK = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the rollout of the benchmark's workload (128 steps of 64 envs), a core of its net's hidden size, 256 = 4 x 64
        dict(name="la_fwd_rollout", kind="la_fwd", type="bf16", T=128, E=64, heads=4, dk=64, dv=64, done=0.01),
        # two long recordings: few chains, many steps, no episode's end
        dict(name="la_fwd_long", kind="la_fwd", type="bf16", T=16384, E=2, heads=8, dk=128, dv=128, done=0.0),
        # the learner's gradients over the widened workload's rollout, 512 = 8 x 64
        dict(name="la_bwd_rollout", kind="la_bwd", type="bf16", T=128, E=128, heads=8, dk=64, dv=64, done=0.01),
        # odd lengths and head sizes in float32, many short episodes
        dict(name="la_bwd_odd", kind="la_bwd", type="f32", T=1001, E=6, heads=5, dk=33, dv=71, done=0.1),
        # one actor call's 128 envs
        dict(name="la_step_actor", kind="la_step", type="bf16", E=128, heads=4, dk=64, dv=64, done=0.01),
        # as many envs as a server might step at once, wide heads
        dict(name="la_step_fleet", kind="la_step", type="bf16", E=4096, heads=8, dk=128, dv=128, done=0.01),
        # one actor call's rows between two blocks: launch and latency
        dict(name="bn_fwd_actor", kind="bn_fwd", type="bf16", n=128, C=256, groups=1, norm="rms", norm2="rms",
             gate="off", res=True, scaled=True, biased=False),
        # the core's output, normalised head by head and gated, for the widened workload's rollout
        dict(name="bn_fwd_heads", kind="bn_fwd", type="f32", n=16384, C=512, groups=8, norm="layer", norm2="off",
             gate="silu", res=False, scaled=False, biased=True),
        # a long rollout of a wide core with everything on
        dict(name="bn_bwd_wide", kind="bn_bwd", type="bf16", n=65536, C=1024, groups=1, norm="rms", norm2="rms",
             gate="silu", res=True, scaled=True, biased=False),
        # odd rows and channels, layer norms with shifts
        dict(name="bn_bwd_odd", kind="bn_bwd", type="f32", n=3001, C=1531, groups=1, norm="layer", norm2="layer",
             gate="sigmoid", res=True, scaled=True, biased=True),
        # the benchmark's net's 36 parameter gradients
        dict(name="clip_net", kind="clip", type="f32", net=True, layers=0, width=0, limit=0.5),
        # that net and the gradients of four wide blocks that were kept in bf16
        dict(name="clip_core", kind="clip", type="bf16", net=True, layers=4, width=2048, limit=0.5),
    ]


def draw(rng):
    """One more case: any kind, sizes over their whole range."""
    def log_int(lo, hi):
        return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))

    kind = rng.choice(("la_fwd", "la_fwd", "la_bwd", "la_bwd", "la_step", "bn_fwd", "bn_bwd", "clip"))
    ty = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("la_fwd", "la_bwd"):
        heads = log_int(1, 16)
        dk = rng.choice((16, 32, 64, 64, 128, log_int(4, 128)))
        dv = rng.choice((dk, dk, log_int(4, 128)))
        most = 2 ** (25 if kind == "la_fwd" else 23) // (heads * max(dk, dv))   # steps of all envs
        T = log_int(1, min(16384, most))
        return dict(kind=kind, type=ty, T=T, E=log_int(1, min(4096, most // T)), heads=heads, dk=dk, dv=dv,
                    done=rng.choice((0.0, 0.003, 0.01, 0.1)))
    if kind == "la_step":
        heads = log_int(1, 16)
        dk = rng.choice((16, 32, 64, 64, 128, log_int(4, 128)))
        dv = rng.choice((dk, dk, log_int(4, 128)))
        return dict(kind=kind, type=ty, E=log_int(1, min(4096, 2 ** 29 // (heads * dk * dv))), heads=heads, dk=dk, dv=dv,
                    done=rng.choice((0.0, 0.01, 0.1)))
    if kind in ("bn_fwd", "bn_bwd"):
        C = rng.choice((log_int(16, 4096), 2 ** rng.randint(5, 12)))
        groups = rng.choice([g for g in (1, 1, 1, 2, 4, 8) if C % (8 * g) == 0 or g == 1])
        norm = rng.choice(("layer", "rms", "off"))
        norm2 = rng.choice(("layer", "rms", "off")) if groups == 1 else "off"
        gate = rng.choice(("off", "linear", "silu", "sigmoid"))
        return dict(kind=kind, type=ty, n=log_int(1, min(65536, 2 ** 26 // C)), C=C, groups=groups, norm=norm, norm2=norm2,
                    gate=gate, res=rng.random() < 0.5, scaled=rng.random() < 0.5, biased=rng.random() < 0.5)
    return dict(kind=kind, type=ty, net=rng.random() < 0.5, layers=log_int(1, 40), width=log_int(16, 512),
                limit=rng.choice((0.5, 40.0)))


# ------------------------------------------------------------------------------- inputs


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _net_sizes():
    """Element counts of the 36 tensors of the standard net, (16, 32, 32) / 256 / 18 on 84 x 84 x 4 frames."""
    out, cin = [], 4
    for c in (16, 32, 32):
        for k in range(5):
            out += [9 * (cin if k == 0 else c) * c, c]
        cin = c
    return out + [11 * 11 * 32 * 256, 256, 256 * 18, 18, 256, 1]


def _clip_tensors(case):
    """[(elements, type)]: the net's in float32; a block's five projections, two feed-forward matrices and five
    vectors in the case's type."""
    out = [(n, torch.float32) for n in _net_sizes()] if case["net"] else []
    w = case["width"]
    for _ in range(case["layers"]):
        out += [(w * w, DTYPES[case["type"]])] * 5 + [(4 * w * w, DTYPES[case["type"]])] * 2
        out += [(w, DTYPES[case["type"]])] * 5
    return out


def _randn(g, dt, *shape):
    return torch.randn(shape, generator=g, device=DEV).to(dt)


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    st = dict(case=case)
    if kind.startswith("la"):
        T, E, H, dk, dv = case.get("T", 1), case["E"], case["heads"], case["dk"], case["dv"]
        dt = DTYPES[case["type"]]
        st["q"], st["k"] = _randn(g, dt, T, E, H, dk), _randn(g, dt, T, E, H, dk)
        st["v"] = _randn(g, dt, T, E, H, dv)
        st["scale"] = dk ** -0.5
        # decays of 1 - 1/2 to 1 - 1/256, spread evenly over the heads in the exponent
        st["log_decay"] = torch.log1p(-(2.0 ** -(1 + 7 * torch.arange(H, device=DEV, dtype=torch.float64) / max(1, H - 1)))).float()
        st["dones"] = (torch.rand(T, E, generator=g, device=DEV) < case["done"]).to(torch.uint8)
        st["s0"] = _randn(g, torch.float32, E, H, dk, dv)
        if kind == "la_bwd":
            st["do"] = _randn(g, dt, T, E, H, dv)
            st["ds_out"] = _randn(g, torch.float32, E, H, dk, dv)
            st["dq"], st["dk"], st["dv"] = (torch.empty_like(st[x]) for x in "qkv")
            st["ds0"] = torch.empty_like(st["s0"])
        else:
            st["o"], st["s_out"] = torch.empty_like(st["v"]), torch.empty_like(st["s0"])
    elif kind.startswith("bn"):
        n, C, dt = case["n"], case["C"], DTYPES[case["type"]]
        st["h"] = (0.3 + 1.5 * torch.randn(n, C, generator=g, device=DEV)).to(dt)
        st["gamma"] = 1 + 0.2 * _randn(g, torch.float32, C)
        st["gamma2"] = 1 + 0.2 * _randn(g, torch.float32, C) if case["norm2"] != "off" else None
        st["beta"] = 0.2 * _randn(g, torch.float32, C) if case["biased"] else None
        st["beta2"] = 0.2 * _randn(g, torch.float32, C) if case["biased"] and case["norm2"] != "off" else None
        st["rscale"] = 0.5 + 0.1 * _randn(g, torch.float32, C) if case["scaled"] else None
        st["gate"] = _randn(g, dt, n, C) if case["gate"] != "off" else None
        st["res"] = _randn(g, dt, n, C) if case["res"] else None
        two = case["norm2"] != "off"
        if kind == "bn_fwd":
            st["out"] = torch.empty_like(st["h"])
            st["out2"] = torch.empty_like(st["h"]) if two else None
        else:
            st["out"] = _randn(g, dt, n, C) if two else None
            st["dout"] = _randn(g, dt, n, C)
            st["dout2"] = _randn(g, dt, n, C) if two else None
            st["dh"] = torch.empty_like(st["h"])
            st["dgate"] = torch.empty_like(st["h"]) if st["gate"] is not None else None
            st["dres"] = torch.empty_like(st["h"]) if case["res"] and two else None
            for x in ("gamma", "beta", "rscale", "gamma2", "beta2"):
                st["d" + x] = torch.empty_like(st[x]) if st[x] is not None else None
    else:
        sizes = _clip_tensors(case)
        st["src"] = [(1e-3 * torch.randn(k, generator=g, device=DEV)).to(dt) for k, dt in sizes]
        st["flat"] = torch.empty(sum(k for k, _ in sizes), device=DEV)
        st["dst"] = list(st["flat"].split([k for k, _ in sizes]))
        st["stats"] = torch.empty(2, device=DEV)
    if own:   # the workspace and the host structs that a program keeps beside its buffers
        _own_prepare(st)
    return st


# ------------------------------------------------------------------------------- the plain forms


def _plain_linattn(q, k, v, log_decay, dones, x0, back):
    """R_p = (1 - cut) g R_{p-1} + k_p v_p^T and o_p = R_p^T q_p for float32 [T, E, H, d], in chunks whose products are
    one batch each; only the states go from chunk to chunk. Forward, a done at p cuts before p, and x0 is R_{-1}; going
    back (rows in reversed order), a done at p cuts after p, and x0 is added to R_0. Returns o and R_{T-1}, or, going
    back, the g R_{T-1} that the cut after the last row leaves."""
    T, E, H, dk = q.shape
    dv = v.shape[-1]
    L = min(CHUNK, T)
    nc = -(-T // L)
    pad = nc * L - T

    def chunks(x):   # [nc, E, H, L, d]
        if pad:
            x = torch.cat([x, x.new_zeros(pad, *x.shape[1:])])
        return x.reshape(nc, L, E, H, x.shape[-1]).permute(0, 2, 3, 1, 4).contiguous()

    q, k, v = chunks(q), chunks(k), chunks(v)
    if pad:
        dones = torch.cat([dones, dones.new_zeros(pad, E)])
    d = dones.reshape(nc, L, E).permute(0, 2, 1).to(torch.int32)               # [nc, E, L]
    cnt = d.cumsum(-1, dtype=torch.int32)
    total = cnt[..., -1:]
    if back:
        cnt = cnt - d
    i = torch.arange(L, device=DEV)
    n = torch.full((nc, 1), L, device=DEV)
    n[-1] = L - pad                                                            # rows of each chunk
    a = log_decay.double()[:, None]
    later = 0 if back else 1
    inter = torch.exp((i + later) * a).float()                                 # [H, L]
    left = n - later - i                                                       # [nc, L]: steps to the chunk's end
    into = torch.where(left[:, None] >= 0, torch.exp(left[:, None].clamp_min(0) * a), 0.0).float()      # [nc, H, L]
    over = torch.exp(n[:, None] * a).float()                                   # [nc, H, 1]
    power = torch.exp((i[:, None] - i).clamp_min(0) * a[..., None]).float()    # [H, L, L]
    seen = ((i[:, None] >= i) & (cnt[..., :, None] == cnt[..., None, :]))[:, :, None]
    inter = inter * (cnt == 0)[:, :, None]                                     # [nc, E, H, L]
    into = into[:, None] * (cnt == total)[:, :, None]
    over = over[:, None] * (total == 0)[:, :, None]                            # [nc, E, H, 1]
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()) * torch.where(seen, power, 0.0)
    o = torch.matmul(p, v)
    add = torch.matmul((k * into[..., None]).transpose(-1, -2).contiguous(), v)   # [nc, E, H, dk, dv]
    x = x0
    start = torch.empty_like(add)
    for c in range(nc):
        start[c] = x
        x = over[c][..., None] * x + add[c]
    o = o + torch.matmul(q, start) * inter[..., None]
    return o.permute(0, 3, 1, 2, 4).reshape(nc * L, E, H, dv)[:T], x


def _plain_la_fwd(st):
    q, k, v = (st[x].float() for x in "qkv")
    o, s = _plain_linattn(q, k, v, st["log_decay"], st["dones"], st["s0"], False)
    return dict(o=(st["scale"] * o).to(st["v"].dtype), s_out=s)


def _plain_la_bwd(st):
    q, k, v, do = (st[x].float() for x in ("q", "k", "v", "do"))
    a, d, dt = st["log_decay"], st["dones"], st["v"].dtype
    do = st["scale"] * do
    dq, _ = _plain_linattn(do, v, k, a, d, st["s0"].transpose(-1, -2), False)
    q, k, v, do, d = (x.flip(0) for x in (q, k, v, do, d))
    dk, _ = _plain_linattn(v, do, q, a, d, st["ds_out"].transpose(-1, -2), True)
    dv, ds0 = _plain_linattn(k, q, do, a, d, st["ds_out"], True)
    return dict(dq=dq.to(dt), dk=dk.flip(0).to(dt), dv=dv.flip(0).to(dt), ds0=ds0)


def _plain_la_step(st):
    q, k, v = (st[x][0].float() for x in "qkv")
    keep = torch.exp(st["log_decay"].double()).float() * (st["dones"][0] == 0)[:, None]
    s = keep[..., None, None] * st["s0"] + k[..., :, None] * v[..., None, :]
    o = st["scale"] * (q[..., :, None] * s).sum(-2)
    return dict(o=o[None].to(st["v"].dtype), s_out=s)


def _norm(x, kind):
    """(the normalised rows, 1 / their deviation) over the last axis."""
    if kind == "off":
        return x, torch.ones_like(x[..., :1])
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return x * r, r


def _norm_back(d, xh, r, kind):
    if kind == "off":
        return d
    out = d - xh * (d * xh).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - d.mean(-1, keepdim=True)
    return out * r


def _gate(x, kind):
    """(act, its derivative)"""
    if kind == "linear":
        return x, torch.ones_like(x)
    s = 1 / (1 + torch.exp(-x))
    if kind == "sigmoid":
        return s, s * (1 - s)
    return x * s, s * (1 + x * (1 - s))


def _plain_bn_fwd(st):
    case, dt = st["case"], st["h"].dtype
    n, C, G = case["n"], case["C"], case["groups"]
    u = _norm(st["h"].float().reshape(n, G, C // G), case["norm"])[0].reshape(n, C) * st["gamma"]
    if st["beta"] is not None:
        u = u + st["beta"]
    if st["gate"] is not None:
        u = u * _gate(st["gate"].float(), case["gate"])[0]
    if st["rscale"] is not None:
        u = u * st["rscale"]
    if st["res"] is not None:
        u = st["res"].float() + u
    res = dict(out=u.to(dt))
    if case["norm2"] != "off":   # of the sum as it is stored
        y = _norm(res["out"].float(), case["norm2"])[0] * st["gamma2"]
        res["out2"] = (y if st["beta2"] is None else y + st["beta2"]).to(dt)
    return res


def _plain_bn_bwd(st):
    case, dt = st["case"], st["h"].dtype
    n, C, G = case["n"], case["C"], case["groups"]
    col = lambda x: x.sum(0, dtype=torch.float64).float()   # noqa: E731
    res = {}
    ds = st["dout"].float()
    if case["norm2"] != "off":
        xh, r = _norm(st["out"].float(), case["norm2"])
        d2 = st["dout2"].float()
        res["dgamma2"] = col(d2 * xh)
        if st["beta2"] is not None:
            res["dbeta2"] = col(d2)
        ds = ds + _norm_back(d2 * st["gamma2"], xh, r, case["norm2"])
        if st["res"] is not None:
            res["dres"] = ds.to(dt)
    xh, r = _norm(st["h"].float().reshape(n, G, C // G), case["norm"])
    z = xh.reshape(n, C) * st["gamma"]
    if st["beta"] is not None:
        z = z + st["beta"]
    du = ds if st["rscale"] is None else ds * st["rscale"]
    if st["gate"] is not None:
        act, slope = _gate(st["gate"].float(), case["gate"])
        res["dgate"] = (du * z * slope).to(dt)
        dz = du * act
    else:
        act, dz = None, du
    if st["rscale"] is not None:
        res["drscale"] = col(ds * (z if act is None else z * act))
    res["dgamma"] = col(dz * xh.reshape(n, C))
    if st["beta"] is not None:
        res["dbeta"] = col(dz)
    d = (dz * st["gamma"]).reshape(n, G, C // G)
    res["dh"] = _norm_back(d, xh, r, case["norm"]).reshape(n, C).to(dt)
    return res


def _plain_clip(st):
    sq = torch.stack([x.double().square().sum() for x in st["src"]]).sum()
    norm = sq.sqrt()
    limit = st["case"]["limit"]
    f = torch.where(norm > limit, limit / norm, torch.ones_like(norm)).float()
    for s, d in zip(st["src"], st["dst"]):
        torch.mul(s.float(), f, out=d)
    st["stats"][0], st["stats"][1] = norm.float(), (~torch.isfinite(norm)).float()
    return dict(flat=st["flat"], stats=st["stats"])


# ------------------------------------------------------------------------------- the framework's calls


def _own_prepare(st):
    import paper_2310_00036_amd as P
    case = st["case"]
    kind = case["kind"]
    prec = P.PREC_BF16 if case["type"] == "bf16" else P.PREC_FP32
    ws = 0
    if kind.startswith("la"):
        if kind == "la_bwd":
            st["shape"] = P.linattn_shape(st["q"], st["k"], st["v"], st["do"], st["dones"], st["scale"], st["dq"], st["dk"],
                                          st["dv"])
        else:
            st["shape"] = P.linattn_shape(st["q"], st["k"], st["v"], st["o"], st["dones"], st["scale"])
        if kind != "la_step":
            ws = P.impala_linattn_workspace_bytes(st["shape"], int(kind == "la_bwd"))
    elif kind.startswith("bn"):
        norms = dict(off=P.NORM_NONE, layer=P.NORM_LAYER, rms=P.NORM_RMS)
        gates = dict(off=P.GATE_LINEAR, linear=P.GATE_LINEAR, silu=P.GATE_SILU, sigmoid=P.GATE_SIGMOID)
        st["shape"] = P.blocknorm_shape(prec, case["n"], case["C"], case["groups"], norms[case["norm"]],
                                        norms[case["norm2"]], gates[case["gate"]], EPS)
        if kind == "bn_bwd":
            ws = P.impala_blocknorm_bwd_workspace_bytes(st["shape"])
    else:
        st["tensors"] = P.grad_tensors(zip(st["src"], st["dst"]))
        ws = P.grad_clip_workspace_bytes(st["tensors"])
    st["ws"] = torch.empty(max(ws, 16), dtype=torch.uint8, device=DEV)


def _own_run(st):
    import paper_2310_00036_amd as P
    case = st["case"]
    kind = case["kind"]
    if kind == "la_fwd":
        P.impala_linattn_fwd(st["shape"], st["q"], st["k"], st["v"], st["log_decay"], st["dones"], st["s0"], st["o"],
                             st["s_out"], st["ws"])
        return dict(o=st["o"], s_out=st["s_out"])
    if kind == "la_step":
        P.impala_linattn_step(st["shape"], st["q"], st["k"], st["v"], st["log_decay"], st["dones"], st["s0"], st["o"],
                              st["s_out"])
        return dict(o=st["o"], s_out=st["s_out"])
    if kind == "la_bwd":
        P.impala_linattn_bwd(st["shape"], st["do"], st["q"], st["k"], st["v"], st["log_decay"], st["dones"], st["s0"],
                             st["ds_out"], st["dq"], st["dk"], st["dv"], st["ds0"], st["ws"])
        return {x: st[x] for x in ("dq", "dk", "dv", "ds0")}
    if kind == "bn_fwd":
        P.impala_blocknorm_fwd(st["shape"], st["h"], st["gamma"], st["beta"], st["gate"], st["rscale"], st["res"], st["out"],
                               st["gamma2"], st["beta2"], st["out2"])
        return {x: st[x] for x in ("out", "out2") if st[x] is not None}
    if kind == "bn_bwd":
        P.impala_blocknorm_bwd(st["shape"], st["dout"], st["dout2"], st["h"], st["gamma"], st["beta"], st["gate"],
                               st["rscale"], st["out"], st["gamma2"], st["dh"], st["dgamma"], st["dbeta"], st["dgate"],
                               st["drscale"], st["dres"], st["dgamma2"], st["dbeta2"], st["ws"])
        return {x: st[x] for x in ("dgamma2", "dbeta2", "dres", "dgate", "drscale", "dgamma", "dbeta", "dh")
                if st[x] is not None}
    P.grad_clip(st["tensors"], case["limit"], st["stats"], st["ws"])
    return dict(flat=st["flat"], stats=st["stats"])


def run(st):
    if own:
        return _own_run(st)
    return dict(la_fwd=_plain_la_fwd, la_bwd=_plain_la_bwd, la_step=_plain_la_step, bn_fwd=_plain_bn_fwd,
                bn_bwd=_plain_bn_bwd, clip=_plain_clip)[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------- work


def work(case):
    kind = case["kind"]
    if kind.startswith("la"):
        es = 2 if case["type"] == "bf16" else 4
        rows, H, dk, dv = case.get("T", 1) * case["E"], case["heads"], case["dk"], case["dv"]
        state = 4 * case["E"] * H * dk * dv
        if kind == "la_bwd":
            return {"bytes": rows * H * (4 * dk + 3 * dv) * es + rows + 3 * state, "flops": 10 * rows * H * dk * dv}
        return {"bytes": rows * H * (2 * dk + 2 * dv) * es + rows + 2 * state, "flops": 4 * rows * H * dk * dv}
    if kind.startswith("bn"):
        es = 2 if case["type"] == "bf16" else 4
        gate, two = case["gate"] != "off", case["norm2"] != "off"
        vecs = 1 + case["scaled"] + two + case["biased"] * (1 + two)
        if kind == "bn_fwd":
            return {"bytes": case["n"] * case["C"] * es * (2 + gate + case["res"] + two) + 4 * case["C"] * vecs,
                    "flops": case["n"] * case["C"] * (8 + 8 * gate + 6 * two)}
        arrays = 3 + 2 * gate + 2 * two + (two and case["res"])
        return {"bytes": case["n"] * case["C"] * es * arrays + 8 * case["C"] * vecs,
                "flops": case["n"] * case["C"] * (16 + 14 * gate + 14 * two)}
    sizes = _clip_tensors(case)
    src = sum(k * (2 if dt == torch.bfloat16 else 4) for k, dt in sizes)
    total = sum(k for k, _ in sizes)
    return {"bytes": src + 4 * total, "flops": 3 * total}


# ------------------------------------------------------------------------------- 64 bits


def _exact_la(st):
    """Step by step, as the recurrence says."""
    kind = st["case"]["kind"]
    q, k, v = (st[x].double() for x in "qkv")
    T, E = st["dones"].shape
    keep = torch.exp(st["log_decay"].double()) * (st["dones"] == 0).double()[..., None]   # [T, E, H]
    keep = keep[..., None, None]
    s = st["s0"].double()
    outer = lambda x, y: x[..., :, None] * y[..., None, :]   # noqa: E731
    if kind != "la_bwd":
        o = torch.empty_like(v)
        for t in range(T):
            s = keep[t] * s + outer(k[t], v[t])
            o[t] = (q[t][..., :, None] * s).sum(-2)
        return dict(o=st["scale"] * o, s_out=s)
    do = st["scale"] * st["do"].double()
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for t in range(T):
        s = keep[t] * s + outer(k[t], v[t])
        dq[t] = (s * do[t][..., None, :]).sum(-1)
    g = st["ds_out"].double()
    for t in range(T - 1, -1, -1):
        g = g + outer(q[t], do[t])
        dk[t] = (g * v[t][..., None, :]).sum(-1)
        dv[t] = (g * k[t][..., :, None]).sum(-2)
        g = keep[t] * g
    return dict(dq=dq, dk=dk, dv=dv, ds0=g)


def _exact_bn(st):
    """The forward in 64 bits, and its gradients by autograd."""
    case, dt = st["case"], st["h"].dtype
    n, C, G = case["n"], case["C"], case["groups"]
    back = case["kind"] == "bn_bwd"

    def leaf(name):
        x = st[name]
        return None if x is None else x.double().requires_grad_(back)

    def normed(x, kind):
        if kind == "rms":
            return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        if kind == "layer":
            var, mean = torch.var_mean(x, dim=-1, keepdim=True, unbiased=False)
            return (x - mean) / torch.sqrt(var + EPS)
        return x

    h, gamma, beta, gate, rscale = (leaf(x) for x in ("h", "gamma", "beta", "gate", "rscale"))
    u = normed(h.view(n, G, C // G), case["norm"]).view(n, C) * gamma
    if beta is not None:
        u = u + beta
    if gate is not None:
        u = u * (gate if case["gate"] == "linear" else torch.sigmoid(gate) * (gate if case["gate"] == "silu" else 1))
    if rscale is not None:
        u = u * rscale
    gamma2, beta2 = leaf("gamma2"), leaf("beta2")

    def second(x):
        y = normed(x, case["norm2"]) * gamma2
        return y if beta2 is None else y + beta2

    if not back:
        out = u if st["res"] is None else st["res"].double() + u
        return dict(out=out) if gamma2 is None else dict(out=out, out2=second(out.to(dt).double()))
    res = {}
    ds = st["dout"].double()
    if gamma2 is not None:
        x = leaf("out")
        leaves = [y for y in (x, gamma2, beta2) if y is not None]
        grads = torch.autograd.grad(second(x), leaves, st["dout2"].double())
        ds = ds + grads[0]
        res["dgamma2"] = grads[1]
        if beta2 is not None:
            res["dbeta2"] = grads[2]
        if st["res"] is not None:
            res["dres"] = ds
    leaves = dict(dgate=gate, drscale=rscale, dgamma=gamma, dbeta=beta, dh=h)
    leaves = {name: x for name, x in leaves.items() if x is not None}
    res.update(zip(leaves, torch.autograd.grad(u, list(leaves.values()), ds)))
    return res


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("la"):
        return _exact_la(st)
    if case["kind"].startswith("bn"):
        return _exact_bn(st)
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in st["src"]))
    f = min(1.0, case["limit"] / norm)
    return dict(flat=torch.cat([f * x.double() for x in st["src"]]),
                stats=torch.tensor([norm, 0.0], dtype=torch.float64, device=DEV))
