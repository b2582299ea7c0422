"""Plain 64-bit evaluations of the memory core's operators, on the CPU, and the sums of magnitudes that their error
bounds are made of."""
import torch


def _outer(x, y):
    return x[..., :, None] * y[..., None, :]


def linattn(q, k, v, log_decay, dones, s0, scale):
    """(o, s_out) step by step: an episode start clears the state."""
    T, E, H, dk = q.shape
    q, k, v = q.double(), k.double(), v.double()
    s = torch.zeros(E, H, dk, v.shape[3], dtype=torch.float64) if s0 is None else s0.double()
    g = torch.exp(log_decay.double())[None, :, None, None]
    o = torch.empty_like(v)
    for t in range(T):
        s = g * s
        if dones is not None:
            s = torch.where(dones[t].bool()[:, None, None, None], torch.zeros_like(s), s)
        s = s + _outer(k[t], v[t])
        o[t] = scale * (q[t][..., :, None] * s).sum(-2)
    return o, s


def linattn_grads(do, q, k, v, log_decay, dones, s0, ds_out, scale):
    """(dq, dk, dv, ds0) from the adjoint recurrence."""
    T, E, H, dk = q.shape
    do, q, k, v = (x.double() for x in (do, q, k, v))
    zeros = torch.zeros(E, H, dk, v.shape[3], dtype=torch.float64)
    g = torch.exp(log_decay.double())[None, :, None, None]
    keep = [g if dones is None else torch.where(dones[t].bool()[:, None, None, None], 0.0, g) for t in range(T)]
    dq, dkk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    s = zeros if s0 is None else s0.double()
    for t in range(T):
        s = keep[t] * s + _outer(k[t], v[t])
        dq[t] = scale * (s * do[t][..., None, :]).sum(-1)
    G = zeros if ds_out is None else ds_out.double()
    for t in range(T - 1, -1, -1):
        G = G + scale * _outer(q[t], do[t])
        dkk[t] = (G * v[t][..., None, :]).sum(-1)
        dv[t] = (G * k[t][..., :, None]).sum(-2)
        G = keep[t] * G
    return dq, dkk, dv, G


def assert_close(name, got, want, mag, terms, bf16, elem_bf16=None):
    """got (from the kernel) against want and mag (64 bits, CPU): want with every term's magnitude.

    float32: a sum of `terms` roundings of half a step each is off by at most terms 2^-24 mag, and, the roundings being
    independent, by about sqrt(terms) 2^-24 |mag| in the 2-norm; twice that is allowed. bf16 inputs: factors held as two
    bf16 numbers add 2^-17 mag. A bf16 output adds its own half step, 2^-8 of the value (2^-9 of it or less in the norm's
    mean square, as mantissas are spread; 2^-8 is allowed)."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, name
    assert torch.isfinite(got).all(), name
    out16 = bf16 if elem_bf16 is None else elem_bf16
    rel = (2.0 ** -17 if bf16 else 0.0)
    tol = (terms * 2.0 ** -24 + rel) * mag + (2.0 ** -8 * (want.abs() + (terms * 2.0 ** -24 + rel) * mag) if out16 else 0.0)
    bad = (got - want).abs() > tol + 1e-37
    assert not bad.any(), (name, int(bad.sum()), float(((got - want).abs() / (tol + 1e-37)).max()))
    norm = float((got - want).norm())
    limit = (2 * terms ** 0.5 * 2.0 ** -24 + rel) * float(mag.norm()) + (2.0 ** -8 * float(want.norm()) if out16 else 0.0)
    assert norm <= limit + 1e-37, (name, norm, limit)


# ------------------------------------------------------------------------------- block norms


def _act(g, kind):
    """(act, slope) of a gate in 64 bits; kind 0 linear, 1 silu, 2 sigmoid."""
    if kind == 0:
        return g, torch.ones_like(g)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if kind == 2 else (g * s, s * (1 + g * (1 - s)))


def _rows(x, kind, eps, size):
    """(xh, rstd, xh's magnitude) of x [n, G, cg]; kind 0 none, 1 layer, 2 rms. size: |x| with the rounded mean's."""
    if kind == 0:
        return x, torch.ones_like(x[..., :1]), size
    if kind == 1:
        size = size + size.mean(-1, keepdim=True)
        x = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return x * r, r, size * r


def blocknorm(h, gamma, beta, gate, rscale, res, groups, kind, act, eps):
    """(out, its magnitude), before out is rounded."""
    n, C = h.shape
    h = h.double()
    xh, _, xm = _rows(h.reshape(n, groups, -1), kind, eps, h.abs().reshape(n, groups, -1))
    z = xh.reshape(n, C) * gamma.double() + beta.double()
    zm = xm.reshape(n, C) * gamma.double().abs() + beta.double().abs()
    if gate is not None:
        a = _act(gate.double(), act)[0]
        z, zm = z * a, zm * a.abs()
    z, zm = z * rscale.double(), zm * rscale.double().abs()
    return (z, zm) if res is None else (z + res.double(), zm + res.double().abs())


def blocknorm_second(out, gamma2, beta2, kind, eps):
    x = out.double()[:, None]
    xh, _, xm = _rows(x, kind, eps, x.abs())
    return xh[:, 0] * gamma2.double() + beta2.double(), xm[:, 0] * gamma2.double().abs() + beta2.double().abs()


def blocknorm_grads(dout, dout2, h, gamma, beta, gate, rscale, out, gamma2, groups, kind, kind2, act, eps):
    """name -> (gradient, magnitude), by the formulas."""
    n, C = h.shape
    gamma, beta, rscale = gamma.double(), beta.double(), rscale.double()

    def back(g, gm, xh, xm, r, kind):
        if kind == 0:
            return g, gm
        m = lambda t: t.mean(-1, keepdim=True)   # noqa: E731
        d, dm = g - xh * m(g * xh), gm + xm * m(gm * xm)
        if kind == 1:
            d, dm = d - m(g), dm + m(gm)
        return r * d, r * dm

    res = {}
    ds = torch.zeros(n, C, dtype=torch.float64) if dout is None else dout.double()
    dm = ds.abs()
    if dout2 is not None:
        x = out.double()
        xh, r, xm = _rows(x, kind2, eps, x.abs())
        d2 = dout2.double()
        res["dgamma2"] = (d2 * xh).sum(0), (d2.abs() * xm).sum(0)
        res["dbeta2"] = d2.sum(0), d2.abs().sum(0)
        g, gm = back(d2 * gamma2.double(), d2.abs() * gamma2.double().abs(), xh, xm, r, kind2)
        ds, dm = ds + g, dm + gm
    res["dres"] = ds, dm
    x = h.double().reshape(n, groups, -1)
    xh, r, xm = _rows(x, kind, eps, x.abs())
    z, zm = xh.reshape(n, C) * gamma + beta, xm.reshape(n, C) * gamma.abs() + beta.abs()
    a, slope, am, sm = 1.0, None, 1.0, None
    if gate is not None:
        a, slope = _act(gate.double(), act)
        am, sm = a.abs(), slope.abs() + (0 if act == 0 else a.abs())   # s (1 + g (1 - s)) may cancel
    res["drscale"] = (ds * z * a).sum(0), (dm * zm * am).sum(0)
    du, um = ds * rscale, dm * rscale.abs()
    if gate is not None:
        res["dgate"] = du * z * slope, um * zm * sm
    dz, dzm = du * a, um * am
    res["dgamma"] = (dz * xh.reshape(n, C)).sum(0), (dzm * xm.reshape(n, C)).sum(0)
    res["dbeta"] = dz.sum(0), dzm.sum(0)
    d, m = back((dz * gamma).reshape(x.shape), (dzm * gamma.abs()).reshape(x.shape), xh, xm, r, kind)
    res["dh"] = d.reshape(n, C), m.reshape(n, C)
    return res
