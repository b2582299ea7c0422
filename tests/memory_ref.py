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
