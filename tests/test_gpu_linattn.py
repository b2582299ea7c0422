"""Linear attention with a decay per head against the step-by-step recurrence in 64 bits: outputs, states and gradients,
from one step to long rollouts, episode starts anywhere, odd sizes, strided arrays, values that are not finite."""
import pytest
import torch

from tests import memory_ref as ref

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

#        T, E, heads, dk, dv
SIZES = [(1, 1, 1, 1, 1), (1, 5, 3, 16, 64), (2, 3, 2, 7, 9), (15, 2, 2, 16, 16), (16, 2, 3, 32, 48), (17, 3, 1, 5, 128),
         (33, 1, 2, 128, 3), (63, 2, 2, 32, 32), (64, 3, 2, 64, 64), (65, 2, 4, 64, 64), (128, 2, 2, 64, 128),
         (130, 2, 3, 33, 71), (200, 1, 2, 128, 128), (257, 2, 1, 100, 40), (700, 1, 2, 48, 64), (1500, 1, 1, 64, 32)]
DONES = ["none", "null", "few", "many", "all", "first", "edge"]


def make(T, E, H, dk, dv, ty, dones, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[ty]
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    x = dict(q=r(T, E, H, dk).to(dt), k=r(T, E, H, dk).to(dt), v=r(T, E, H, dv).to(dt), do=r(T, E, H, dv).to(dt),
             s0=r(E, H, dk, dv), ds=r(E, H, dk, dv),
             a=torch.log1p(-(2.0 ** -(1.0 + torch.arange(H) * 2.5))))
    d = torch.zeros(T, E, dtype=torch.uint8)
    if dones in ("few", "many"):
        d = (torch.rand(T, E, generator=g) < (0.02 if dones == "few" else 0.3)).to(torch.uint8)
    elif dones == "all":
        d += 1
    elif dones == "first":
        d[0] = 1
    elif dones == "edge":   # about the borders of the chunks of 64
        for t in (63, 64, 65, 127, 128):
            if t < T:
                d[t, t % E] = 1
    x["d"] = None if dones == "null" else d
    return x


def dev(x):
    return None if x is None else x.to(DEV)


def workspace(shape, backward=0):
    n = P.impala_linattn_workspace_bytes(shape, backward)
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def forward(x, scale, s0=True, want_state=True):
    q, k, v, a, d = (dev(x[n]) for n in ("q", "k", "v", "a", "d"))
    o = torch.empty_like(v)
    st = dev(x["s0"]) if s0 else None
    s_out = torch.empty(*x["s0"].shape, device=DEV) if want_state else None
    shape = P.linattn_shape(q, k, v, o, d, scale)
    P.impala_linattn_fwd(shape, q, k, v, a, d, st, o, s_out, workspace(shape))
    return o, s_out


def backward(x, scale, s0=True, ds=True, want_state=True):
    q, k, v, a, d, do = (dev(x[n]) for n in ("q", "k", "v", "a", "d", "do"))
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ds0 = torch.empty(*x["s0"].shape, device=DEV) if want_state else None
    shape = P.linattn_shape(q, k, v, do, d, scale, dq, dk, dv)
    P.impala_linattn_bwd(shape, do, q, k, v, a, d, dev(x["s0"]) if s0 else None, dev(x["ds"]) if ds else None, dq, dk, dv,
                         ds0, workspace(shape, 1))
    return dq, dk, dv, ds0


def magnitudes(x, *names):
    return [None if x[n] is None else x[n].double().abs() for n in names]


def check_forward(x, ty, scale, got, s0=True):
    o, s = ref.linattn(x["q"], x["k"], x["v"], x["a"], x["d"], x["s0"] if s0 else None, scale)
    q, k, v, st = magnitudes(x, "q", "k", "v", "s0")
    om, sm = ref.linattn(q, k, v, x["a"], x["d"], st if s0 else None, abs(scale))
    T, dk = x["q"].shape[0], x["q"].shape[3]
    ref.assert_close("o", got[0], o, om, T + dk + 16, ty == "bf16")
    if got[1] is not None:   # its products are exact or held in 24 bits: no share of 2^-17
        ref.assert_close("s_out", got[1], s, sm, T + 16, False)


def check_backward(x, ty, scale, got, s0=True, ds=True):
    args = ("do", "q", "k", "v")
    want = ref.linattn_grads(*(x[n] for n in args), x["a"], x["d"], x["s0"] if s0 else None, x["ds"] if ds else None, scale)
    mag = ref.linattn_grads(*magnitudes(x, *args), x["a"], x["d"], x["s0"].abs() if s0 else None,
                            x["ds"].abs() if ds else None, abs(scale))
    T, _, _, dk = x["q"].shape
    terms = T + max(dk, x["v"].shape[3]) + 16
    for name, g, w, m in zip(("dq", "dk", "dv"), got, want, mag):
        ref.assert_close(name, g, w, m, terms, ty == "bf16")
    if got[3] is not None:
        ref.assert_close("ds0", got[3], want[3], mag[3], T + 16, False)


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, ty):
    for i, dones in enumerate(DONES):
        x = make(*size, ty, dones, seed=i)
        check_forward(x, ty, 0.3, forward(x, 0.3))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES)
def test_backward(size, ty):
    for i, dones in enumerate(DONES):
        x = make(*size, ty, dones, seed=10 + i)
        check_backward(x, ty, 0.3, backward(x, 0.3))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 2, 2, 16, 16), (70, 2, 2, 64, 48), (700, 1, 1, 32, 32)])
def test_optional_states(size, ty):
    x = make(*size, ty, "few")
    check_forward(x, ty, 1.0, forward(x, 1.0, s0=False), s0=False)
    check_forward(x, ty, 1.0, forward(x, 1.0, want_state=False))
    check_backward(x, ty, 1.0, backward(x, 1.0, s0=False, ds=False), s0=False, ds=False)
    check_backward(x, ty, 1.0, backward(x, 1.0, want_state=False))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 4, 2, 64, 64), (1, 3, 5, 31, 70), (1, 130, 2, 128, 128)])
def test_step(size, ty):
    for dones in ("none", "null", "many", "all"):
        x = make(*size, ty, dones)
        q, k, v, a, d, s = (dev(x[n]) for n in ("q", "k", "v", "a", "d", "s0"))
        o, s_out = torch.empty_like(v), torch.empty_like(s)
        shape = P.linattn_shape(q, k, v, o, d, 0.3)
        P.impala_linattn_step(shape, q, k, v, a, d, s, o, s_out)
        check_forward(x, ty, 0.3, (o, s_out))
        o2 = torch.empty_like(o)
        P.impala_linattn_step(shape, q, k, v, a, d, s, o2, s)   # in place
        assert torch.equal(s, s_out) and torch.equal(o, o2)
        P.impala_linattn_step(shape, q, k, v, a, d, None, o, s_out)
        check_forward(x, ty, 0.3, (o, s_out), s0=False)


@pytest.mark.parametrize("ty", ["bf16", "f32"])
def test_actor_steps_follow_the_learners_rollout(ty):
    """The same rollout in single steps and at once, and in two rollouts with the state handed over, also in place."""
    T, E, H, dk, dv = 150, 3, 2, 64, 32
    x = make(T, E, H, dk, dv, ty, "few", seed=3)
    q, k, v, a, d = (dev(x[n]) for n in ("q", "k", "v", "a", "d"))
    state, outs = dev(x["s0"]).clone(), []
    for t in range(T):
        o = torch.empty(1, E, H, dv, dtype=v.dtype, device=DEV)
        s = slice(t, t + 1)
        P.impala_linattn_step(P.linattn_shape(q[s], k[s], v[s], o, d[s], 0.2), q[s], k[s], v[s], a, d[s], state, o, state)
        outs.append(o)
    check_forward(x, ty, 0.2, (torch.cat(outs), state))
    state, outs = dev(x["s0"]).clone(), []
    for s in (slice(0, 77), slice(77, T)):
        o = torch.empty_like(v[s])
        shape = P.linattn_shape(q[s], k[s], v[s], o, d[s], 0.2)
        P.impala_linattn_fwd(shape, q[s], k[s], v[s], a, d[s], state, o, state, workspace(shape))
        outs.append(o)
    check_forward(x, ty, 0.2, (torch.cat(outs), state))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(5, 24), (90, 64), (90, 27), (800, 32)])
def test_strided_arrays(ty, T, d):
    """Parts of one projection's output, env-major arrays, an env block of a larger rollout, keys shared by all heads:
    the same bits as from contiguous arrays, and nothing written beside the outputs."""
    E, H = 3, 2
    x = make(T, E, H, d, d, ty, "few", seed=T)
    want = forward(x, 0.5)
    grads = backward(x, 0.5)
    a, s0, ds, dt = dev(x["a"]), dev(x["s0"]), dev(x["ds"]), TYPES[ty]

    packed = torch.full((T, E, 8, H, d), 7.0, dtype=dt, device=DEV)
    block = torch.full((T, E + 3, 8, H, d), 7.0, dtype=dt, device=DEV)[:, 2:2 + E]
    major = torch.full((E, T, H, 8 * d), 7.0, dtype=dt, device=DEV)
    wide = torch.zeros(T, E + 3, dtype=torch.uint8, device=DEV)
    wide[:, 2:2 + E] = x["d"].to(DEV)
    for kind in ("packed", "block", "major"):
        if kind == "major":
            part = [major[..., i * d:(i + 1) * d].transpose(0, 1) for i in range(8)]
            dones = dev(x["d"]).t().contiguous().t()
        else:
            part = [(packed if kind == "packed" else block)[:, :, i] for i in range(8)]
            dones = dev(x["d"]) if kind == "packed" else wide[:, 2:2 + E]
        q, k, v, o, do, dq, dk, dv = part
        for n, t in (("q", q), ("k", k), ("v", v), ("do", do)):
            t.copy_(dev(x[n]))
        s_out, ds0 = torch.empty_like(s0), torch.empty_like(s0)
        shape = P.linattn_shape(q, k, v, o, dones, 0.5)
        P.impala_linattn_fwd(shape, q, k, v, a, dones, s0, o, s_out, workspace(shape))
        assert torch.equal(o, want[0]) and torch.equal(s_out, want[1]), kind
        assert (dq == 7).all() and (dk == 7).all() and (dv == 7).all(), kind
        shape = P.linattn_shape(q, k, v, do, dones, 0.5, dq, dk, dv)
        P.impala_linattn_bwd(shape, do, q, k, v, a, dones, s0, ds, dq, dk, dv, ds0, workspace(shape, 1))
        for g, w in zip((dq, dk, dv, ds0), grads):
            assert torch.equal(g, w), kind
        for n, t in (("q", q), ("k", k), ("v", v), ("do", do)):
            assert torch.equal(t, dev(x[n])), (kind, n)
    assert (block._base[:, :2] == 7).all() and (block._base[:, 2 + E:] == 7).all()

    x["k"] = x["k"][:, :, :1].expand(T, E, H, d)   # one key for all heads
    full = {**x, "k": x["k"].contiguous()}
    o = torch.empty(T, E, H, d, dtype=dt, device=DEV)
    s_out = torch.empty_like(s0)
    q, v, dones, do = (dev(x[n]) for n in ("q", "v", "d", "do"))
    k = dev(full["k"])[:, :, :1].expand(T, E, H, d)
    shape = P.linattn_shape(q, k, v, o, dones, 0.5)
    P.impala_linattn_fwd(shape, q, k, v, a, dones, s0, o, s_out, workspace(shape))
    assert k.stride(2) == 0 and all(torch.equal(g, w) for g, w in zip((o, s_out), forward(full, 0.5)))
    dq, dk, dv, ds0 = (torch.empty_like(t) for t in (q, q, v, s0))
    shape = P.linattn_shape(q, k, v, do, dones, 0.5, dq, dk, dv)
    P.impala_linattn_bwd(shape, do, q, k, v, a, dones, s0, ds, dq, dk, dv, ds0, workspace(shape, 1))
    assert all(torch.equal(g, w) for g, w in zip((dq, dk, dv, ds0), backward(full, 0.5)))


@pytest.mark.parametrize("d", [7, 27, 66])
def test_odd_sizes_at_even_strides(d):
    """bf16 rows that end inside a 4-byte word, or between two, in wider arrays at 4-byte addresses: up to the last row's
    last element, with infinities behind it."""
    T, E, H, w = 130, 2, 2, 72
    x = make(T, E, H, d, d, "bf16", "few", seed=d)
    want = forward(x, 0.5), backward(x, 0.5)
    a, s0, ds = dev(x["a"]), dev(x["s0"]), dev(x["ds"])

    def wide(t):
        base = torch.full((T, E, H, w), float("inf"), dtype=torch.bfloat16, device=DEV)
        base[..., :d].copy_(t.to(DEV))
        return base[..., :d]

    q, k, v, do, o = (wide(x[n]) for n in ("q", "k", "v", "do", "do"))
    dones, s_out = dev(x["d"]), torch.empty_like(s0)
    shape = P.linattn_shape(q, k, v, o, dones, 0.5)
    P.impala_linattn_fwd(shape, q, k, v, a, dones, s0, o, s_out, workspace(shape))
    assert torch.equal(o, want[0][0]) and torch.equal(s_out, want[0][1])
    dq, dk, dv, ds0 = wide(x["q"]), wide(x["k"]), wide(x["v"]), torch.empty_like(s0)
    shape = P.linattn_shape(q, k, v, do, dones, 0.5, dq, dk, dv)
    P.impala_linattn_bwd(shape, do, q, k, v, a, dones, s0, ds, dq, dk, dv, ds0, workspace(shape, 1))
    assert all(torch.equal(g, y) for g, y in zip((dq, dk, dv, ds0), want[1]))
    for t in (o, dq, dk, dv):
        assert torch.isinf(t._base[..., d:]).all()


def poison(x, where, value):
    for n in ("q", "k", "v", "do"):
        x[n][where] = value


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 9, 64, 150, 900])
def test_what_is_not_finite_stays_in_its_episode_and_time(ty, T, value):
    """Env 0 has such values at one step of its second episode: earlier steps' outputs, later episodes' and other envs'
    are those of clean inputs; so are the gradients of other episodes and, behind it in time, none is changed before it."""
    E, H, d = 2, 2, 40
    x = make(T, E, H, d, d, ty, "none", seed=T)
    t0, t1, bad = T // 3, 2 * T // 3, T // 2
    x["d"][t0, 0] = x["d"][t1, 0] = 1
    clean = forward(x, 0.5), backward(x, 0.5)
    y = {n: v.clone() for n, v in x.items()}
    poison(y, (bad, 0), value)
    got = forward(y, 0.5), backward(y, 0.5)
    lo, hi = (t0, t1) if bad < t1 else (t1, T)     # the poisoned episode's steps
    if lo < hi:
        touched = torch.zeros(T, E, dtype=torch.bool)
        touched[bad:hi, 0] = True                  # outputs: from the step on
        assert torch.equal(got[0][0][~touched.to(DEV)], clean[0][0][~touched.to(DEV)])
        assert not torch.isfinite(got[0][0][bad, 0]).any()
        touched[lo:hi, 0] = True                   # gradients: anywhere in the episode
        for g, w in zip(got[1][:3], clean[1][:3]):
            assert torch.equal(g[~touched.to(DEV)], w[~touched.to(DEV)])
        if hi < T:
            assert torch.equal(got[0][1], clean[0][1])
        if lo > 0:
            assert torch.equal(got[1][3], clean[1][3])
    # a state that is not finite ends at the episode's start
    z = {n: v.clone() for n, v in x.items()}
    z["d"][0] = 1
    want = forward(z, 0.5)
    z["s0"][:] = value
    assert all(torch.equal(g, w) for g, w in zip(forward(z, 0.5), want))


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(16, 1), (1, 16), (7, 1), (1, 1), (5, 3)])
def test_a_states_number_reaches_its_row_and_column_only(dk, dv, ty):
    x = make(70, 1, 1, dk, dv, ty, "none", seed=dk)
    clean = forward(x, 1.0), backward(x, 1.0)
    k, n = dk - 1, dv - 1
    x["s0"][0, 0, k, n] = float("nan")
    (o, s), (dq, dkk, dvv, ds0) = forward(x, 1.0), backward(x, 1.0)
    for g, w, axis, i in ((o, clean[0][0], 3, n), (dq, clean[1][0], 3, k)):
        keep = [j for j in range(g.shape[axis]) if j != i]
        assert torch.equal(g[..., keep], w[..., keep]) and g[..., i].isnan().all()
    bad = torch.zeros_like(s, dtype=torch.bool)
    bad[0, 0, k, n] = True
    assert torch.equal(s[~bad], clean[0][1][~bad]) and s[bad].isnan().all()
    assert all(torch.equal(g, w) for g, w in zip((dkk, dvv, ds0), clean[1][1:]))


def test_decays_of_none_and_of_everything():
    """Decay 1 (sums over all steps), decay 0 (log of -infinity: one step's memory) and a fast one that underflows."""
    for T in (3, 200):
        x = make(T, 2, 3, 32, 32, "f32", "few")
        x["a"] = torch.tensor([0.0, -float("inf"), -60.0])
        check_forward(x, "f32", 1.0, forward(x, 1.0))
        check_backward(x, "f32", 1.0, backward(x, 1.0))


@pytest.mark.parametrize("T", [7, 100])
def test_gradients_against_differences(T):
    """The kernel's own gradient along a direction against central differences of the 64-bit forward."""
    x = make(T, 2, 2, 24, 40, "f32", "few", seed=5)
    g = torch.Generator().manual_seed(9)
    u = {n: torch.randn(*x[n].shape, generator=g).double() for n in ("q", "k", "v", "s0")}
    grads = dict(zip(("q", "k", "v", "s0"), backward(x, 0.4)))

    def loss(h):
        y = {n: x[n].double() + h * u[n] for n in u}
        o, s = ref.linattn(y["q"], y["k"], y["v"], x["a"], x["d"], y["s0"], 0.4)
        return float((o * x["do"].double()).sum() + (s * x["ds"].double()).sum())

    h = 1e-4   # cubic in the step: the difference's own error is h^2 times a third derivative of the loss's size
    slope = (loss(h) - loss(-h)) / (2 * h)
    got = sum(float((grads[n].double().cpu() * u[n]).sum()) for n in u)
    size = sum(float((grads[n].double().cpu() * u[n]).abs().sum()) for n in u)
    assert abs(got - slope) < 1e-5 * size


@pytest.mark.parametrize("ty", ["bf16", "f32"])
def test_no_rows(ty):
    x = make(4, 2, 2, 16, 8, ty, "none")
    q, k, v, a, d = (dev(x[n])[:0] if n != "a" else dev(x[n]) for n in ("q", "k", "v", "a", "d"))
    s0, out = dev(x["s0"]), torch.full((2, 2, 16, 8), 3.0, device=DEV)
    shape = P.linattn_shape(q, k, v, v.clone(), d, 1.0)
    P.impala_linattn_fwd(shape, q, k, v, a, d, s0, v.clone(), out, workspace(shape))
    assert torch.equal(out, s0)
    P.impala_linattn_fwd(shape, q, k, v, a, d, None, v.clone(), out, workspace(shape))
    assert (out == 0).all()
    shape = P.linattn_shape(q, k, v, v, d, 1.0, q, k, v)
    P.impala_linattn_bwd(shape, v, q, k, v, a, d, None, s0, q, k, v, out, workspace(shape, 1))
    assert torch.equal(out, s0)
    e = [dev(x[n])[:, :0] for n in ("q", "k", "v", "d")]
    shape = P.linattn_shape(e[0], e[1], e[2], e[2], e[3], 1.0)
    P.impala_linattn_fwd(shape, e[0], e[1], e[2], a, e[3], None, e[2], None, None)


@pytest.mark.parametrize("T,E", [(128, 3), (900, 1)])
def test_streams_graphs_and_repeats(T, E):
    """Two streams at once, a captured call replayed between eager ones, repeated calls: the same bits."""
    xs = [make(T, E, 2, 64, 64, "bf16", "few", seed=i) for i in range(2)]
    want = [(forward(x, 0.5), backward(x, 0.5)) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append((forward(x, 0.5), backward(x, 0.5)))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for y, z in zip(g, w) for a, b in zip(y, z))

    x = xs[0]
    q, k, v, a, d, do, s0, ds = (dev(x[n]) for n in ("q", "k", "v", "a", "d", "do", "s0", "ds"))
    o, s_out = torch.empty_like(v), torch.empty_like(s0)
    dq, dk, dv, ds0 = (torch.empty_like(t) for t in (q, k, v, s0))
    f, b = P.linattn_shape(q, k, v, o, d, 0.5), P.linattn_shape(q, k, v, do, d, 0.5, dq, dk, dv)
    ws = [workspace(f), workspace(b, 1)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.impala_linattn_fwd(f, q, k, v, a, d, s0, o, s_out, ws[0])
        P.impala_linattn_bwd(b, do, q, k, v, a, d, s0, ds, dq, dk, dv, ds0, ws[1])
    for i in (0, 1, 0):
        for n, t in (("q", q), ("k", k), ("v", v), ("d", d), ("do", do), ("s0", s0), ("ds", ds)):
            t.copy_(xs[i][n])
        for t in (o, s_out, dq, dk, dv, ds0):
            t.fill_(9)
        graph.replay()
        forward(xs[1 - i], 0.5)
        torch.cuda.synchronize()
        for g, w in zip((o, s_out), want[i][0]):
            assert torch.equal(g, w)
        for g, w in zip((dq, dk, dv, ds0), want[i][1]):
            assert torch.equal(g, w)


def test_offsets_beyond_32_bits():
    """Steps 128 KB apart, 9 GB from the first to the last: the bits of contiguous arrays."""
    T, d, w = 70000, 16, 65536
    x = make(T, 1, 1, d, d, "bf16", "few", seed=4)
    x["d"][::1500] = 1
    big = torch.empty(T, 1, 1, w, dtype=torch.bfloat16, device=DEV)
    q, k, v, do, o, dq, dk, dv = (big[..., i * 1000:i * 1000 + d] for i in range(8))
    for n, t in (("q", q), ("k", k), ("v", v), ("do", do)):
        t.copy_(dev(x[n]))
    a, s0, ds, dones = dev(x["a"]), dev(x["s0"]), dev(x["ds"]), dev(x["d"])
    s_out, ds0 = torch.empty_like(s0), torch.empty_like(s0)
    shape = P.linattn_shape(q, k, v, o, dones, 0.5)
    P.impala_linattn_fwd(shape, q, k, v, a, dones, s0, o, s_out, workspace(shape))
    shape = P.linattn_shape(q, k, v, do, dones, 0.5, dq, dk, dv)
    P.impala_linattn_bwd(shape, do, q, k, v, a, dones, s0, ds, dq, dk, dv, ds0, workspace(shape, 1))
    for g, want in zip((o, s_out, dq, dk, dv, ds0), (*forward(x, 0.5), *backward(x, 0.5))):
        assert torch.equal(g, want)
