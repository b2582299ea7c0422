"""Orthogonalised updates and the Muon step against their formulas in 64 bits.

Tolerances. The exact result comes from the steps one by one in float64. The kernels iterate on Gram matrices held to
2^-22 of their norm; within a segment of at most 3 steps P A P multiplies what is small, its rounding included, by
a^2 = 11.9 a step, and P = a + b A + .. turns an error of A into |b| / a = 1.4 times as large a relative one. So the
results differ from the exact ones, relative to their Frobenius norm, by at most
  float32  2^-22 x 11.9^2 x 1.4 (2^-22 x 199) from one segment and a^2 = 12 times less from the other: 2^-14
  bf16     2^-14 as well, and 2^-9 from storing it
and typical matrices (well-conditioned ones) by far less, 2^-17 and 2^-8.5: both are checked. One element is off by at
most 16 times the root mean square error allowed (errors spread over directions), plus its own half step.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import gpu_util as G  # noqa: E402

P = pytest.importorskip("paper_2310_00036_amd")

QUINTIC = (3.4445, -4.7750, 2.0315)
WORST = {G.FP32: 2.0 ** -14, G.BF16: 2.0 ** -14 + 2.0 ** -9}
TYPICAL = {G.FP32: 2.0 ** -17, G.BF16: 2.0 ** -8.5}
U = 2.0 ** -24


def ns(x, steps=5, coeffs=None, eps=1e-7):
    """[..., rows, cols] float64, one step after the other on the smaller side."""
    x = np.asarray(x, np.float64)
    tall = x.shape[-2] > x.shape[-1]
    X = np.swapaxes(x, -1, -2) if tall else x
    X = X / np.maximum(np.sqrt((X * X).sum((-1, -2), keepdims=True)), eps)
    for k in range(steps):
        a, b, c = (np.float64(np.float32(v)) for v in (QUINTIC if coeffs is None else coeffs[k]))
        A = X @ np.swapaxes(X, -1, -2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return np.swapaxes(X, -1, -2) if tall else X


def _orth(prec, x, steps=5, coeffs=None, eps=1e-7, inplace=False, shift=0):
    t = G.torch()
    b, r, c = x.shape
    buf = t.zeros(x.size + shift, dtype=t.bfloat16 if prec == G.BF16 else t.float32, device="cuda:0")
    dx = buf[shift:]
    dx.copy_(G.dev_act(x, prec).reshape(-1))
    out = t.full((x.size + shift,), 7.0, dtype=buf.dtype, device="cuda:0")
    y = dx if inplace else out[shift:]
    ws = G.ws_bytes(P.muon_orthogonalize_workspace_bytes(prec, b, r, c, steps))
    ws.fill_(0xff)   # whatever it held before (NaNs in every type)
    P.muon_orthogonalize(prec, b, r, c, dx, y, ws, steps, coeffs, eps)
    G.sync()
    return G.host(y).reshape(x.shape)


def _close(got, want, prec, tol, what=""):
    """Per matrix: relative Frobenius error, and every element."""
    half = 2.0 ** -8 if prec == G.BF16 else U
    for k in range(len(want)):
        g, w = got[k], want[k]
        assert np.isfinite(g).all(), (what, k)
        r = G.rel_l2(g, w)
        assert r <= tol, (what, k, r)
        rms = np.sqrt((w * w).mean())
        assert np.all(np.abs(g - w) <= 16 * tol * rms + half * np.abs(w) + 1e-30), (what, k, np.abs(g - w).max() / rms)


def _gauss(seed, b, r, c, scale=1e-3):
    return np.random.default_rng(seed).standard_normal((b, r, c)) * scale


def _gradient(seed, b, r, c):
    rng = np.random.default_rng(seed)
    k = min(4, r, c)
    return 1e-3 * ((rng.standard_normal((b, r, k)) * 0.6 ** np.arange(k)) @ rng.standard_normal((b, k, c))
                   + 0.5 * rng.standard_normal((b, r, c)))


PREC = pytest.mark.parametrize("prec", [G.BF16, G.FP32], ids=["bf16", "fp32"])
# one row, one column, one element; sides around the 16-, 64- and 128-wide tiles; the nets' kernels and dense layers;
# wide and tall; batches that change the tile
SHAPES = [(1, 1, 1), (3, 1, 40), (2, 40, 1), (2, 7, 5), (5, 36, 16), (4, 144, 16), (2, 16, 17), (1, 64, 64), (2, 65, 64),
          (2, 63, 130), (2, 576, 64), (1, 65, 65), (2, 128, 127), (2, 129, 200), (1, 300, 129), (1, 257, 256), (2, 100, 1000),
          (1, 1000, 100), (1, 512, 600), (200, 96, 130), (70, 200, 260), (70, 261, 200), (1, 3872, 256), (1, 33, 5000)]
# what one workgroup does by itself, at the edges of its tiles of 16, of its lanes and of its memory
SMALL = [(3, 2, 3), (2, 16, 16), (2, 15, 33), (3, 48, 49), (5, 288, 32), (2, 432, 27), (2, 320, 64), (2, 321, 64), (1, 64, 336),
         (64, 432, 64), (64, 64, 448), (64, 449, 64), (1, 2000, 16), (1, 8, 2100), (1, 2300, 16), (1, 1, 2048), (1, 2048, 1),
         (300, 9, 4)]


@PREC
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize(prec, shape):
    b = min(shape[0], 3)
    for k, make in enumerate((_gauss, _gradient)):
        x = G.q(make(k, *shape), prec)
        got = _orth(prec, x)
        pick = np.unique(np.linspace(0, shape[0] - 1, b).astype(int))
        # a square Gaussian matrix or a gradient with many small directions is not well conditioned
        tol = TYPICAL[prec] if max(shape[1:]) >= 4 * min(shape[1:]) and make is _gauss else WORST[prec]
        _close(got[pick], ns(x[pick]), prec, tol, make.__name__)


@PREC
@pytest.mark.parametrize("shape", SMALL, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_small(prec, shape):
    # One rounding to bf16 is off by 2^-8 of the value at most, and so is a matrix of roundings in norm;
    # half of that, which WORST has, is where the errors of many elements average.
    tol = 2.0 ** -8 + 2.0 ** -14 if prec == G.BF16 and shape[1] * shape[2] < 64 else WORST[prec]
    for k, make in enumerate((_gauss, _gradient)):
        x = G.q(make(k, *shape), prec)
        got = _orth(prec, x)
        pick = np.unique(np.linspace(0, shape[0] - 1, 3).astype(int))
        _close(got[pick], ns(x[pick]), prec, tol, make.__name__)


@PREC
def test_small_step_counts_and_coefficients(prec):
    co = np.array([[3.0, -3.2, 1.2], [1.5, -0.5, 0.0], [2.0, -1.5, 0.5]], np.float32)
    for shape in ((2, 70, 16), (2, 30, 200), (3, 50, 60)):
        x = G.q(_gradient(15, *shape), prec)
        for steps in (1, 2, 3, 8, 16):
            _close(_orth(prec, x, steps), ns(x, steps), prec, WORST[prec])
        _close(_orth(prec, x, 3, co), ns(x, 3, co), prec, WORST[prec])


@PREC
@pytest.mark.parametrize("shape", [(8, 1030, 1100), (9, 1100, 1030), (30, 1024, 516)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_more_tiles_than_compute_units(prec, shape):
    """Batches whose products fill the chip; the last matrix of each against the formula."""
    x = G.q(_gradient(14, *shape), prec)
    _close(_orth(prec, x)[-1:], ns(x[-1:]), prec, WORST[prec])


@PREC
def test_spread_singular_values_and_low_rank(prec):
    """Singular values from 1 to 1e-6 and to exactly 0: directions far below the matrix's rounding stay below 1.3."""
    rng = np.random.default_rng(3)
    for r, c in ((150, 90), (90, 150), (60, 300)):
        m = min(r, c)
        u, _ = np.linalg.qr(rng.standard_normal((r, m)))
        v, _ = np.linalg.qr(rng.standard_normal((c, m)))
        for s in (np.logspace(0, -6, m), np.r_[np.ones(5), np.zeros(m - 5)], np.r_[1.0, np.full(m - 1, 1e-3)]):
            x = G.q(((u * s) @ v.T)[None], prec)
            _close(_orth(prec, x), ns(x), prec, WORST[prec], (r, c, s[-1]))


@PREC
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 10, 11, 16])
def test_step_counts(prec, steps):
    """Every count around the segments' ends."""
    x = G.q(_gauss(4, 2, 150, 700), prec)
    _close(_orth(prec, x, steps), ns(x, steps), prec, WORST[prec])
    x = G.q(_gauss(5, 2, 300, 48), prec)
    _close(_orth(prec, x, steps), ns(x, steps), prec, WORST[prec])


@PREC
def test_coefficients_per_step(prec):
    """Other polynomials in every step; the cubic Newton-Schulz one (c = 0)."""
    x = G.q(_gauss(6, 2, 70, 400), prec)
    # a singular value of 0.53 becomes 1.3, then 1.9, 6.9 and 5900: refused
    with pytest.raises(P.LibraryError):
        _orth(prec, x, 4, [(3.9, -6.0, 2.9), (3.1, -4.0, 1.8), (2.5, -2.2, 0.7), (1.9, -1.3, 0.4)])
    for co in ([(3.4445, -4.775, 2.0315), (3.0, -3.2, 1.2), (2.5, -2.2, 0.7), (1.875, -1.25, 0.375)],
               [(1.5, -0.5, 0.0)] * 9, [(2.0, 0.0, 0.0)]):
        _close(_orth(prec, x, len(co), co), ns(x, len(co), co), prec, WORST[prec], co)


@PREC
def test_scale_of_the_input_does_not_matter(prec):
    """Norms from 1e-15 (eps 0) to 1e15; below eps the division is by eps."""
    x = G.q(_gauss(7, 1, 96, 200, 1.0), prec)
    want = ns(x)
    for s in (2.0 ** -50, 2.0 ** 50):
        _close(_orth(prec, x * s, eps=0.0), want, prec, WORST[prec], s)
    small = x * 2.0 ** -40
    got, want = _orth(prec, small, eps=1.0), ns(small, eps=1.0)
    assert G.rel_l2(got, want) <= WORST[prec]


@PREC
def test_zero_and_non_finite_matrices_stay_alone(prec):
    for r, c in ((144, 16), (100, 160)):
        x = G.q(_gauss(8, 5, r, c), prec)
        want = _orth(prec, x)
        x[1] = 0
        x[2, 3, 4] = np.nan
        x[3, r - 1, c - 1] = np.inf
        got = _orth(prec, x)
        assert not got[1].any() and np.isnan(got[2]).all() and np.isnan(got[3]).all()
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[4], want[4])


@PREC
def test_in_place_unaligned_and_repeated(prec):
    for r, c in ((144, 32), (130, 301)):
        x = G.q(_gauss(9, 2, r, c), prec)
        want = _orth(prec, x)
        assert np.array_equal(_orth(prec, x), want)
        assert np.array_equal(_orth(prec, x, inplace=True), want)
        for shift in (1, 2, 3):
            assert np.array_equal(_orth(prec, x, shift=shift), want)


def test_no_matrices():
    P.muon_orthogonalize(G.FP32, 0, 4, 4, None, None, None)
    G.sync()


# ------------------------------------------------------------------------------------------- the step


def _flat(seed, n):
    rng = np.random.default_rng(seed)
    f = lambda s: (rng.standard_normal(n) * s).astype(np.float32)  # noqa: E731
    return dict(p=f(0.1), g=f(1e-3), m=f(1e-3), v=np.abs(f(1e-6)))


CFG = dict(lr=0.02, momentum=0.95, weight_decay=0.1, adam_lr=2.5e-4, beta1=0.9, beta2=0.999, adam_eps=1e-5,
           max_grad_norm=0.5)


def _step_gpu(b, mats, step=3, n_calls=1, grads=None, **kw):
    n = b["p"].size
    d = {k: G.dev_f32(v) for k, v in b.items()}
    cfg = P.muon_cfg(**{**CFG, **kw})
    mm = P.muon_matrices(mats)
    st = G.dev_f32(np.full(2, -1.0))
    ws = G.ws_bytes(P.muon_workspace_bytes(n, mm, cfg))
    ws.fill_(0xff)
    for k in range(n_calls):
        if grads is not None:
            d["g"].copy_(G.dev_f32(grads[k]))
        P.muon_step(n, mm, cfg, d["p"], d["g"], d["m"], d["v"], step + k, st, ws)
    G.sync()
    return [G.host(d[k]) for k in ("p", "m", "v")] + [G.host(st)]


def _f32(v):
    return np.float64(np.float32(v))


def _step_want(b, mats, step=3, nesterov=True, scale=0, steps=5, **kw):
    """Formulas in float64, and a bound on each output's error."""
    c = {k: _f32(v) for k, v in {**CFG, **kw}.items()}
    p, g, m, v = (b[k].astype(np.float64) for k in ("p", "g", "m", "v"))
    norm = np.sqrt((g * g).sum())
    g = g * (c["max_grad_norm"] / norm if 0 < c["max_grad_norm"] < norm else 1.0)
    m2 = c["beta1"] * m + (1 - c["beta1"]) * g
    v2 = c["beta2"] * v + (1 - c["beta2"]) * g * g
    upd = c["adam_lr"] * (m2 / (1 - c["beta1"] ** step)) / (np.sqrt(v2 / (1 - c["beta2"] ** step)) + c["adam_eps"])
    p2 = p - upd
    tol_p = U * 4 * np.abs(p) + 2.0 ** -18 * np.abs(upd) + 2.0 ** -18 * c["adam_lr"] * np.abs(m) / c["adam_eps"] * 1e-3
    for off, r, k in mats:
        at = slice(off, off + r * k)
        m2[at] = c["momentum"] * m[at] + (1 - c["momentum"]) * g[at]
        u = c["momentum"] * m2[at] + (1 - c["momentum"]) * g[at] if nesterov else m2[at]
        O = ns(u.reshape(r, k), steps).reshape(-1)
        s = np.sqrt(max(1.0, k / r)) if scale == 0 else 0.2 * np.sqrt(max(r, k))
        p2[at] = p[at] * (1 - c["lr"] * c["weight_decay"]) - c["lr"] * s * O
        v2[at] = v[at]
        rms = np.sqrt((O * O).mean())
        tol_p[at] = U * 4 * np.abs(p[at]) + c["lr"] * s * (16 * WORST[G.FP32] * rms + 4 * U * np.abs(O))
    tol_m = 8 * U * (np.abs(m) + np.abs(g))
    return p2, m2, v2, norm, tol_p, tol_m


def _check_step(b, mats, **kw):
    p, m, v, st = _step_gpu(b, mats, **kw)
    wp, wm, wv, norm, tp, tm = _step_want(b, mats, **kw)
    assert np.all(np.abs(m - wm) <= tm), np.abs(m - wm).max()
    assert np.all(np.abs(v - wv) <= 8 * U * (b["v"] + wv)), np.abs(v - wv).max()
    bad = np.abs(p - wp) > tp
    assert not bad.any(), (int(bad.sum()), np.flatnonzero(bad)[:5], (np.abs(p - wp) / tp).max())
    assert abs(st[0] - norm) <= 2 * U * norm and st[1] == 0
    covered = np.zeros(b["p"].size, bool)
    for off, r, c in mats:
        covered[off:off + r * c] = True
    assert np.array_equal(v[covered], b["v"][covered].astype(np.float64))


# offsets that are no multiple of four, gaps of one element and of none, wide and tall, a single row and column
MATS = [(3, 36, 16), (3 + 576, 17, 9), (733, 1, 50), (800, 50, 1), (851, 70, 130), (10001, 260, 100), (36001, 36, 16)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", [0, 1])
def test_step(nesterov, scale):
    _check_step(_flat(1, 40003), MATS, nesterov=nesterov, scale=scale)


def test_step_without_clip_decay_or_momentum():
    _check_step(_flat(2, 40003), MATS, max_grad_norm=0.0, weight_decay=0.0, momentum=0.0)
    _check_step(_flat(3, 40003), MATS, max_grad_norm=1e9, steps=3)


def test_step_on_no_matrices_is_adam():
    """Everything left to Adam: adam_step's results within the two sums' order."""
    b = _flat(4, 10007)
    _check_step(b, [])
    _check_step(_flat(5, 3), [])


def test_step_on_matrices_alone():
    _check_step(_flat(6, 144 * 16 + 300 * 100), [(144 * 16, 300, 100), (0, 144, 16)])


def test_step_with_more_shapes_and_matrices_than_one_pass():
    """150 matrices of 20 shapes, given in another order than they lie."""
    rng = np.random.default_rng(7)
    shapes = [(int(rng.integers(1, 90)), int(rng.integers(1, 90))) for _ in range(20)]
    mats, at = [], 5
    for k in range(150):
        r, c = shapes[k % 20] if k < 100 else shapes[0]
        mats.append((at, r, c))
        at += r * c + int(rng.integers(0, 3)) * int(rng.integers(0, 40))
    order = rng.permutation(len(mats))
    _check_step(_flat(8, at + 11), [mats[i] for i in order])


def test_opposed_gradient_and_momentum():
    """u is all but cancelled by the momentum: what is left is rounding, and the update stays bounded."""
    b = _flat(9, 100 * 80)
    b["g"] = (-(0.95 ** 2) / (0.05 * 1.95) * b["m"].astype(np.float64)).astype(np.float32)
    p, m, _, st = _step_gpu(b, [(0, 100, 80)], max_grad_norm=0.0)
    assert np.isfinite(p).all() and st[1] == 0
    # an orthogonalised matrix has singular values below 1.3: entries too
    assert np.abs(p - b["p"].astype(np.float64) * (1 - _f32(0.02) * _f32(0.1))).max() <= 0.02 * 1.3 + 1e-6


def test_non_finite_gradient_is_flagged_and_stays_in_its_matrix_without_the_clip():
    b = _flat(10, 40003)
    clean = _step_gpu(b, MATS, max_grad_norm=0.0)
    off, r, c = MATS[4]
    b["g"][off + 77] = np.inf
    p, m, v, st = _step_gpu(b, MATS, max_grad_norm=0.0)
    assert st[1] == 1
    assert np.isnan(p[off:off + r * c]).all()
    keep = np.ones(b["p"].size, bool)
    keep[off:off + r * c] = False
    assert np.array_equal(p[keep], clean[0][keep]) and np.array_equal(m[keep], clean[1][keep])


def test_several_steps_follow_the_formulas():
    rng = np.random.default_rng(11)
    b = _flat(11, 40003)
    grads = [(rng.standard_normal(40003) * 1e-3).astype(np.float32) for _ in range(4)]
    p, m, v, _ = _step_gpu(b, MATS, step=1, n_calls=4, grads=grads)
    w = dict(b)
    tol = 0
    for k, g in enumerate(grads):
        wp, wm, wv, _, tp, _ = _step_want({**w, "g": g}, MATS, step=1 + k)
        tol = tol + tp
        w = dict(p=wp, m=wm, v=wv)
    assert np.all(np.abs(m - w["m"]) <= 64 * U * (np.abs(w["m"]) + 1e-3))
    # a difference of the momentum by its rounding passes through the iteration's slope (at most a^5 = 485)
    assert G.rel_l2(p - b["p"], w["p"] - b["p"]) <= 4 * WORST[G.FP32]
    assert np.all(np.abs(p - w["p"]) <= 16 * tol)


def test_captured_and_replayed():
    """A captured step replayed on new gradients equals the eager one bit for bit, with eager steps in other workspaces
    between the replays; two graphs on one workspace run in turn."""
    t = G.torch()
    b = _flat(12, 40003)
    n = 40003
    cfg, mm = P.muon_cfg(**CFG), P.muon_matrices(MATS)
    d = {k: G.dev_f32(v) for k, v in b.items()}
    e = {k: G.dev_f32(v) for k, v in b.items()}
    st, est = G.dev_f32(np.zeros(2)), G.dev_f32(np.zeros(2))
    ws, ews = (G.ws_bytes(P.muon_workspace_bytes(n, mm, cfg)) for _ in range(2))
    x = t.empty((2, 130, 70), device="cuda:0")
    y, ey = t.empty_like(x), t.empty_like(x)
    xws = G.ws_bytes(P.muon_orthogonalize_workspace_bytes(G.FP32, 2, 130, 70, 5))

    def run(q, s, w, out):
        P.muon_step(n, mm, cfg, q["p"], q["g"], q["m"], q["v"], 5, s, w)
        P.muon_orthogonalize(G.FP32, 2, 130, 70, x, out, xws)

    x.normal_()
    side = t.cuda.Stream()
    with t.cuda.stream(side):
        run(e, est, ews, ey)
    side.synchronize()
    e = {k: G.dev_f32(v) for k, v in b.items()}
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        run(d, st, ws, y)
    for k in range(3):
        g = t.randn(n, device="cuda:0") * 1e-3
        d["g"].copy_(g)
        e["g"].copy_(g)
        x.normal_()
        run(e, est, ews, ey)
        G.sync()
        graph.replay()
        G.sync()
        assert all(t.equal(d[q], e[q]) for q in ("p", "m", "v")) and t.equal(st, est) and t.equal(y, ey), k


# ------------------------------------------------------------------------------------------- in the learner


@pytest.mark.parametrize("prec", [G.BF16, G.FP32], ids=["bf16", "fp32"])
def test_learner_step_with_muon_equals_its_abi_calls(prec):
    """learner_step (PPO, optimizer muon) is GAE, then per minibatch forward, loss, backward and muon_step on
    muon_net_matrices, bit for bit; in bf16 the next forward reads the dense weights as the step left them."""
    from tests.test_gpu_network import _c1_like_inputs, _gpu_rollout, _learner_gpu
    torch = G.torch()
    wl, params, ro, perm = _c1_like_inputs(wid=0)
    wl = wl.replace(epochs=2, num_minibatches=1, optimizer="muon")
    perm = np.concatenate([perm, perm[:, ::-1]])
    net = wl.net
    got = _learner_gpu(wl, prec, params, ro, perm)
    d = _gpu_rollout(ro, wl)
    T, E, A, mb = wl.T, wl.E, net.num_actions, wl.mb
    adv = torch.empty((T, E), dtype=torch.float32, device="cuda:0")
    ret = torch.empty_like(adv)
    P.gae_advantages(T, E, d["rewards"], d["values"], d["dones"], d["next_value"], d["next_done"], wl.gamma, wl.lam, adv,
                     ret)
    p = G.dev_f32(params)
    m, v, grads = torch.zeros_like(p), torch.zeros_like(p), torch.empty_like(p)
    mats = P.muon_net_matrices(net)
    cfg = P.muon_cfg(lr=0.02, adam_lr=wl.lr, beta1=wl.beta1, beta2=wl.beta2, adam_eps=wl.adam_eps,
                     max_grad_norm=wl.max_grad_norm)
    ws = G.ws_bytes(P.impala_workspace_bytes(net, mb, prec, 1))
    mws = G.ws_bytes(P.muon_workspace_bytes(p.numel(), mats, cfg))
    logits = torch.empty((mb, A), dtype=torch.float32, device="cuda:0")
    value = torch.empty(mb, dtype=torch.float32, device="cuda:0")
    dz, dv = torch.empty_like(logits), torch.empty_like(value)
    stats = torch.zeros((wl.n_updates, 8), dtype=torch.float32, device="cuda:0")
    dperm = G.dev_i32(perm)
    for u in range(2):
        rows = dperm[u].contiguous()
        P.impala_cnn_fwd(net, prec, p, d["obs"], rows, mb, ws, 1, logits, value)
        rl = rows.long()
        P.ppo_loss_grad(mb, A, logits, value, d["actions"][rl].contiguous(), d["logp"][rl].contiguous(),
                        adv.view(-1)[rl].contiguous(), ret.view(-1)[rl].contiguous(), 1, wl.clip_eps, wl.vf_coef,
                        wl.ent_coef, dz, dv, stats[u])
        P.impala_cnn_bwd(net, prec, p, d["obs"], rows, mb, ws, dz, dv, grads)
        P.muon_step(p.numel(), mats, cfg, p, grads, m, v, u + 1, stats[u, 6:], mws)
    G.sync()
    assert torch.equal(got[0], p) and torch.equal(got[1], m) and torch.equal(got[2], v)
    assert torch.equal(got[4], stats) and got[3] == 2
    assert not torch.equal(p, G.dev_f32(params))


def test_normalised_conv_trained_with_orthogonalised_updates():
    """The operators as they are used together: conv, group norm + relu, conv backward, and the step on its kernel. The
    gradients of kernel, scale and shift against the chain rule in 64 bits on the same stored activations, and the step
    on them; a kernel in front of a group norm is scale-invariant, so its gradient is orthogonal to it."""
    torch = G.torch()
    n, H, W, C, groups = 3, 9, 8, 16, 4
    rng = np.random.default_rng(13)
    x = rng.standard_normal((n, H, W, C)).astype(np.float32)
    w = (rng.standard_normal((3, 3, C, C)) * (2 / (9 * C)) ** 0.5).astype(np.float32)
    gamma = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    beta = (0.2 * rng.standard_normal(C)).astype(np.float32)
    dy = rng.standard_normal((n, H, W, C)).astype(np.float32)
    flat = G.dev_f32(np.concatenate([w.ravel(), np.zeros(C, np.float32), gamma, beta]))
    N = 9 * C * C
    wv, bias, ga, be = flat[:N], flat[N:N + C], flat[N + C:N + 2 * C], flat[N + 2 * C:]
    grads = torch.zeros_like(flat)
    dw, db, dga, dbe = grads[:N], grads[N:N + C], grads[N + C:N + 2 * C], grads[N + 2 * C:]
    dx_, t_, y_, dt_ = (torch.empty((n, H, W, C), device="cuda:0") for _ in range(4))
    xd = G.dev_f32(x)
    mean, rstd = (torch.empty((n, groups), device="cuda:0") for _ in range(2))
    P.impala_conv3x3_fwd(G.FP32, n, H, W, C, C, xd, P.X_PLAIN, None, wv, bias, None, t_)
    fws = G.ws_bytes(P.impala_groupnorm_fwd_workspace_bytes(G.FP32, n, H, W, C, groups))
    P.impala_groupnorm_fwd(G.FP32, n, H, W, C, groups, t_, ga, be, 1e-5, P.ACT_RELU, y_, mean, rstd, fws)
    bws = G.ws_bytes(P.impala_groupnorm_bwd_workspace_bytes(G.FP32, n, H, W, C, groups))
    P.impala_groupnorm_bwd(G.FP32, n, H, W, C, groups, G.dev_f32(dy), t_, ga, be, mean, rstd, P.ACT_RELU, dt_, dga, dbe, bws)
    wws = G.ws_bytes(P.impala_conv3x3_wgrad_workspace_bytes(G.FP32, H, W, C, C))
    P.impala_conv3x3_wgrad(G.FP32, n, H, W, C, C, xd, P.X_PLAIN, None, dt_, dw, db, wws)
    g0 = G.host(grads)
    p0 = G.host(flat)
    mats, cfg = P.muon_matrices([(0, 9 * C, C)]), P.muon_cfg(**CFG)
    m, v = torch.zeros_like(flat), torch.zeros_like(flat)
    st = torch.zeros(2, device="cuda:0")
    ws = G.ws_bytes(P.muon_workspace_bytes(flat.numel(), mats, cfg))
    P.muon_step(flat.numel(), mats, cfg, flat, grads, m, v, 1, st, ws)
    G.sync()
    # the chain rule in 64 bits (autograd on the CPU)
    tw, tg, tb = (torch.from_numpy(a.astype(np.float64)).requires_grad_() for a in (w, gamma, beta))
    tx = torch.from_numpy(x.astype(np.float64))
    z = torch.nn.functional.conv2d(tx.permute(0, 3, 1, 2), tw.permute(3, 2, 0, 1), padding=1)
    zz = z.reshape(n, groups, -1)
    mu = zz.mean(2, keepdim=True)
    xh = ((zz - mu) / torch.sqrt(((zz - mu) ** 2).mean(2, keepdim=True) + 1e-5)).reshape(z.shape)
    out = torch.relu(xh * tg[:, None, None] + tb[:, None, None])
    (out * torch.from_numpy(dy.astype(np.float64)).permute(0, 3, 1, 2)).sum().backward()
    # relu decisions of activations next to zero may differ by the convolution's rounding: none is that near here
    pre = (xh * tg[:, None, None] + tb[:, None, None]).detach().numpy()
    assert np.abs(pre).min() > 1e-6
    want = np.concatenate([tw.grad.numpy().ravel(), np.zeros(C), tg.grad.numpy(), tb.grad.numpy()])
    keep = np.r_[0:N, N + C:N + 3 * C]   # (a bias in front of a group norm is not quite without effect)
    assert G.rel_l2(g0[keep], want[keep]) <= 1e-5
    assert abs((g0[:N] * p0[:N]).sum()) <= 1e-4 * np.linalg.norm(g0[:N]) * np.linalg.norm(p0[:N])
    b = dict(p=p0.astype(np.float32), g=g0.astype(np.float32), m=np.zeros(p0.size, np.float32),
             v=np.zeros(p0.size, np.float32))
    wp, _, _, _, tp, _ = _step_want(b, [(0, 9 * C, C)], step=1)
    assert np.all(np.abs(G.host(flat)[:N] - wp[:N]) <= tp[:N])


@PREC
def test_orthogonalize_captured_and_beside_another_stream(prec):
    """Calls of every form on two streams at once, each with its own workspace, and the same captured into one
    graph and replayed on new inputs with eager work between: the eager results, bit for bit."""
    t = G.torch()
    shapes = [(4, 144, 16), (3, 576, 64), (1, 300, 520), (1, 1100, 1200)]
    xs = [[G.dev_act(G.q(_gauss(20 + r, *s), prec), prec) for s in shapes] for r in range(3)]
    want = [[t.empty_like(x) for x in v] for v in xs]
    ws = [[G.ws_bytes(P.muon_orthogonalize_workspace_bytes(prec, *s)) for s in shapes] for _ in range(2)]

    def run(inputs, outputs, k):
        for s, x, y, w in zip(shapes, inputs, outputs, ws[k]):
            P.muon_orthogonalize(prec, *s, x, y, w)

    for v, w in zip(xs, want):
        run(v, w, 0)
    G.sync()
    got = [[t.empty_like(x) for x in v] for v in xs]
    streams = [t.cuda.Stream() for _ in range(2)]
    for st in streams:
        st.wait_stream(t.cuda.current_stream())
    for k, st in enumerate(streams):
        with t.cuda.stream(st):
            run(xs[k], got[k], k)
            run(xs[k], got[k], k)
    G.sync()
    for k in range(2):
        assert all(t.equal(a, b) for a, b in zip(got[k], want[k]))
    held = [x.clone() for x in xs[0]]
    with t.cuda.stream(streams[0]):
        run(held, got[2], 0)
    G.sync()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        run(held, got[2], 0)
    for r in (1, 2, 0):
        for h, x in zip(held, xs[r]):
            h.copy_(x)
        graph.replay()
        run(xs[r], got[1], 1)
        G.sync()
        assert all(t.equal(a, b) for a, b in zip(got[2], want[r])) and all(t.equal(a, b) for a, b in zip(got[1], want[r]))
