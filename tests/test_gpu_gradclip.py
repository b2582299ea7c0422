"""The clip over many gradient tensors against sums in 64 bits: types, odd sizes and offsets, in place and gathered, the
norm alone, several launches, what is not finite."""
import math

import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, F = torch.bfloat16, torch.float32


def run(pairs, limit):
    t = P.grad_tensors(pairs)
    ws = torch.empty(P.grad_clip_workspace_bytes(t), dtype=torch.uint8, device=DEV)
    stats = torch.full((2,), 7.0, device=DEV)
    P.grad_clip(t, limit, stats, ws)
    return stats.cpu().tolist()


def norm_of(srcs):
    return math.sqrt(math.fsum(float(s.double().square().sum()) for s in srcs))


def tensors(sizes, types, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 0.1).to(types[i % len(types)]).to(DEV) for i, n in enumerate(sizes)]


def check(srcs, dsts, limit, stats):
    """The norm is a 64-bit sum rounded once; a value is rounded by the factor, the product and its type."""
    n = norm_of([s.cpu() for s in srcs])
    assert abs(stats[0] - n) <= 2.0 ** -23 * n and stats[1] == 0
    for s, d in zip(srcs, dsts):
        if limit > 0 and n > limit:
            want = s.double() * (limit / n)
            assert ((d.double() - want).abs() <= (2.0 ** -8 if d.dtype == B else 2.0 ** -23) * want.abs() + 1e-38).all()
        else:
            assert torch.equal(d, s.to(d.dtype))


SIZES = [1, 0, 7, 8, 9, 2047, 2048, 8191, 8192, 8193, 100000, 3, 16384, 1, 65537]


@pytest.mark.parametrize("limit", [0.5, 1e6, 0.0, -1.0])
@pytest.mark.parametrize("src,dst", [((F,), F), ((B,), B), ((B, F), F), ((F, B), B)])
def test_sizes_and_types(src, dst, limit):
    srcs = tensors(SIZES, src)
    dsts = [torch.full((s.numel(),), 9.0, dtype=dst, device=DEV) for s in srcs]
    check(srcs, dsts, limit, run(zip(srcs, dsts), limit))


@pytest.mark.parametrize("count", [1, 95, 96, 97, 300, 1000])
def test_many_tensors_into_one_buffer(count):
    """Odd sizes one behind the other, so that most start off any alignment; a guard behind the last."""
    g = torch.Generator().manual_seed(count)
    sizes = [int(n) for n in torch.randint(0, 3000, (count,), generator=g)]
    srcs = tensors(sizes, (B, F, F), seed=count)
    flat = torch.full((sum(sizes) + 8,), 9.0, device=DEV)
    dsts = list(flat[:sum(sizes)].split(sizes))
    check(srcs, dsts, 0.5, run(zip(srcs, dsts), 0.5))
    assert (flat[sum(sizes):] == 9).all()


def test_in_place_and_norm_only():
    for limit in (0.5, 1e6):
        srcs = tensors(SIZES, (B, F))
        keep = [s.clone() for s in srcs]
        check(keep, srcs, limit, run(zip(srcs, srcs), limit))
        srcs = [s.clone() for s in keep]
        # every other tensor only counts
        stats = run([(s, s if i % 2 else None) for i, s in enumerate(srcs)], limit)
        check(keep[1::2] + keep[::2], srcs[1::2] + [s.clone() if limit > 100 else (s.double() * (0.5 / norm_of(keep))).to(s.dtype)
                                                   for s in keep[::2]], limit, stats)
        assert all(torch.equal(a, b) for a, b in zip(srcs[::2], keep[::2]))


def test_odd_offsets():
    for ty in (B, F):
        for off in range(1, 9):
            base = tensors([5000], (ty,), seed=off)[0]
            out = torch.full((5000,), 9.0, dtype=ty, device=DEV)
            s, d = base[off:off + 4100], out[9 - off:9 - off + 4100]
            check([s], [d], 0.5, run([(s, d)], 0.5))
            assert (out[:9 - off] == 9).all() and (out[9 - off + 4100:] == 9).all()


def test_empty_calls():
    assert run([], 0.5) == [0.0, 0.0]
    e = torch.empty(0, device=DEV)
    assert run([(e, e), (e, None)], 0.5) == [0.0, 0.0]


def test_the_same_source_twice_counts_twice():
    s = tensors([3000], (F,))[0]
    d = [torch.empty_like(s) for _ in range(2)]
    check([s, s], d, 0.5, run([(s, d[0]), (s, d[1])], 0.5))


def test_not_finite():
    """As adam_step's clip: a norm of NaN clips nothing, an infinite one scales by zero."""
    a, b = tensors([100, 9000], (F,))
    da, db = torch.empty_like(a), torch.empty_like(b)
    a[3] = float("nan")
    stats = run([(a, da), (b, db)], 0.5)
    assert math.isnan(stats[0]) and stats[1] == 1 and torch.equal(db, b)
    a[3] = float("inf")
    stats = run([(a, da), (b, db)], 0.5)
    assert stats == [math.inf, 1] and (db == 0).all() and da[3].isnan()
    a[3] = 3e38   # its square overflows 32 bits
    stats = run([(a, da), (b, db)], 0.5)
    assert stats[1] == 0 and abs(stats[0] / 3e38 - 1) < 1e-6


def test_the_clip_then_adam_without_one_is_adam_with_one():
    """On one float32 buffer, the norm and the factor being the same to a rounding: results to a few of them."""
    n = 50001
    g = torch.Generator().manual_seed(2)
    p, gr, m = (torch.randn(n, generator=g).to(DEV) for _ in range(3))
    v = m.square()
    cfg = (5, 1e-3, 0.9, 0.999, 1e-5)
    ws = torch.empty(P.adam_workspace_bytes(n), dtype=torch.uint8, device=DEV)
    st = torch.empty(2, device=DEV)
    want = [t.clone() for t in (p, m, v)]
    P.adam_step(n, want[0], gr, want[1], want[2], *cfg, 0.5, st, ws)
    flat = torch.empty_like(gr)
    cut = [1, 17, 4000, 30000]
    parts = torch.tensor_split(gr, cut)
    stats = run([(s.clone(), d) for s, d in zip(parts, torch.tensor_split(flat, cut))], 0.5)
    P.adam_step(n, p, flat, m, v, *cfg, 0.0, None, ws)
    assert stats[0] == pytest.approx(float(st[0]), rel=2.0 ** -22)
    for a, b in zip((p, m, v), want):
        assert ((a - b).abs() <= 2.0 ** -21 * b.abs() + 1e-9).all()


def test_streams_graphs_and_repeats():
    sets = [tensors(SIZES, (B, F), seed=i) for i in range(2)]
    outs = [[torch.empty(s.numel(), device=DEV) for s in x] for x in sets]
    want = []
    for x, y in zip(sets, outs):
        st = run(zip(x, y), 0.5)
        want.append((st, [t.clone() for t in y]))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    tabs = [P.grad_tensors(zip(x, y)) for x, y in zip(sets, outs)]
    wss = [torch.empty(P.grad_clip_workspace_bytes(t), dtype=torch.uint8, device=DEV) for t in tabs]
    sts = [torch.empty(2, device=DEV) for _ in tabs]
    torch.cuda.synchronize()
    for _ in range(3):
        for t, w, s, stream in zip(tabs, wss, sts, streams):
            P.grad_clip(t, 0.5, s, w, stream=stream)
        torch.cuda.synchronize()
        for (st, w), s, y in zip(want, sts, outs):
            assert s.cpu().tolist() == st and all(torch.equal(a, b) for a, b in zip(w, y))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        P.grad_clip(tabs[0], 0.5, sts[0], wss[0])
    orig = [t.clone() for t in sets[0]]
    for k in (1.0, 3.0, 1.0):
        for t, o in zip(sets[0], orig):
            t.copy_(o * k)
        graph.replay()
        eager = [torch.empty_like(t) for t in outs[0]]
        st = run(zip(sets[0], eager), 0.5)
        torch.cuda.synchronize()
        assert sts[0].cpu().tolist() == st and all(torch.equal(a, b) for a, b in zip(outs[0], eager))


def test_a_tensor_of_more_than_2_31_elements():
    """Zeros with a few numbers about the border and at the end, in place; sources of it by parts give the same norm."""
    n = 2 ** 31 + 70001
    t = torch.zeros(n, dtype=B, device=DEV)
    at = torch.tensor([0, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 1, n - 2, n - 1], device=DEV)
    t[at] = torch.tensor([3.0, 4.0, 12.0, 84.0, 5.0, 12.0], dtype=B, device=DEV)
    whole = math.sqrt(9 + 16 + 144 + 7056 + 25 + 144)
    stats = run([(t[:2 ** 30], None), (t[2 ** 30:], None)], 1.0)
    assert stats[0] == pytest.approx(whole, rel=2.0 ** -23)
    stats = run([(t, t)], whole / 2)
    assert stats[0] == pytest.approx(whole, rel=2.0 ** -23) and stats[1] == 0
    assert t[at].tolist() == [1.5, 2.0, 6.0, 42.0, 2.5, 6.0] and int((t != 0).sum()) == 6
