"""The binding's checks of the memory core's tensors against the shape structs: on the host, before any HIP call."""
import pytest
import torch

P = pytest.importorskip("paper_2310_00036_amd")
B, F = torch.bfloat16, torch.float32


class Stream:
    cuda_stream = None


def la(T=4, E=3, H=2, dk=16, dv=8):
    """A forward's arguments by name, as CPU tensors."""
    q, v = torch.zeros(T, E, H, dk, dtype=B), torch.zeros(T, E, H, dv, dtype=B)
    return dict(q=q, k=q.clone(), v=v, log_decay=torch.zeros(H), dones=torch.zeros(T, E, dtype=torch.uint8),
                s0=torch.zeros(E, H, dk, dv), o=v.clone(), s_out=torch.zeros(E, H, dk, dv))


def la_calls(x):
    f = P.linattn_shape(x["q"], x["k"], x["v"], x["o"], x["dones"], 1.0)
    b = P.linattn_shape(x["q"], x["k"], x["v"], x["o"], x["dones"], 1.0, x["q"], x["k"], x["v"])
    return {"fwd": lambda y: P.impala_linattn_fwd(f, y["q"], y["k"], y["v"], y["log_decay"], y["dones"], y["s0"], y["o"],
                                                  y["s_out"], None, Stream),
            "step": lambda y: P.impala_linattn_step(f, y["q"], y["k"], y["v"], y["log_decay"], y["dones"], y["s0"], y["o"],
                                                    y["s_out"], Stream),
            "bwd": lambda y: P.impala_linattn_bwd(b, y["o"], y["q"], y["k"], y["v"], y["log_decay"], y["dones"], y["s0"],
                                                  y["s_out"], y["q"], y["k"], y["v"], y["s0"], None, Stream)}


def wide(t):
    """t's values in wider rows."""
    return torch.cat([t, t], -1)[..., :t.shape[-1]]


def refused(call, args, words):
    with pytest.raises(ValueError, match=words):
        call(args)


@pytest.mark.parametrize("which", ["fwd", "step", "bwd"])
def test_linattn(which):
    """A tensor of another size, type or stride than the struct's, and of another device, is refused by name. (Here every
    tensor is on the CPU, so a call whose tensors agree with the struct is refused for that, at its first one.)"""
    x = la()
    call = la_calls(x)[which]
    refused(call, x, "(q|d_o) has to be .*cpu")
    names = dict(q="q", k="k", v="v", o="d_o" if which == "bwd" else "o", log_decay="log_decay", dones="dones",
                 s0="s_in" if which == "step" else "s0", s_out="ds_out" if which == "bwd" else "s_out")
    for k, name in names.items():
        t = x[k]
        others = {j: 4096 for j in x}   # plain addresses pass
        bad = [t[:1].clone() if t.shape[0] > 1 else None, t.double(), t.to(F) if t.dtype is B else t.to(torch.int8), t[:0]]
        bad.append(torch.stack([t, t], -1)[..., 0])                     # its last axis is not contiguous
        if t.dtype in (B, torch.uint8):
            bad += [wide(t), t.transpose(0, 1).contiguous().transpose(0, 1)]
        for y in bad:
            if y is not None:
                refused(call, {**others, k: y}, f"{name} has to be")
        refused(call, {**others, k: t}, f"{name} has to be .*cpu")


def test_the_struct_counts_as_it_is_at_the_call():
    x = la()
    s = P.linattn_shape(x["q"], x["k"], x["v"], x["o"], x["dones"], 1.0)
    args = [4096] * 8
    for field, value in (("T", 5), ("E", 2), ("heads", 3), ("dk", 17), ("prec", P.PREC_FP32)):
        s2 = P.linattn_shape(x["q"], x["k"], x["v"], x["o"], x["dones"], 1.0)
        for change in (False, True):
            if change:
                setattr(s2, field, value)
            with pytest.raises(ValueError, match=r"\(4, 3, 2, 16\) of torch.bfloat16" if not change else "q has to be (?!.4, 3, 2, 16. of torch.bf)"):
                P.impala_linattn_fwd(s2, x["q"], *args[1:], stream=Stream)
        assert s2.expected() != s.expected()
    with pytest.raises(ValueError, match="dones"):   # a struct without episode starts
        s2 = P.linattn_shape(x["q"], x["k"], x["v"], x["o"], None, 1.0)
        P.impala_linattn_fwd(s2, *args[:4], x["dones"], *args[5:], stream=Stream)


def steps_as(t, size, strides):
    return P._lib._steps_as(t, size, strides)


def test_equal_steps():
    t = torch.zeros(4, 3, 8)
    assert steps_as(t, (12, 8), (8, 1)) and steps_as(t.reshape(-1), (12, 8), (8, 1)) and steps_as(t, (4, 3, 8), (24, 8, 1))
    assert not steps_as(t, (12, 8), (9, 1)) and not steps_as(t, (11, 8), (8, 1)) and not steps_as(t[:, :2], (8, 8), (8, 1))
    assert steps_as(t[:, :, :5], (12, 5), (8, 1)) and not steps_as(t.transpose(0, 1), (12, 8), (8, 1))
    assert steps_as(t[:1], (1, 3, 8), (999, 8, 1)) and steps_as(t[:0], (0, 8), (5, 1)) and not steps_as(t[:0], (1, 8), (8, 1))
    assert steps_as(t[:, :1].expand(4, 3, 8), (4, 3, 8), (24, 0, 1)) and not steps_as(t[:, :1].expand(4, 3, 8), (12, 8), (8, 1))
    assert steps_as(torch.zeros(()), (1, 1), (7, 7))


def test_blocknorm():
    n, c = 6, 64
    rows, vec = torch.zeros(n, c, dtype=B), torch.zeros(c)
    s = P.blocknorm_shape(P.PREC_BF16, n, c, ld_gate=80, ld_dgate=80)
    fwd = ("h", "gamma", "beta", "gate", "rscale", "res", "out", "gamma2", "beta2", "out2")
    bwd = ("dout", "dout2", "h", "gamma", "beta", "gate", "rscale", "out", "gamma2", "dh", "dgamma", "dbeta", "dgate", "drscale",
           "dres", "dgamma2", "dbeta2")
    for call, names in ((P.impala_blocknorm_fwd, fwd), (P.impala_blocknorm_bwd, bwd)):
        for k in names:
            is_row = k.lstrip("d") in ("h", "gate", "res", "out", "out2") and "gamma" not in k
            good = rows if is_row else vec
            if k in ("gate", "dgate"):
                good = torch.zeros(n, 80, dtype=B)[:, :c]
            bad = [good[1:], good.double(), good[..., :c - 1], torch.stack([good, good], -1)[..., 0]]
            bad += [good.float(), rows if k in ("gate", "dgate") else wide(good)] if is_row else [good.to(B)]
            for y, words in [(y, f"{k} has to be") for y in bad] + [(good, f"{k} has to be .*cpu")]:
                a = {j: 4096 for j in names}
                a[k] = y
                if call is P.impala_blocknorm_bwd:
                    a["ws"] = 4096
                with pytest.raises(ValueError, match=words):
                    call(s, **a, stream=Stream)
    with pytest.raises(ValueError, match="ws has to be"):
        P.impala_blocknorm_bwd(s, *[4096] * len(bwd), torch.zeros(100), stream=Stream)


def test_grad_clip():
    t = P.grad_tensors([(torch.zeros(3), None), (torch.zeros(0), torch.zeros(0, dtype=B))])
    with pytest.raises(ValueError, match="on one GPU"):
        P.grad_clip(t, 0.5, 4096, None, stream=Stream)
    t = P.grad_tensors([])
    for stats in (torch.zeros(1), torch.zeros(2, dtype=B), torch.zeros(2, 2).t(), torch.zeros(2)):
        with pytest.raises(ValueError, match="stats has to be"):
            P.grad_clip(t, 0.5, stats, None, stream=Stream)
    with pytest.raises(ValueError, match="ws has to be"):
        P.grad_clip(t, 0.5, None, torch.zeros(8), stream=Stream)
