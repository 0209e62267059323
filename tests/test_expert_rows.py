"""Rows of an expert layer: slots sorted by expert, rows laid out in that order, the weighted sum back per token, and their
gradients, against plain implementations in 64 bits."""
import ctypes as C

import numpy as np
import pytest

import expert_plain as P

gpu = pytest.mark.gpu
BF16_HALF, FP32_HALF = 2.0 ** -8, 2.0 ** -24           # half a step, relative to the value


# ---- refusals: nothing of these calls reaches the device ------------------------------------------------------------
def refused(name, *args):
    from paper_2405_10951_b200 import binding as Bd
    rc = getattr(Bd.lib(), name)(*args)
    assert rc == -1, (name, rc)
    assert len(Bd.lib().bsr_last_error(None)) > 0


A, O = 4096, 4098            # an aligned and an unaligned address: never read, the arguments are checked first


def test_refusals():
    for bad in [dict(tokens=-1), dict(top_k=0), dict(experts=0), dict(experts=1025), dict(tokens=1 << 29, top_k=3), dict(expert=None), dict(pos=None), dict(seg=None)]:
        a = dict(expert=A, tokens=4, top_k=2, experts=8, pos=A, seg=A) | bad
        refused("bsr_expert_sort", a["expert"], a["tokens"], a["top_k"], a["experts"], a["pos"], a["seg"], None)
    for bad in [dict(dtype=2), dict(tokens=-1), dict(top_k=0), dict(dim=0), dict(dim=12), dict(x=None), dict(x=O), dict(pos=None), dict(rows=O), dict(tokens=1 << 30, top_k=2)]:
        a = dict(x=A, dtype=1, tokens=4, dim=16, top_k=2, pos=A, rows=A) | bad
        refused("bsr_expert_scatter", a["x"], a["dtype"], a["tokens"], a["dim"], a["top_k"], a["pos"], a["rows"], None)
        refused("bsr_expert_scatter_e4m3", a["x"], a["dtype"], a["tokens"], a["dim"], a["top_k"], a["pos"], a["rows"], A, None)
    refused("bsr_expert_scatter_e4m3", A, 1, 4, 24, 2, A, A, A, None)          # whole 16-byte units of codes
    refused("bsr_expert_scatter_e4m3", A, 1, 4, 16, 2, A, A, O, None)
    for bad in [dict(rdt=3), dict(dt=-1), dict(dim=4), dict(rows=None), dict(rows=O), dict(out=O), dict(res=O), dict(pos=None), dict(tokens=-2)]:
        a = dict(rows=A, rdt=1, pos=A, w=A, res=A, out=A, dt=0, tokens=4, dim=8, top_k=2) | bad
        refused("bsr_expert_combine", a["rows"], a["rdt"], a["pos"], a["w"], a["res"], a["out"], a["dt"], a["tokens"], a["dim"], a["top_k"], None)
    for bad in [dict(rdt=3), dict(dt=-1), dict(dim=4), dict(rows=None), dict(dout=O), dict(drows=O), dict(w=None), dict(dw=None), dict(pos=None)]:
        a = dict(dout=A, dt=0, rows=A, rdt=1, pos=A, w=A, drows=A, dw=A, tokens=4, dim=8, top_k=2) | bad
        refused("bsr_expert_combine_backward", a["dout"], a["dt"], a["rows"], a["rdt"], a["pos"], a["w"], a["drows"], a["dw"], a["tokens"], a["dim"], a["top_k"], None)


def test_no_tokens_needs_no_device():
    from paper_2405_10951_b200 import binding as Bd
    L = Bd.lib()
    assert L.bsr_expert_scatter(None, 1, 0, 16, 2, None, None, None) == 0
    assert L.bsr_expert_scatter_e4m3(None, 1, 0, 16, 2, None, None, None, None) == 0
    assert L.bsr_expert_combine(None, 1, None, None, None, None, 0, 0, 16, 2, None) == 0
    assert L.bsr_expert_combine_backward(None, 1, None, 0, None, None, None, None, 0, 16, 2, None) == 0


def test_wrong_tensors_are_refused_by_the_binding():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    x, pos = torch.zeros(4, 16), torch.zeros(4, 2, dtype=torch.int32)
    rows = torch.zeros(8, 16)
    for call in [lambda: Bd.bsr_expert_sort(pos.long(), 4), lambda: Bd.bsr_expert_sort(pos.t().contiguous().t(), 4), lambda: Bd.bsr_expert_sort(pos, 4, seg_start=torch.zeros(4, dtype=torch.int32)),
                 lambda: Bd.bsr_expert_scatter(x.half(), pos), lambda: Bd.bsr_expert_scatter(x, pos[:3]), lambda: Bd.bsr_expert_scatter(x, pos, rows=rows[:, ::2]),
                 lambda: Bd.bsr_expert_combine(rows[:7], pos), lambda: Bd.bsr_expert_combine(rows, pos, weights=torch.zeros(4, 2, dtype=torch.float64)),
                 lambda: Bd.bsr_expert_combine(rows, pos, residual=x, out=x.bfloat16()),
                 lambda: Bd.bsr_expert_combine_backward(x, rows, pos, None or torch.zeros(2, 4)), lambda: Bd.bsr_expert_combine_backward(x, rows, pos, torch.zeros(4, 2), drows=rows.bfloat16())]:
        with pytest.raises(Bd.BsrError) as e:
            call()
        assert e.value.status == -1


# ---- positions ----------------------------------------------------------------------------------------------------------
def expert_ids(kind, tokens, top_k, experts):
    rng = np.random.default_rng(tokens * 7 + top_k * 3 + experts)
    if kind == "routed":
        return P.routing(rng, tokens, top_k, experts)[0]
    if kind == "masked":
        return P.routing(rng, tokens, top_k, experts, masked=0.4)[0]
    if kind == "one":
        return np.full((tokens, top_k), experts - 1, np.int32)             # all in one expert, the same one twice a token
    if kind == "none":
        return np.full((tokens, top_k), -1, np.int32)
    return rng.integers(-3, experts + 3, (tokens, top_k)).astype(np.int32)    # anything, ids outside on both sides


@gpu
@pytest.mark.parametrize("kind", ["routed", "masked", "one", "none", "any"])
@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (1, 4, 16), (5, 2, 3), (33, 3, 1024), (512, 8, 64), (513, 8, 64), (2049, 2, 16), (12608, 2, 16), (3000, 8, 256), (4097, 7, 1000), (40000, 8, 33)])
def test_sort(kind, tokens, top_k, experts):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    expert = expert_ids(kind, tokens, top_k, experts)
    pos, seg = Bd.bsr_expert_sort(torch.as_tensor(expert).cuda(), experts)
    want_pos, want_seg = P.sort(expert, experts)
    assert np.array_equal(seg.cpu().numpy(), want_seg)
    assert np.array_equal(pos.cpu().numpy(), want_pos)


@gpu
def test_sort_without_tokens():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    seg = torch.full((9,), 7, dtype=torch.int32, device="cuda")
    Bd.bsr_expert_sort(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 8, seg_start=seg)
    assert seg.cpu().tolist() == [0] * 9


# ---- rows ---------------------------------------------------------------------------------------------------------------
def to(a, dtype):
    import torch
    return torch.as_tensor(np.asarray(a, np.float32)).cuda().to(torch.float32 if dtype == "fp32" else torch.bfloat16)


def back(t):
    return t.float().cpu().numpy().astype(np.float64)


SHAPES = [(1, 1, 1, 8), (1, 4, 16, 384), (3, 2, 5, 16), (70, 3, 9, 1000), (129, 8, 64, 264), (2000, 2, 16, 384), (7, 8, 16, 4096), (40, 17, 6, 40)]


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,top_k,experts,dim", SHAPES)
def test_scatter(dtype, tokens, top_k, experts, dim):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(dim + tokens)
    pos, _ = P.sort(P.routing(rng, tokens, top_k, experts, masked=0.3)[0], experts)
    x, rows = to(rng.standard_normal((tokens, dim)), dtype), to(rng.standard_normal((tokens * top_k, dim)), dtype)
    want = P.scatter(back(x), pos, back(rows))
    got = Bd.bsr_expert_scatter(x, torch.as_tensor(pos).cuda(), rows=rows)
    assert np.array_equal(back(got), want)                # rows behind the last one are what they were


@gpu
def test_positions_outside_the_rows_are_left_out():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    pos = torch.tensor([[0, 4], [-7, 1], [2 ** 31 - 1, 6]], dtype=torch.int32, device="cuda")       # rows 0 .. 5
    x, rows = torch.ones(3, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    Bd.bsr_expert_scatter(x, pos, rows=rows)
    assert rows[:, 0].cpu().tolist() == [1, 1, 0, 0, 1, 0]
    out = Bd.bsr_expert_combine(rows + 1, pos)
    assert out[:, 0].cpu().tolist() == [4, 2, 0]
    drows, dw = Bd.bsr_expert_combine_backward(x, rows, pos, torch.full((3, 2), 3.0, device="cuda"), drows=torch.zeros_like(rows))
    assert drows[:, 0].cpu().tolist() == [3, 3, 0, 0, 3, 0] and dw.cpu().tolist() == [[8, 8], [0, 8], [0, 0]]


@gpu
@pytest.mark.parametrize("rows_type,out_type", [("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("tokens,top_k,experts,dim", SHAPES)
def test_combine_and_its_gradient(rows_type, out_type, tokens, top_k, experts, dim):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(dim * 3 + tokens)
    expert, w = P.routing(rng, tokens, top_k, experts, masked=0.3)
    pos, _ = P.sort(expert, experts)
    w[pos < 0] = np.nan                                    # of no slot that has a row
    rows = to(rng.standard_normal((tokens * top_k, dim)), rows_type)
    rows[int((pos >= 0).sum()):] = float("nan")            # nor of any token
    res, dout = to(rng.standard_normal((tokens, dim)), out_type), to(rng.standard_normal((tokens, dim)), out_type)
    tp, tw = torch.as_tensor(pos).cuda(), torch.as_tensor(w).cuda()
    half = FP32_HALF if out_type == "fp32" else BF16_HALF
    for weights, residual in [(tw, res), (tw, None), (None, None)]:
        got = back(Bd.bsr_expert_combine(rows, tp, weights, residual=residual, out=torch.empty_like(res)))
        want, mag = P.combine(back(rows), pos, None if weights is None else w, None if residual is None else back(res))
        # top_k fused multiply-adds, each off by half a step of a partial sum, and the result's own rounding
        assert np.all(np.abs(got - want) <= (top_k + 1) * FP32_HALF * mag * 1.01 + half * np.abs(want) * 1.01)
    drows0 = to(rng.standard_normal((tokens * top_k, dim)), rows_type)
    want, want_dw, mag = P.combine_backward(back(dout), np.nan_to_num(back(rows)), pos, w, back(drows0))
    drows, dw = Bd.bsr_expert_combine_backward(dout, rows, tp, tw, drows=drows0.clone())
    n = int((pos >= 0).sum())
    got = back(drows)
    half = FP32_HALF if rows_type == "fp32" else BF16_HALF
    assert np.array_equal(got[n:], back(drows0)[n:])
    assert np.all(np.abs(got - want) <= (half + FP32_HALF) * 1.01 * np.abs(want))
    # a lane's chain of multiply-adds over its share of the row, then five additions over the lanes
    assert np.all(np.abs(back(dw) - want_dw) <= (dim / 32 + 16 + 5) * FP32_HALF * mag)
    assert np.all(back(dw)[pos < 0] == 0)


@gpu
def test_combine_gradient_against_differences():
    """The sum is linear in the rows and in the weights: differences are exact up to rounding whatever their size."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(5)
    expert, w = P.routing(rng, 50, 3, 7, masked=0.2)
    pos, _ = P.sort(expert, 7)
    rows, step, wstep, dout = (rng.standard_normal(s) for s in [(150, 64), (150, 64), (50, 3), (50, 64)])
    tp = torch.as_tensor(pos).cuda()
    run = lambda r, ww: back(Bd.bsr_expert_combine(to(r, "fp32"), tp, to(ww, "fp32")))
    drows, dw = Bd.bsr_expert_combine_backward(to(dout, "fp32"), to(rows, "fp32"), tp, to(w, "fp32"), drows=torch.zeros(150, 64, device="cuda"))
    scale = np.abs(dout).sum() * 4                          # magnitudes below 4: each of the sums is off by a few of 2^-24 of that
    d = (dout * (run(rows + step, w) - run(rows - step, w))).sum() / 2
    assert abs(d - (back(drows) * step).sum()) <= 32 * FP32_HALF * scale
    d = (dout * (run(rows, w + wstep) - run(rows, w - wstep))).sum() / 2
    assert abs(d - (back(dw) * wstep).sum()) <= 64 * FP32_HALF * scale


@gpu
def test_scatter_gradient_is_the_plain_sum():
    """<rows', scatter(x)> = <combine(rows'), x>: the adjoint, on the same positions."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(6)
    pos, seg = P.sort(P.routing(rng, 90, 4, 11, masked=0.2)[0], 11)
    x, g = to(rng.standard_normal((90, 72)), "fp32"), to(rng.standard_normal((360, 72)), "fp32")
    tp = torch.as_tensor(pos).cuda()
    rows = back(Bd.bsr_expert_scatter(x, tp, rows=torch.zeros(360, 72, device="cuda")))
    dx = back(Bd.bsr_expert_combine(g, tp))
    scale = np.abs(back(g)).sum()
    assert abs((rows * back(g)).sum() - (dx * back(x)).sum()) <= 8 * FP32_HALF * 4 * scale


@gpu
def test_calls_on_another_device_are_refused():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    with pytest.raises(Bd.BsrError) as e:
        Bd.bsr_expert_scatter(torch.zeros(4, 16), torch.zeros(4, 2, dtype=torch.int32))
    assert e.value.status == -1 and "current device" in str(e.value)
