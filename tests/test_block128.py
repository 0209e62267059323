"""E4M3 with a power-of-two scale per block of 128: quantisation, products (dense and with a weight per expert's rows) and the expert
layer built from them, against plain implementations in 64 bits."""
import numpy as np
import pytest

import expert_plain as P

gpu = pytest.mark.gpu
A, O = 4096, 4104            # a 16-byte aligned address and one that is not (never read)
BF16_HALF = 2.0 ** -8


def refused(name, *args):
    from paper_2405_10951_b200 import binding as Bd
    assert getattr(Bd.lib(), name)(*args) == -1, name
    assert len(Bd.lib().bsr_last_error(None)) > 0


def test_refusals():
    for bad in [dict(dt=2), dict(m=-1), dict(k=0), dict(k=24), dict(x=None), dict(x=O), dict(q=O), dict(s=4098)]:
        a = dict(x=A, dt=1, m=4, k=32, q=A, s=A) | bad
        refused("bsr_quantize_e4m3_rows128", a["x"], a["dt"], a["m"], a["k"], a["q"], a["s"], None)
    for bad in [dict(dt=2), dict(c=0), dict(c=65536), dict(n=0), dict(n=128 * 65535 + 1), dict(k=8), dict(w=None), dict(qt=A, st=None), dict(qt=None, st=A), dict(qt=A, st=A, n=24),
                dict(q=O), dict(qt=O, st=A)]:
        a = dict(w=A, dt=0, c=2, n=32, k=32, q=A, s=A, qt=None, st=None) | bad
        refused("bsr_quantize_e4m3_blocks128", a["w"], a["dt"], a["c"], a["n"], a["k"], a["q"], a["s"], a["qt"], a["st"], None)
    for bad in [dict(x=None), dict(x=O), dict(w=None), dict(xs=None), dict(ws=4098), dict(b=O), dict(y=None), dict(y=O), dict(m=-1), dict(m=(1 << 30) + 1), dict(n=(1 << 30) + 8), dict(k=(1 << 30) + 16), dict(n=4), dict(n=12), dict(k=8), dict(act=3), dict(act=-1),
                dict(act=0, z=A), dict(act=2, z=None), dict(act=1, z=O)]:
        a = dict(x=A, xs=A, w=A, ws=A, b=A, z=None, y=A, m=4, n=16, k=32, act=0) | bad
        refused("bsr_linear_forward_e4m3_block128", a["x"], a["xs"], a["w"], a["ws"], a["b"], a["z"], a["y"], a["m"], a["n"], a["k"], a["act"], None)
        refused("bsr_expert_linear_e4m3_block128", a["x"], a["xs"], a["w"], a["ws"], a["b"], A, a["z"], a["y"], a["m"], a["n"], a["k"], 2, a["act"], None)
    for experts, n, seg in [(0, 16, A), (1025, 16, A), (1024, 1 << 21, A), (2, 16, None)]:
        refused("bsr_expert_linear_e4m3_block128", A, A, A, A, None, seg, None, A, 4, n, 32, experts, 0, None)


def test_no_rows_needs_no_device():
    from paper_2405_10951_b200 import binding as Bd
    L = Bd.lib()
    assert L.bsr_quantize_e4m3_rows128(None, 1, 0, 32, None, None, None) == 0
    assert L.bsr_linear_forward_e4m3_block128(None, None, None, None, None, None, None, 0, 16, 32, 0, None) == 0
    assert L.bsr_expert_linear_e4m3_block128(None, None, None, None, None, None, None, None, 0, 16, 32, 4, 0, None) == 0


def test_scale_stride():
    from paper_2405_10951_b200 import binding as Bd
    for k in (1, 16, 128, 511, 512, 513, 1024, 7168):
        assert Bd.lib().bsr_e4m3_scale_stride(k) == Bd.bsr_e4m3_scale_stride(k) == P.stride(k)
    assert Bd.lib().bsr_e4m3_scale_stride(0) == 0


def test_wrong_tensors_are_refused_by_the_binding():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    x, xs, w, ws = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.uint8)
    for call in [lambda: Bd.bsr_quantize_e4m3_rows128(torch.zeros(4, 32, dtype=torch.float16)), lambda: Bd.bsr_quantize_e4m3_rows128(torch.zeros(32, 4).t()),
                 lambda: Bd.bsr_quantize_e4m3_blocks128(torch.zeros(2, 2, 16, 16)), lambda: Bd.bsr_quantize_e4m3_blocks128(torch.zeros(16, 16), scale=torch.zeros(1, 1, dtype=torch.uint8)),
                 lambda: Bd.bsr_linear_forward_e4m3_block128(x.float(), xs, w, ws), lambda: Bd.bsr_linear_forward_e4m3_block128(x, xs[:, :1], w, ws),
                 lambda: Bd.bsr_linear_forward_e4m3_block128(x, xs, w[:, :16], ws), lambda: Bd.bsr_linear_forward_e4m3_block128(x, xs, w, ws, bias=torch.zeros(8)),
                 lambda: Bd.bsr_linear_forward_e4m3_block128(x, xs, w, ws, y=torch.zeros(4, 16)),
                 lambda: Bd.bsr_expert_linear_e4m3_block128(x, xs, w[None], ws[None], torch.zeros(3, dtype=torch.int32))]:
        with pytest.raises(Bd.BsrError) as e:
            call()
        assert e.value.status == -1


def test_plain_derivative_of_gelu():
    z = np.linspace(-7, 7, 301)
    h = 1e-5
    assert np.abs((P.gelu(z + h) - P.gelu(z - h)) / (2 * h) - P.gelu_grad(z)).max() < 1e-9


# ---- quantisation -----------------------------------------------------------------------------------------------------
def values(rng, shape, dtype):
    """Blocks of every size: exponents from 2^-120 to 2^100, zeros, values on the codes' borders."""
    x = rng.standard_normal(shape) * np.ldexp(1.0, rng.integers(-3, 4, shape))
    x *= np.ldexp(1.0, rng.integers(-40, 40, shape[:-1] + (1,)))
    x[rng.random(shape) < 0.02] = 0.0
    at = x.reshape(-1, shape[-1])
    if at.shape[0] > 4:
        at[0] = 0.0
        at[1] *= np.ldexp(1.0, 60)
        at[2] = np.ldexp(1.0, -127) * rng.standard_normal(shape[-1])          # scales below the least one, values without a leading bit
        at[3] = np.ldexp(448.0 + 32.0 * rng.integers(-1, 2, shape[-1]), 3)    # just at, above and below the line between two scales
        at[4, ::2] = 17.0
        at[4, 1::2] = 272.0                                                   # ties
    import torch
    return torch.as_tensor(x.astype(np.float32)).to(torch.float32 if dtype == "fp32" else torch.bfloat16)


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,k", [(1, 16), (5, 128), (9, 144), (33, 512), (7, 528), (130, 768), (3, 2048), (6, 7168)])
def test_quantize_rows(dtype, m, k):
    from paper_2405_10951_b200 import binding as Bd
    x = values(np.random.default_rng(m + k), (m, k), dtype)
    q, scale = Bd.bsr_quantize_e4m3_rows128(x.cuda())
    want_q, want_scale = P.quantize(wide(x), 1)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    assert np.array_equal(wide(q), want_q)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("stack,n,k", [((), 16, 16), ((), 8, 144), ((3,), 128, 128), ((2,), 144, 272), ((2,), 1040, 528), ((1,), 256, 1040), ((5,), 48, 16)])
def test_quantize_blocks(dtype, stack, n, k):
    from paper_2405_10951_b200 import binding as Bd
    w = values(np.random.default_rng(n + k), stack + (n, k), dtype)
    both = n % 16 == 0
    out = Bd.bsr_quantize_e4m3_blocks128(w.cuda(), transposed=both)
    mats = wide(w).reshape((-1, n, k))
    for i, mat in enumerate(mats):
        at = lambda t: t.reshape((len(mats),) + tuple(t.shape[len(stack):]))[i]
        want_q, want_scale = P.quantize(mat, 128)
        assert np.array_equal(at(out[1]).cpu().numpy(), want_scale)
        assert np.array_equal(wide(at(out[0])), want_q)
        if both:
            want_q, want_scale = P.quantize(mat.T, 128)
            assert np.array_equal(at(out[3]).cpu().numpy(), want_scale)
            assert np.array_equal(wide(at(out[2])), want_q)


@gpu
def test_values_that_are_not_finite_stay_with_themselves():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((20, 256)).astype(np.float32), rng.standard_normal((40, 256)).astype(np.float32)
    x[3, 7], x[11, 200], w[5, 130] = np.inf, np.nan, -np.inf
    for dtype in (torch.float32, torch.bfloat16):
        tx, tw = torch.as_tensor(x).to(dtype), torch.as_tensor(w).to(dtype)
        for t, per, call in [(tx, 1, Bd.bsr_quantize_e4m3_rows128), (tw, 128, Bd.bsr_quantize_e4m3_blocks128)]:
            q, s = call(t.cuda())
            want_q, want_s = P.quantize(wide(t), per)
            assert np.array_equal(wide(q), want_q, equal_nan=True) and np.array_equal(s.cpu().numpy(), want_s)
        y = wide(Bd.bsr_linear_forward_e4m3_block128(*Bd.bsr_quantize_e4m3_rows128(tx.cuda()), *Bd.bsr_quantize_e4m3_blocks128(tw.cuda())))
        lost = np.zeros((20, 40), bool)
        lost[[3, 11]] = True
        lost[:, 5] = True
        assert np.array_equal(np.isnan(y), lost) and not np.isinf(y).any()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,top_k,experts,dim", [(1, 1, 1, 16), (1, 4, 16, 384), (70, 3, 9, 1040), (129, 8, 64, 528), (9, 17, 4, 144)])
def test_scatter_in_blocks_is_the_scattered_rows_in_blocks(dtype, tokens, top_k, experts, dim):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(dim)
    pos = torch.as_tensor(P.sort(P.routing(rng, tokens, top_k, experts, masked=0.3)[0], experts)[0]).cuda()
    x = values(rng, (tokens, dim), dtype).cuda()
    n = int((pos >= 0).sum())
    q0 = torch.full((tokens * top_k, dim), 33, dtype=torch.uint8, device="cuda")
    s0 = torch.full((tokens * top_k, P.stride(dim)), 44, dtype=torch.uint8, device="cuda")
    q, scale = Bd.bsr_expert_scatter_e4m3(x, pos, q=q0, scale=s0)
    rows = Bd.bsr_expert_scatter(x, pos, rows=torch.zeros((tokens * top_k, dim), dtype=x.dtype, device="cuda"))
    want_q, want_scale = Bd.bsr_quantize_e4m3_rows128(rows)
    assert torch.equal(q[:n], want_q[:n].view(torch.uint8)) and torch.equal(scale[:n], want_scale[:n])
    assert bool((q[n:] == 33).all()) and bool((scale[n:] == 44).all())          # rows behind the last one


# ---- products -----------------------------------------------------------------------------------------------------------
def operands(rng, m, stack, n, k):
    """Codes and scales of operands whose blocks differ in size by up to 2^12, so that a scale in the wrong place shows."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    x = rng.standard_normal((m, k)) * np.ldexp(1.0, rng.integers(-6, 7, (m, -(-k // 128))).repeat(128, 1)[:, :k])
    w = rng.standard_normal(stack + (n, k)) / np.sqrt(k)
    blocks = rng.integers(-6, 7, stack + (-(-n // 128), -(-k // 128)))
    w *= np.ldexp(1.0, blocks.repeat(128, -1).repeat(128, -2)[..., :n, :k])
    t = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    xq, xs = Bd.bsr_quantize_e4m3_rows128(t(x))
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(t(w))
    mats = [P.dequantize(wide(a), b.cpu().numpy(), 128) for a, b in zip(wq.reshape((-1, n, k)), ws.reshape((-1,) + tuple(ws.shape[-2:])))]
    return xq, xs, wq, ws, P.dequantize(wide(xq), xs.cpu().numpy(), 1), mats


def near(got, want, mag, k, lip=1.0, off=0.0):
    """Each of the k / 32 instructions of a sum adds to a 24-bit accumulator and drops what is below (a step, 2^-23, of the
    sum of magnitudes); lip: what the activation makes of that, `off`: how far it is off itself; the result is rounded to bf16 once."""
    acc = (k / 32 + 2) * 2.0 ** -23 * mag * lip + off
    ok = np.abs(got - want) <= acc + 2.0 ** -22 * np.abs(want) + BF16_HALF * 1.01 * (np.abs(want) + acc) + 1e-37
    assert ok.all(), (np.abs(got - want)[~ok][:5], want[~ok][:5], np.argwhere(~ok)[:5], (~ok).sum())


def phi_off(z):
    """The kernel forms Phi(-t) = exp(-t^2 / 2) R(t) with an R that is within 2.9e-5 of its value for every t; the exponential is 2 to a
    power of up to 126 that is rounded to 2^-24 of itself, twice: 126 * 2^-23 * ln 2 = 1.04e-5; and nine operations of at most 2^-22 each.
    An exponential below 2^-126 is flushed to zero."""
    return 2.0 ** -126 + (2.9e-5 + 1.04e-5 + 9 * 2.0 ** -22) * P.phi(z)


def gelu_grad_off(z):
    """GELU' = Phi + z phi, two terms of either sign: near z = -0.75 they cancel, and what each is off by is not small beside
    their sum.  z phi has the exponential's error and some products' roundings; above zero Phi is 1 - Phi(-z)."""
    return phi_off(-np.abs(z)) + 2.0 ** -22 * P.phi(z) + (2.0 ** -126 + (1.04e-5 + 9 * 2.0 ** -22) * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)) * np.abs(z)


def check(got, zgot, act, part, mag, z, k):
    if act == 0:
        near(got, part, mag, k)
    elif act == 1:
        near(zgot, part, mag, k)
        near(got, P.gelu(part), mag, k, 1.13, np.abs(part) * phi_off(-np.abs(part)))     # |GELU'| < 1.13; the tail is what is approximated
    else:
        near(got, part * P.gelu_grad(z), mag * np.abs(P.gelu_grad(z)), k, 1.0, np.abs(part) * gelu_grad_off(z))


@gpu
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("m,n,k", [(1, 8, 16), (1, 264, 144), (33, 72, 512), (127, 64, 128), (128, 128, 640), (129, 200, 528), (300, 1000, 1040), (64, 384, 1536), (97, 2304, 768),
                                   # few tiles: k over 2, 4 and 8 CTAs, shares of rows that do not come out even
                                   (1, 2000, 7168), (7, 72, 4112), (130, 64, 2064), (200, 1000, 1040), (65, 512, 8192), (127, 8, 4096),
                                   # several tiles a CTA, of 192 columns; many slabs; more stages of scales than there are
                                   (2600, 1544, 400), (1300, 2000, 2576), (700, 3000, 4112),
                                   # tiles over two CTAs
                                   (2600, 1544, 4112), (4200, 776, 5136)])
def test_product(act, m, n, k):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(m + n + k + act)
    xq, xs, wq, ws, x, (w,) = operands(rng, m, (), n, k)
    bias = rng.standard_normal(n).astype(np.float32)
    z = torch.as_tensor(3 * rng.standard_normal((m, n)).astype(np.float32)).cuda().bfloat16() if act == 2 else torch.zeros((m, n), dtype=torch.bfloat16, device="cuda") if act == 1 else None
    y = Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws, torch.as_tensor(bias).cuda(), act=act, z=z)
    part, mag = x @ w.T + bias, np.abs(x) @ np.abs(w).T + np.abs(bias)
    check(wide(y), None if z is None else wide(z), act, part, mag, None if z is None else wide(z), k)
    if act == 1:                                            # without a place for the pre-activation, and without a bias
        assert torch.equal(Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws, torch.as_tensor(bias).cuda(), act=1), y)
    if act == 0:
        near(wide(Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws)), x @ w.T, np.abs(x) @ np.abs(w).T, k)


@gpu
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("counts,n,k", [([1], 64, 128), ([0, 0, 3, 0], 72, 144), ([5, 0, 1, 130, 0, 64], 200, 528), ([0] * 7, 64, 128), ([1] * 64, 264, 512), ([128, 129, 127], 384, 400),
                                        ([300, 31, 33, 0, 700, 97, 2], 1544, 272), ([2] * 400, 64, 144), ([1500, 0, 1300, 7, 1290], 1544, 3216)])
def test_product_per_expert(act, counts, n, k):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(sum(counts) + n + k + act)
    m = sum(counts) + 9                                     # rows behind the last segment
    xq, xs, wq, ws, x, mats = operands(rng, m, (len(counts),), n, k)
    bias = rng.standard_normal((len(counts), n)).astype(np.float32)
    seg = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    z0 = torch.as_tensor(rng.standard_normal((m, n)).astype(np.float32)).cuda().bfloat16()
    z = z0.clone() if act else None
    y0 = torch.as_tensor(rng.standard_normal((m, n)).astype(np.float32)).cuda().bfloat16()
    y = Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, torch.as_tensor(seg).cuda(), torch.as_tensor(bias).cuda(), act=act, z=z, y=y0.clone())
    assert torch.equal(y[seg[-1]:], y0[seg[-1]:])
    if act:
        assert torch.equal(z[seg[-1]:], z0[seg[-1]:])
    for e, w in enumerate(mats):
        at = np.s_[seg[e]:seg[e + 1]]
        part, mag = x[at] @ w.T + bias[e], np.abs(x[at]) @ np.abs(w).T + np.abs(bias[e])
        if counts[e]:
            check(wide(y)[at], None if z is None else wide(z)[at], act, part, mag, wide(z0)[at], k)


@gpu
@pytest.mark.parametrize("m,n,k,experts", [(620000, 8, 16, 0), (9000, 1544, 16, 1024), (160000, 776, 768, 0), (170000, 776, 768, 5), (5000, 776, 4112, 3)])
def test_many_tiles_a_worker(m, n, k, experts):
    """More tiles a CTA, or pair of them, than its list holds; the last case: segments of no rows at all.  Rows are compared by sample."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(n)
    x = (torch.randn((m, k), device="cuda") * torch.exp2(torch.randint(-6, 7, (m, 1), device="cuda").float())).bfloat16()
    w = (torch.randn((max(experts, 1), n, k), device="cuda") / np.sqrt(k)).bfloat16()
    xq, xs = Bd.bsr_quantize_e4m3_rows128(x)
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(w)
    ends = np.zeros(experts + 1, np.int32)
    if experts and m != 5000:
        ends[1:] = np.sort(rng.integers(0, m - 50, experts))
        ends[1:4] = ends[3]                               # two experts without rows
    y0 = torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda")
    if experts:
        y = Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, torch.as_tensor(ends).cuda(), y=y0.clone())
    else:
        y = Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq[0], ws[0], y=y0.clone())
    pick = np.unique(np.concatenate([np.arange(0, m, m // 700), np.arange(m - 300, m), ends[:-1], np.maximum(ends - 1, 0)]))
    at = torch.as_tensor(pick).cuda()
    X, Y = P.dequantize(wide(xq[at]), xs[at].cpu().numpy(), 1), wide(y[at])
    of = np.searchsorted(ends[1:], pick, side="right") if experts else np.zeros(len(pick), int)
    for e in np.unique(of):
        rows = of == e
        if experts and e == experts:
            assert np.all(Y[rows] == 7.0)
            continue
        W = P.dequantize(wide(wq[e]), ws[e].cpu().numpy(), 128)
        near(Y[rows], X[rows] @ W.T, np.abs(X[rows]) @ np.abs(W).T, k)


@gpu
def test_segments_outside_the_rows_are_cut():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(8)
    xq, xs, wq, ws, x, mats = operands(rng, 40, (4,), 64, 128)
    seg = torch.tensor([-5, 10, 7, 30, 90], dtype=torch.int32, device="cuda")           # a segment that ends before it begins has no rows
    y = wide(Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, seg, y=torch.zeros((40, 64), dtype=torch.bfloat16, device="cuda")))
    for e, a, b in [(0, 0, 7), (2, 7, 30), (3, 30, 40)]:
        near(y[a:b], x[a:b] @ mats[e].T, np.abs(x[a:b]) @ np.abs(mats[e]).T, 128)


@gpu
def test_a_row_does_not_depend_on_its_neighbours():
    """Rows hold what their own operands give, bit for bit, wherever they lie (NaN and infinite neighbours included)."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(9)
    xq, xs, wq, ws, _, _ = operands(rng, 200, (3,), 264, 528)
    seg = torch.tensor([0, 40, 170, 200], dtype=torch.int32, device="cuda")
    y = Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, seg)
    bad = xq.view(torch.uint8).clone()
    bad[170:] = 0x7f                                        # NaN in the next expert's rows, which the tile loads too
    bad[:40] = 0xff
    y2 = Bd.bsr_expert_linear_e4m3_block128(bad, xs, wq, ws, seg)
    assert torch.equal(y[40:170], y2[40:170]) and bool(torch.isnan(y2[170:]).all())


@gpu
@pytest.mark.parametrize("m,n,k", [(5, 72, 144), (300, 1000, 1040), (2, 512, 4096)])
def test_scales_far_apart(m, n, k):
    """Rows and blocks from 2^-100 to 2^100, the least scale (2^-127) among them: a scale is an exponent, nothing of it is lost."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(k)
    far = rng.integers(-100, 101, (m, 1))
    x = rng.standard_normal((m, k)) * np.ldexp(1.0, far)
    w = rng.standard_normal((n, k)) / np.sqrt(k)
    x[0] = np.ldexp(rng.standard_normal(k), -124)
    w[:min(n, 128)] *= np.ldexp(1.0, 20)
    t = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    xq, xs = Bd.bsr_quantize_e4m3_rows128(t(x))
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(t(w))
    assert int(xs[0, 0]) == 0
    X, W = P.dequantize(wide(xq), xs.cpu().numpy(), 1), P.dequantize(wide(wq), ws.cpu().numpy(), 128)
    y = wide(Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws))
    part, mag = X @ W.T, np.abs(X) @ np.abs(W).T
    normal = mag > 2.0 ** -100                              # (below, float32 has fewer bits, or flushes)
    near(y[normal], part[normal], mag[normal], k)
    assert np.all(np.abs(y[~normal]) <= 2.0 ** -99)


@gpu
@pytest.mark.parametrize("m,k", [(40, 128), (40, 2048), (20000, 128)])
def test_activations_of_infinities(m, k):
    """GELU(inf) = inf, GELU(-inf) = 0, GELU'(inf) = 1, GELU'(-inf) = 0, and NaN stays itself: as limits say."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    xq, xs, wq, ws, _, _ = operands(np.random.default_rng(k), m, (), 64, k)
    bias = torch.zeros(64, device="cuda")
    bias[3], bias[5], bias[7] = float("inf"), float("-inf"), float("nan")
    y = wide(Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws, bias, act=Bd.ACT_GELU))
    assert np.all(y[:, 3] == np.inf) and np.all(y[:, 5] == 0) and np.all(np.isnan(y[:, 7])) and np.isfinite(y[:, [0, 1, 2, 4, 6] + list(range(8, 64))]).all()
    z = bias.bfloat16().expand(m, 64).contiguous()
    g, plain = (wide(Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws, act=a, z=zz)) for a, zz in [(Bd.ACT_GELU_GRAD, z), (Bd.ACT_NONE, None)])
    assert np.array_equal(g[:, 3], plain[:, 3]) and np.all(g[:, 5] == 0) and np.all(np.isnan(g[:, 7]))


# ---- the layer ------------------------------------------------------------------------------------------------------------
def layer(Bd, x, expert, weights, dout, W1, W2, b1, b2, experts):
    """An expert layer with frozen weights in 8 bits, forward and backward, as a program calls it."""
    import torch
    pos, seg = Bd.bsr_expert_sort(expert, experts)
    xq, xs = Bd.bsr_expert_scatter_e4m3(x, pos)
    rows, hidden = xq.shape[0], W1[0].shape[1]
    z, h, o = (torch.zeros((rows, n), dtype=torch.bfloat16, device=x.device) for n in (hidden, hidden, x.shape[1]))
    Bd.bsr_expert_linear_e4m3_block128(xq, xs, W1[0], W1[1], seg, b1, act=Bd.ACT_GELU, z=z, y=h)
    hq, hs = Bd.bsr_quantize_e4m3_rows128(h)
    Bd.bsr_expert_linear_e4m3_block128(hq, hs, W2[0], W2[1], seg, b2, y=o)
    out = Bd.bsr_expert_combine(o, pos, weights, residual=x)
    do, dw = Bd.bsr_expert_combine_backward(dout, o, pos, weights, drows=torch.zeros_like(o))
    doq, dos = Bd.bsr_quantize_e4m3_rows128(do)
    dz, dxr = torch.zeros_like(h), torch.zeros_like(o)
    Bd.bsr_expert_linear_e4m3_block128(doq, dos, W2[2], W2[3], seg, act=Bd.ACT_GELU_GRAD, z=z, y=dz)
    dzq, dzs = Bd.bsr_quantize_e4m3_rows128(dz)
    Bd.bsr_expert_linear_e4m3_block128(dzq, dzs, W1[2], W1[3], seg, y=dxr)
    dx = Bd.bsr_expert_combine(dxr, pos, residual=dout)
    return dict(pos=pos, seg=seg, out=out, dw=dw, dx=dx)


def layer_inputs(seed, tokens, top_k, experts, dim, hidden, masked):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(seed)
    expert, weights = P.routing(rng, tokens, top_k, experts, masked=masked)
    t = lambda a: torch.as_tensor(np.asarray(a, np.float32)).cuda()
    w1, w2 = t(rng.standard_normal((experts, hidden, dim)) / np.sqrt(dim)).bfloat16(), t(rng.standard_normal((experts, dim, hidden)) / np.sqrt(hidden)).bfloat16()
    return dict(x=t(rng.standard_normal((tokens, dim))), expert=torch.as_tensor(expert).cuda(), weights=t(weights), dout=t(rng.standard_normal((tokens, dim))),
                W1=Bd.bsr_quantize_e4m3_blocks128(w1, transposed=True), W2=Bd.bsr_quantize_e4m3_blocks128(w2, transposed=True),
                b1=t(rng.standard_normal((experts, hidden))), b2=t(rng.standard_normal((experts, dim))), experts=experts)


def plain_layer(a, dx_step=None):
    """The same layer in 64 bits on the weights as they are held, without rounding of activations."""
    x, expert, wt, dout = (a[n].cpu().numpy().astype(np.float64) for n in ("x", "expert", "weights", "dout"))
    if dx_step is not None:
        x = x + dx_step
    expert = expert.astype(int)
    W1, W2 = ([P.dequantize(wide(q), s.cpu().numpy(), 128) for q, s in zip(a[n][0], a[n][1])] for n in ("W1", "W2"))
    b1, b2 = wide(a["b1"]), wide(a["b2"])
    out, dx, dw = x.copy(), dout.copy(), np.zeros(expert.shape)
    for e in range(a["experts"]):
        t, s = np.nonzero(expert == e)
        z = x[t] @ W1[e].T + b1[e]
        o = P.gelu(z) @ W2[e].T + b2[e]
        np.add.at(out, t, wt[t, s][:, None] * o)
        dw[t, s] = (dout[t] * o).sum(1)
        dz = (wt[t, s][:, None] * dout[t]) @ W2[e] * P.gelu_grad(z)
        np.add.at(dx, t, dz @ W1[e])
    return out, dx, dw


def test_plain_layer_gradient_against_differences():
    """(The oracle's own check, on the CPU.)"""
    import torch
    rng = np.random.default_rng(1)
    t = torch.as_tensor
    q = lambda s: (t(rng.integers(-8, 9, s).astype(np.float32)), t(np.full((s[0], -(-s[1] // 128), P.stride(s[2])), 124, np.uint8)))
    a = dict(x=t(rng.standard_normal((6, 16))), expert=t(P.routing(rng, 6, 2, 3, masked=0.2)[0]), weights=t(rng.random((6, 2))), dout=t(rng.standard_normal((6, 16))), W1=q((3, 32, 16)), W2=q((3, 16, 32)),
             b1=t(rng.standard_normal((3, 32))), b2=t(rng.standard_normal((3, 16))), experts=3)
    _, dx, _ = plain_layer(a)
    step = 1e-5 * rng.standard_normal((6, 16))
    d = (a["dout"].numpy() * (plain_layer(a, step)[0] - plain_layer(a, -step)[0])).sum() / 2
    assert abs(d - (dx * step).sum()) < 1e-8


def rel(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@gpu
@pytest.mark.parametrize("tokens,top_k,experts,dim,hidden,masked", [(1, 4, 16, 384, 1536, 0.0), (197, 2, 16, 384, 1536, 0.2), (700, 3, 5, 272, 528, 0.1)])
def test_expert_layer_forward_and_backward(tokens, top_k, experts, dim, hidden, masked):
    """The layer's outputs against 64 bits.  Each 8-bit rounding of activations is off by at most 2^-4 of a value, uniformly
    in its step: the root mean square is 2^-3 / sqrt(12) / 1.5 (the mean of a value over its leading power of two) = 2.4 %, at most 3.6 %.
    The layer's term passes two of them in either direction (the backward pass has its own two, and GELU' of a z that
    carries the first), each of which a random sum passes on in proportion: 3.6 % * sqrt(2) = 5.1 %, and 3.6 % * sqrt(4) = 7.2 %."""
    from paper_2405_10951_b200 import binding as Bd
    a = layer_inputs(tokens, tokens, top_k, experts, dim, hidden, masked)
    got = layer(Bd, **a)
    out, dx, dw = plain_layer(a)
    x, dout = wide(a["x"]), wide(a["dout"])
    assert rel(wide(got["out"]) - x, out - x) < 0.051
    assert rel(wide(got["dx"]) - dout, dx - dout) < 0.072
    assert rel(wide(got["dw"]), dw) < 0.072


@gpu
def test_expert_layer_on_another_stream_and_in_a_graph():
    """The same bits on the default stream, on another one, and from a captured graph replayed on new inputs beside a second one."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    a, b = layer_inputs(1, 150, 2, 8, 272, 528, 0.1), layer_inputs(2, 150, 2, 8, 272, 528, 0.1)
    want_a, want_b = layer(Bd, **a), layer(Bd, **b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = layer(Bd, **a)
    torch.cuda.synchronize()
    held = {k: v.clone() if torch.is_tensor(v) else tuple(u.clone() for u in v) if isinstance(v, tuple) else v for k, v in a.items()}
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer(Bd, **held)
        graphs.append((g, out))
    for inputs, want in [(a, want_a), (b, want_b), (a, want_a)]:
        for k, v in inputs.items():
            if torch.is_tensor(v):
                held[k].copy_(v)
            elif isinstance(v, tuple):
                for to, frm in zip(held[k], v):
                    to.view(torch.uint8).copy_(frm.view(torch.uint8))
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        n = int(want["seg"][-1])
        for _, out in graphs:
            for k in want:
                assert torch.equal(out[k], want[k]), k
    for k in want_a:
        assert torch.equal(on_side[k], want_a[k]), k


def large_calls(Bd, a):
    """A sort over a cluster of sixteen CTAs, rows in blocks, a product over pairs of CTAs, one over a cluster, the weighted sum."""
    import torch
    pos, seg = Bd.bsr_expert_sort(a["expert"], 12)
    q, s = Bd.bsr_expert_scatter_e4m3(a["x"], pos, q=torch.zeros((a["expert"].numel(), 272), dtype=torch.uint8, device="cuda"), scale=torch.zeros((a["expert"].numel(), 4), dtype=torch.uint8, device="cuda"))
    y = Bd.bsr_linear_forward_e4m3_block128(a["xq"], a["xs"], a["wq"], a["ws"])
    few = Bd.bsr_linear_forward_e4m3_block128(a["xq"][:40], a["xs"][:40], a["wq"], a["ws"], act=Bd.ACT_GELU)
    out = Bd.bsr_expert_combine(a["rows"], pos, a["weights"])
    return [pos, seg, q, s, y, few, out]


def large_inputs(seed):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(seed)
    expert, weights = P.routing(rng, 17000, 5, 12, masked=0.1)
    torch.manual_seed(seed)
    a = dict(expert=torch.as_tensor(expert).cuda(), weights=torch.as_tensor(weights).cuda(), x=torch.randn((17000, 272), device="cuda"), rows=torch.randn((85000, 272), device="cuda").bfloat16())
    a["xq"], a["xs"] = Bd.bsr_quantize_e4m3_rows128(torch.randn((2600, 4112), device="cuda"))
    a["wq"], a["ws"] = Bd.bsr_quantize_e4m3_blocks128(torch.randn((1544, 4112), device="cuda"))
    return a


@gpu
def test_large_calls_captured_and_replayed():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    a, b = large_inputs(1), large_inputs(2)
    want = [[t.clone() for t in large_calls(Bd, v)] for v in (a, b)]
    held = {k: v.clone() for k, v in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = large_calls(Bd, held)
    for inputs, expected in [(a, want[0]), (b, want[1]), (a, want[0])]:
        for k, v in inputs.items():
            held[k].view(torch.uint8).copy_(v.view(torch.uint8))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, expected):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
def test_calls_on_two_streams_at_once():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    inputs = [large_inputs(3), large_inputs(4)]
    want = [[t.clone() for t in large_calls(Bd, v)] for v in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(large_calls(Bd, inputs[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for outs in got[i]:
            for x, y in zip(outs, want[i]):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
def test_long_offsets():
    """More than 2^31 values of an operand: offsets pass 32 bits."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    tokens, dim = 270000, 8192                              # 2.2e9 values, 4.4 GB a tensor
    x = torch.zeros((tokens, dim), dtype=torch.bfloat16, device="cuda")
    pick = torch.tensor([0, 131071, 262143, 262145, tokens - 1], device="cuda")
    x[pick] = torch.randn((5, dim), device="cuda").bfloat16()
    pos = torch.arange(tokens - 1, -1, -1, dtype=torch.int32, device="cuda").view(tokens, 1)
    rows = Bd.bsr_expert_scatter(x, pos)
    assert torch.equal(rows[tokens - 1 - pick], x[pick])
    q, scale = Bd.bsr_expert_scatter_e4m3(x, pos)
    want_q, want_scale = Bd.bsr_quantize_e4m3_rows128(x[pick].contiguous())
    assert torch.equal(q[tokens - 1 - pick].view(torch.uint8), want_q.view(torch.uint8)) and torch.equal(scale[tokens - 1 - pick], want_scale)
    back = Bd.bsr_expert_combine(rows, pos)
    assert torch.equal(back[pick], x[pick])
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(torch.randn((64, dim), device="cuda"))
    y = Bd.bsr_linear_forward_e4m3_block128(q, scale, wq, ws)
    want = Bd.bsr_linear_forward_e4m3_block128(want_q, want_scale, wq, ws)
    assert torch.equal(y[tokens - 1 - pick], want) and float(y[1000:2000].abs().max()) == 0.0
