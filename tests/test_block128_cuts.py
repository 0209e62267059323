"""Products in 8-bit blocks, each kernel and width by name: the cases say which one they are for, and fail where a rule sends them elsewhere."""
import numpy as np
import pytest

import expert_plain as P
import test_block128 as base

ONE, PAIR, CLUSTER = 0, 1, 2

# (kernel, columns a tile, CTAs a tile's k): rows, columns, k, experts (0: dense)
CASES = [
    # a CTA a tile: several groups of scales a tile (k > 512), more of them than there are stages (k > 2048), several tiles a CTA; last tiles full and not
    ((ONE, 64, 1), 40000, 64, 1040, 0), ((ONE, 64, 1), 40000, 40, 2576, 4), ((ONE, 128, 1), 40000, 128, 1040, 0), ((ONE, 128, 1), 40000, 104, 2576, 0), ((ONE, 128, 1), 40000, 104, 528, 4),
    ((ONE, 192, 1), 20003, 576, 2576, 0), ((ONE, 192, 1), 20003, 1000, 640, 0), ((ONE, 192, 1), 20003, 536, 2576, 0), ((ONE, 192, 1), 20003, 536, 2576, 5), ((ONE, 192, 1), 12608, 768, 1040, 5),
    # k over a cluster
    ((CLUSTER, 64, 2), 1, 4096, 1024, 0), ((CLUSTER, 64, 2), 300, 72, 1040, 0), ((CLUSTER, 64, 4), 130, 64, 2064, 0), ((CLUSTER, 64, 8), 65, 512, 8192, 0),
]
# pairs of CTAs, every width: two tiles of columns, the last full, 8 short of it and 24 short (but for the narrowest)
for w, k in [(128, 2064), (144, 2064), (160, 2064), (176, 3088), (192, 4112), (208, 2064), (224, 2064), (240, 2064)]:
    CASES += [((PAIR, w, 1), 20003, 2 * w, k, 0), ((PAIR, w, 1), 20003, 2 * w - (24 if w > 128 else 8), k, 0), ((PAIR, w, 1), 20003, 2 * w - 8, k, 5)]
CASES += [((PAIR, 240, 1), 40000, 680, 1040, 0), ((PAIR, 240, 1), 40000, 680, 2064, 5)]       # seven tiles a pair


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("cut,m,n,k,experts", CASES)
def test_the_case_is_for_this_kernel(cut, m, n, k, experts, act):
    from paper_2405_10951_b200 import binding as Bd
    assert Bd.bsr_e4m3_block128_cut(m, n, k, experts, act) == cut
    if cut[0] != CLUSTER:                                              # workers of 148 SMs walk several tiles
        rows, workers = (256, 74) if cut[0] == PAIR else (128, 148)
        assert -(-m // rows) * -(-n // cut[1]) > workers


def test_sizes_that_a_product_refuses():
    from paper_2405_10951_b200 import binding as Bd
    for bad in [(0, 8, 16, 0, 0), (4, 12, 16, 0, 0), (4, 8, 24, 0, 0), (4, 8, 1 << 25, 0, 0), (4, 8, 16, 1025, 0), (4, 8, 16, -1, 0), (4, 8, 16, 0, 3)]:
        with pytest.raises(Bd.BsrError) as e:
            Bd.bsr_e4m3_block128_cut(*bad)
        assert e.value.status == -1
    assert Bd.lib().bsr_e4m3_block128_cut(4, 8, 16, 0, 0, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("cut,m,n,k,experts", CASES)
def test_product_by_kernel(cut, m, n, k, experts, act):
    """Rows are compared by sample: every 50th, the ends, and those beside a segment's ends; all columns."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    assert Bd.bsr_e4m3_block128_cut(m, n, k, experts, act) == cut
    rng = np.random.default_rng(m + n + k + experts + act)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + n + k + act)
    stack = (experts, n, k) if experts else (n, k)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    size = lambda *s: torch.exp2(torch.randint(-6, 7, s, generator=gen, device="cuda").float())
    x = normal(m, k) * size(m, -(-k // 128)).repeat_interleave(128, 1)[:, :k]
    w = normal(*stack) / k ** 0.5 * size(*stack[:-2], -(-n // 128), -(-k // 128)).repeat_interleave(128, -1).repeat_interleave(128, -2)[..., :n, :k]
    bias = normal(*stack[:-1])
    xq, xs = Bd.bsr_quantize_e4m3_rows128(x)
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(w)
    del x, w
    z0, y0 = normal(m, n).bfloat16(), torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda")
    z = z0.clone() if act else None
    ends = np.array([0, m], np.int32)
    if experts:
        ends = np.concatenate([[0], np.sort(rng.integers(0, m - 40, experts))]).astype(np.int32)     # uneven, rows behind the last
        y = Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, torch.as_tensor(ends).cuda(), bias, act=act, z=z, y=y0.clone())
        assert torch.equal(y[int(ends[-1]):], y0[int(ends[-1]):])
        assert not act or torch.equal(z[int(ends[-1]):], z0[int(ends[-1]):])
    else:
        y = Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq, ws, bias, act=act, z=z, y=y0.clone())
    near = np.concatenate([ends + d for d in range(-3, 4)])
    pick = np.unique(np.concatenate([np.arange(0, m, 50), np.arange(min(m, 140)), np.arange(max(0, m - 140), m), near[(near >= 0) & (near < m)]]))
    at = torch.as_tensor(pick).cuda()
    wide = base.wide
    X, Y, Z, Z0 = P.dequantize(wide(xq[at]), xs[at].cpu().numpy(), 1), wide(y[at]), None if z is None else wide(z[at]), wide(z0[at])
    for e in range(len(ends) - 1):
        rows = (pick >= ends[e]) & (pick < ends[e + 1])
        if not rows.any():
            continue
        one = (lambda t: t[e]) if experts else (lambda t: t)
        W, b = P.dequantize(wide(one(wq)), one(ws).cpu().numpy(), 128), wide(one(bias))
        part, mag = X[rows] @ W.T + b, np.abs(X[rows]) @ np.abs(W).T + np.abs(b)
        base.check(Y[rows], None if Z is None else Z[rows], act, part, mag, Z0[rows], k)
