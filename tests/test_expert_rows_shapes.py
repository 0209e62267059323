"""Row kernels of an expert layer at shapes that change how a row is shared out: the longest rows, and rows of odd lengths at many tokens."""
import numpy as np
import pytest

import expert_plain as P

FP32_HALF = 2.0 ** -24
gpu = pytest.mark.gpu


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


@gpu
@pytest.mark.parametrize("dtype,dim", [("bfloat16", 1032), ("float32", 1028), ("float32", 516), ("bfloat16", 2056), ("bfloat16", 520)])
@pytest.mark.parametrize("tokens,top_k", [(2368, 3), (4800, 2)])
def test_combine_gradient_of_odd_rows_and_many_tokens(tokens, top_k, dtype, dim):
    """One chunk more than 4, 2 or 8 warps share evenly, and tokens enough to give each fewer warps."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    chunks = dim // (4 if dtype == "float32" else 8)
    warps = 1 if chunks <= 64 else 2 if chunks <= 128 else 4 if chunks <= 256 else 8
    lanes = lambda w: 32 * w * -(-chunks // (32 * w))
    assert warps > 1 and tokens * warps >= 32 * 148 and lanes(warps) * 9 > lanes(1) * 10          # the rule that is meant
    rng = np.random.default_rng(tokens + dim)
    expert, w = P.routing(rng, tokens, top_k, 7, masked=0.2)
    pos, _ = P.sort(expert, 7)
    to = lambda a: torch.as_tensor(a.astype(np.float32)).cuda().to(getattr(torch, dtype))
    rows, dout, drows0 = to(rng.standard_normal((tokens * top_k, dim))), to(rng.standard_normal((tokens, dim))), to(rng.standard_normal((tokens * top_k, dim)))
    drows, dw = Bd.bsr_expert_combine_backward(dout, rows, torch.as_tensor(pos).cuda(), torch.as_tensor(w).cuda(), drows=drows0.clone())
    want, want_dw, mag = P.combine_backward(wide(dout), wide(rows), pos, w, wide(drows0))
    half = FP32_HALF if dtype == "float32" else 2.0 ** -8
    assert np.all(np.abs(wide(drows) - want) <= (half + FP32_HALF) * 1.01 * np.abs(want))
    # a lane's chain of multiply-adds over its share of the row, additions over lanes and warps
    assert np.all(np.abs(wide(dw) - want_dw) <= (dim / 32 + 16 + 5 + 8) * FP32_HALF * mag)
    assert np.all(wide(dw)[pos < 0] == 0)


@gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_longest_rows(dtype):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    dim, t = 1 << 25, getattr(torch, dtype)
    pos = torch.tensor([[3, -1], [0, 1]], dtype=torch.int32, device="cuda")
    x = (torch.arange(2 * dim, device="cuda").view(2, dim) % 251 - 125).to(t)                     # whole numbers that bf16 holds
    rows = Bd.bsr_expert_scatter(x, pos, rows=torch.full((4, dim), 7.0, dtype=t, device="cuda"))
    assert torch.equal(rows, torch.stack([x[1], x[1], torch.full_like(x[0], 7.0), x[0]]))
    w = torch.tensor([[0.5, 9.0], [0.25, 0.75]], device="cuda")
    assert torch.equal(Bd.bsr_expert_combine(rows, pos, w), torch.stack([x[0] / 2, x[1]]))
    drows, dw = Bd.bsr_expert_combine_backward(x, rows, pos, w, drows=torch.full_like(rows, 7.0))
    assert torch.equal(drows[:2], torch.stack([(x[1].float() / 4).to(t), (x[1].float() * 0.75).to(t)])) and torch.equal(drows[3], (x[0].float() / 2).to(t)) and bool((drows[2] == 7).all())
    # eight warps walk a row: each lane's chain of multiply-adds has 2^25 / 256 terms, then come the additions over lanes and warps
    want = (x.double() ** 2).sum(1)
    got = dw.double()
    assert got[0, 1] == 0
    steps = dim / 256 + 16
    for a, b in [(got[0, 0], want[0]), (got[1, 0], want[1]), (got[1, 1], want[1])]:
        assert abs(float(a - b)) <= steps * FP32_HALF * float(b)
