"""Segments that are not as the sort writes them."""
import numpy as np
import pytest

import expert_plain as P


@pytest.mark.gpu
@pytest.mark.parametrize("ends", [[0, 100, 50, 80], [0, 300, 20, 10, 200], [90, 60, 30, 0], [0, 200, 200, 0, 200]])
def test_a_segment_ends_where_a_later_one_begins(ends):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    rng = np.random.default_rng(len(ends) + ends[1])
    m, n, k, experts = 200, 72, 144, len(ends) - 1
    wide = lambda t: t.float().cpu().numpy().astype(np.float64)
    xq, xs = Bd.bsr_quantize_e4m3_rows128(torch.as_tensor(rng.standard_normal((m, k)).astype(np.float32)).cuda())
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(torch.as_tensor(rng.standard_normal((experts, n, k)).astype(np.float32)).cuda())
    y = wide(Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, torch.tensor(ends, dtype=torch.int32, device="cuda"), y=torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda")))
    x, at = P.dequantize(wide(xq), xs.cpu().numpy(), 1), np.clip(ends, 0, m)
    owner = np.full(m, -1)
    for e in range(experts):
        owner[at[e:].min():at[e + 1:].min()] = e
    assert np.all(y[owner < 0] == 7.0)
    for e in np.unique(owner[owner >= 0]):
        w, rows = P.dequantize(wide(wq[e]), ws[e].cpu().numpy(), 128), owner == e
        part, mag = x[rows] @ w.T, np.abs(x[rows]) @ np.abs(w).T
        # k / 32 instructions, each of which drops what is below 2^-23 of the sum of magnitudes; one rounding to bf16
        acc = (k / 32 + 2) * 2.0 ** -23 * mag
        assert np.all(np.abs(y[rows] - part) <= acc + 2.0 ** -8 * 1.01 * (np.abs(part) + acc))
