"""Sizes that the calls of an expert layer refuse.  Nothing of these calls reaches a device."""
import pytest

A = 4096                     # an aligned address, never read: the arguments are checked first


def status(name, *args):
    from paper_2405_10951_b200 import binding as Bd
    return getattr(Bd.lib(), name)(*args)


@pytest.mark.parametrize("dim", [(1 << 25) + 16, 1 << 26, (1 << 31) - 16])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_too_long_for_a_grid_are_refused(dtype, dim):
    """A row's parts lie along the grid's second axis (65535 at most), and a lane walks its columns in 32 bits: within 2048 of 2^31 the
    combination's gradient would step past the end to negative columns."""
    assert status("bsr_expert_scatter", A, dtype, 1, dim, 1, A, A, None) == -1
    assert status("bsr_expert_combine", A, dtype, A, A, A, A, 1 - dtype, 1, dim, 1, None) == -1
    assert status("bsr_expert_combine_backward", A, dtype, A, 1 - dtype, A, A, A, A, 1, dim, 1, None) == -1


@pytest.mark.parametrize("chunk,threads", [(4, 1024), (8, 2048)])
def test_the_longest_row_fits(chunk, threads):
    """The kernels' own arithmetic at the longest row: parts of at most 256 chunks, columns of the last step of eight warps."""
    chunks = -(-(1 << 25) // chunk)
    assert -(-chunks // 256) <= 65535
    assert (1 << 25) + threads < 1 << 31


@pytest.mark.parametrize("k", [(1 << 24) + 16, 1 << 28, 1 << 30])
def test_sums_longer_than_a_wait_are_refused(k):
    """A warp waits for a whole tile's sums, two seconds at most: about 0.37 us a slab of 128 values is 3.1 s at k = 2^30."""
    assert status("bsr_linear_forward_e4m3_block128", A, A, A, A, None, None, A, 8, 8, k, 0, None) == -1
    assert status("bsr_expert_linear_e4m3_block128", A, A, A, A, None, A, None, A, 8, 8, k, 1, 0, None) == -1


def test_the_longest_sum_is_far_inside_a_wait():
    assert (1 << 24) / 128 * 0.37e-6 < 2.0 / 40


@pytest.mark.gpu
def test_quantised_rows_up_to_the_last_block_of_31_bits():
    """k within 127 of 2^31: the number of blocks along k does not pass 31 bits on the way."""
    import torch
    from paper_2405_10951_b200 import binding as Bd
    k = (1 << 31) - 16
    w = torch.zeros((1, k), dtype=torch.bfloat16, device="cuda")
    w[0, k - 1], w[0, k - 112], w[0, k - 113], w[0, 5] = 448.0, 3.0, -896.0, 1.0
    for q, scale in (Bd.bsr_quantize_e4m3_blocks128(w), Bd.bsr_quantize_e4m3_rows128(w)):
        assert scale.shape == (1, 1 << 24)
        at = [0, 1, (1 << 24) - 3, (1 << 24) - 2, (1 << 24) - 1]
        assert scale[0, at].tolist() == [119, 127, 127, 128, 127]
        code = q.view(torch.uint8)[0, [5, k - 113, k - 112, k - 1]]
        assert code.view(torch.float8_e4m3fn).float().tolist() == [256.0, -448.0, 3.0, 448.0]
        del q, scale


@pytest.mark.gpu
def test_the_longest_sum_is_there():
    import torch
    from paper_2405_10951_b200 import binding as Bd
    m, n, k = 9, 16, 1 << 24
    x = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    for row in range(m):
        x[row, row * 1000 + 7] = 2.0
        x[row, k - 1 - row * 130] = -(row + 4.0)
    w = torch.ones((1, n, k), dtype=torch.bfloat16, device="cuda")
    w[0, 3, k // 2:] = 0.5
    xq, xs = Bd.bsr_quantize_e4m3_rows128(x)
    wq, ws = Bd.bsr_quantize_e4m3_blocks128(w)
    want = torch.tensor([[2.0 - (row + 4.0) * (0.5 if col == 3 else 1.0) for col in range(n)] for row in range(m)], device="cuda")     # exact in bf16
    Bd.bsr_standalone_status()
    seg = torch.tensor([0, m], dtype=torch.int32, device="cuda")
    assert Bd.bsr_e4m3_block128_cut(m, n, k)[2] == 8 and Bd.bsr_e4m3_block128_cut(m, n, k, 1)[2] == 1      # k over a cluster, and not
    for y in (Bd.bsr_linear_forward_e4m3_block128(xq, xs, wq[0], ws[0]), Bd.bsr_expert_linear_e4m3_block128(xq, xs, wq, ws, seg)):
        assert torch.equal(y.float(), want)
    Bd.bsr_standalone_status()
