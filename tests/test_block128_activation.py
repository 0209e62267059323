"""GELU and its derivative in products of 8-bit blocks, value by value: the operands are zero, so that the bias alone is what is activated."""
import numpy as np
import pytest

import expert_plain as P

# The tail Phi(-t) = exp(-t^2 / 2) R(t).  R's fit is within 1.1e-5 of its value.  The exponential's argument t^2 / 2 log2(e) is rounded twice, and its
# constant once: t^2 / 2 * 3 * 2^-24.  Nine operations of at most 2^-22 each.  An exponential below 2^-126 is flushed.
FIT = 1.1e-5


def tail_off(t):
    return 2.0 ** -126 + (FIT + t * t * 2.0 ** -23 + 9 * 2.0 ** -22) * P.phi(-t)


def half_step(v):
    return np.ldexp(0.5, np.maximum(np.frexp(v)[1] - 1, -126) - 7)


def points(n):
    rng = np.random.default_rng(n)
    z = rng.uniform(-5.5, 5.5, n)
    z[::7] = np.ldexp(z[::7], rng.integers(-20, 2, len(z[::7])))          # small ones, and some as far as the exponential goes
    z[:12] = [0.0, -0.0, 1e-30, -1e-30, -13.1, -13.3, 13.1, -16.0, 16.5, -40.0, 1e20, -1e20]
    return z.astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(2, 160000, 16), (1, 4096, 1024), (300, 4096, 16)])       # a CTA a tile; k over a cluster; many rows
def test_gelu(m, n, k):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    bias = points(n)
    x = Bd.bsr_quantize_e4m3_rows128(torch.zeros((m, k), device="cuda"))
    w = Bd.bsr_quantize_e4m3_blocks128(torch.ones((n, k), device="cuda"))
    z = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    y = Bd.bsr_linear_forward_e4m3_block128(*x, *w, torch.as_tensor(bias).cuda(), act=Bd.ACT_GELU, z=z)
    assert torch.equal(z, torch.as_tensor(bias).cuda().bfloat16().expand(m, n))
    assert torch.equal(y, y[:1].expand(m, n))
    got, v = y[0].float().cpu().numpy().astype(np.float64), bias.astype(np.float64)
    t = np.abs(v)
    want = np.maximum(v, 0.0) - t * P.phi(-t)
    off = half_step(want) + t * tail_off(t) + 2.0 ** -23 * np.abs(want)
    bad = np.abs(got - want) > off
    assert not bad.any(), (bad.sum(), v[bad][:5], got[bad][:5], want[bad][:5])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(2, 160000, 16), (1, 4096, 1024), (300, 4096, 16)])
def test_gelu_derivative(m, n, k):
    import torch
    from paper_2405_10951_b200 import binding as Bd
    g = np.random.default_rng(k).uniform(0.5, 2.0, n).astype(np.float32)
    zt = torch.as_tensor(points(n)).bfloat16()
    x = Bd.bsr_quantize_e4m3_rows128(torch.zeros((m, k), device="cuda"))
    w = Bd.bsr_quantize_e4m3_blocks128(torch.ones((n, k), device="cuda"))
    y = Bd.bsr_linear_forward_e4m3_block128(*x, *w, torch.as_tensor(g).cuda(), act=Bd.ACT_GELU_GRAD, z=zt.cuda().expand(m, n).contiguous())
    assert torch.equal(y, y[:1].expand(m, n))
    got, v = y[0].float().cpu().numpy().astype(np.float64), zt.float().numpy().astype(np.float64)
    t = np.abs(v)
    peak = t * np.exp(-0.5 * t * t) / np.sqrt(2.0 * np.pi)
    want = g * P.gelu_grad(v)
    # two terms of either sign: Phi (1 - the tail above zero) and z phi, whose exponential is the tail's
    off = half_step(want) + g * (tail_off(t) + 2.0 ** -126 * t + (t * t * 2.0 ** -23 + 9 * 2.0 ** -22) * peak + 2.0 ** -22 * (P.phi(v) + peak)) + 2.0 ** -23 * np.abs(want)
    bad = np.abs(got - want) > off
    assert not bad.any(), (bad.sum(), v[bad][:5], got[bad][:5], want[bad][:5])
