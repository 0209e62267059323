"""The operators of an expert layer in 64 bits, from their definitions (numpy; shared by the tests)."""
import math

import numpy as np


def sort(expert, experts):
    """(pos, seg_start): slots in the order of (expert, token, slot), -1 without an expert."""
    flat = expert.reshape(-1)
    pos = np.full(flat.shape, -1, np.int32)
    seg = np.zeros(experts + 1, np.int32)
    at = 0
    for e in range(experts):
        mine = np.nonzero(flat == e)[0]
        pos[mine] = np.arange(at, at + len(mine))
        at += len(mine)
        seg[e + 1] = at
    return pos.reshape(expert.shape), seg


def scatter(x, pos, rows):
    out = rows.copy()
    for t, s in zip(*np.nonzero(pos >= 0)):
        out[pos[t, s]] = x[t]
    return out


def combine(rows, pos, weights, residual):
    """(sum, sum of magnitudes)"""
    tokens, top_k = pos.shape
    out = np.zeros((tokens, rows.shape[1])) if residual is None else residual.astype(np.float64).copy()
    mag = np.abs(out)
    for t, s in zip(*np.nonzero(pos >= 0)):
        term = (1.0 if weights is None else float(weights[t, s])) * rows[pos[t, s]].astype(np.float64)
        out[t] += term
        mag[t] += np.abs(term)
    return out, mag


def combine_backward(dout, rows, pos, weights, drows):
    drows, dw, mag = drows.astype(np.float64).copy(), np.zeros(pos.shape), np.zeros(pos.shape)
    for t, s in zip(*np.nonzero(pos >= 0)):
        drows[pos[t, s]] = float(weights[t, s]) * dout[t]
        dw[t, s] = np.dot(dout[t], rows[pos[t, s]])
        mag[t, s] = np.dot(np.abs(dout[t]), np.abs(rows[pos[t, s]]))
    return drows, dw, mag


def stride(k):
    return 4 * -(-k // 512)


def exponent(v):
    """The least e >= -127 with max|v| <= 448 * 2^e over the finite values, 0 for zeros."""
    v = np.abs(v[np.isfinite(v)])
    top = v.max() if v.size else 0.0
    if top == 0.0:
        return 0
    e = math.frexp(top)[1] - 12
    while top > math.ldexp(448.0, e):
        e += 1
    return max(e, -127)


def e4m3(u):
    """Nearest E4M3 values, ties to even (|u| <= 448); NaN for what is not finite."""
    out = np.full(u.shape, np.nan)
    fine = np.isfinite(u)
    x = u[fine]
    step = np.ldexp(1.0, np.maximum(np.frexp(x)[1] - 1, -6) - 3)
    out[fine] = np.round(x / step) * step                # numpy rounds halves to even
    return out


def quantize(v, rows_per_block):
    """Codes' values and scale bytes of a matrix in blocks of rows_per_block x 128."""
    n, k = v.shape
    nb, kb = -(-n // rows_per_block), -(-k // 128)
    q, b = np.zeros((n, k)), np.full((nb, stride(k)), 127, np.uint8)
    for i in range(nb):
        for j in range(kb):
            at = np.s_[i * rows_per_block:(i + 1) * rows_per_block, j * 128:(j + 1) * 128]
            e = exponent(v[at])
            b[i, j] = e + 127
            q[at] = e4m3(np.ldexp(v[at].astype(np.float64), -e))
    return q, b


def dequantize(q, b, rows_per_block):
    n, k = q.shape
    e = np.repeat(np.repeat(b.astype(np.int64) - 127, rows_per_block, 0)[:n], 128, 1)[:, :k]
    return np.ldexp(q.astype(np.float64), e)


def phi(z):
    """The normal distribution function, its lower tail included."""
    return 0.5 * np.vectorize(math.erfc, otypes=[float])(-z / math.sqrt(2.0))


def gelu(z):
    return z * phi(z)


def gelu_grad(z):
    return phi(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def routing(rng, tokens, top_k, experts, masked=0.0):
    """Distinct experts a token (as far as there are any), some tokens without; weights that add up to one."""
    order = np.argsort(rng.standard_normal((tokens, experts)) + np.linspace(1.5, 0.0, experts), axis=1)[:, ::-1]
    expert = np.ascontiguousarray(order[:, np.arange(top_k) % experts].astype(np.int32))
    expert[rng.random(tokens) < masked] = -1
    w = rng.random((tokens, top_k)) + 0.1
    return expert, (w / w.sum(1, keepdims=True)).astype(np.float32)
