"""Plain definitions of the block-scaled 8-bit operators in 64 bits (numpy): quantisation, grouped products, the experts' two passes
and the clipped norm.  Written from the definitions in include/moe_hip.h; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def _table():
    """The values of codes 0 .. 126, ascending (127 is NaN)."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


VALUES = _table()


def decode(codes):
    c = np.asarray(codes).astype(np.int64)
    v = np.append(VALUES, math.nan)[c & 127]
    return np.where(c & 128, -v, v)


def encode(x):
    """Nearest code, ties to the even one; magnitudes up to 448."""
    a = np.abs(x)
    mid = 0.5 * (VALUES[1:] + VALUES[:-1])   # between code i and i + 1
    lo = np.searchsorted(mid, a, side="left")    # a tie goes down ..
    hi = np.searchsorted(mid, a, side="right")   # .. or up
    c = np.where(lo % 2 == 0, lo, hi)
    c = np.where(np.isfinite(x), c, 127)
    return (c | np.where(np.signbit(x) & np.isfinite(x), 128, 0)).astype(np.uint8)


def exponent(a):
    """The smallest whole e >= -126 with a <= 448 * 2^e; 0 for a = 0."""
    if a == 0:
        return 0
    m, p = math.frexp(a)          # a = m 2^p, 448 = 0.875 * 2^9
    return max(p - 9 if m <= 0.875 else p - 8, -126)


def _pad(n):
    return -(-n // BLOCK) * BLOCK


def _exponents(amax):
    return np.vectorize(exponent, otypes=[np.int64])(amax)


def quant_rows(x):
    """codes [n, pad], exponent bytes [n, pad / 128] of x [n, cols] in 64 bits."""
    x = np.asarray(x, np.float64)
    n, cols = x.shape
    b = np.zeros((n, _pad(cols)))
    b[:, :cols] = x
    b = b.reshape(n, -1, BLOCK)
    e = _exponents(np.where(np.isfinite(b), np.abs(b), 0).max(2)) if n else np.zeros((0, b.shape[1]), np.int64)
    with np.errstate(invalid="ignore"):
        q = encode(np.ldexp(b, -e[:, :, None]))
    return q.reshape(n, -1), (e + 127).astype(np.uint8)


def quant_matrix(w):
    """codes [K, pad(N)] (of the stored rows) and exponent bytes [K / 128, N / 128] of w [K, N]."""
    w = np.asarray(w, np.float64)
    K, N = w.shape
    b = np.zeros((_pad(K), _pad(N)))
    b[:K, :N] = w
    t = b.reshape(_pad(K) // BLOCK, BLOCK, _pad(N) // BLOCK, BLOCK)
    e = _exponents(np.where(np.isfinite(t), np.abs(t), 0).max((1, 3)))
    with np.errstate(invalid="ignore"):
        q = encode(np.ldexp(t, -e[:, None, :, None]))
    return q.reshape(_pad(K), _pad(N))[:K], (e + 127).astype(np.uint8)


def values(q, s, per=1):
    """64-bit values of codes [n, pad] with exponent bytes [n / per, pad / 128]."""
    e = np.repeat(np.repeat(s.astype(np.int64) - 127, BLOCK, 1), per, 0)[:q.shape[0]]
    return np.ldexp(decode(q), e)


def quantised(x):
    """The values that quantised rows stand for."""
    q, s = quant_rows(x)
    return values(q, s)[:, :x.shape[1]]


def quantised_matrix(w):
    q, s = quant_matrix(w)
    return values(q, s, BLOCK)[:, :w.shape[1]]


def bf16(x):
    """Nearest bfloat16, ties to even, of 64-bit values in its normal range."""
    m, p = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), p - 8)


def grouped(rows, offsets, matrices):
    """rows of group g times matrices[g] [K, N]; rows of no group are zero."""
    out = np.zeros((rows.shape[0], matrices[0].shape[1]))
    for g, w in enumerate(matrices):
        out[offsets[g]:offsets[g + 1]] = rows[offsets[g]:offsets[g + 1]] @ w
    return out


def _sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def _phi(z):
    return 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-z / math.sqrt(2))


def experts_fwd(x, offsets, Wg, Wu, Wd, quant_h=True):
    """x [n, d] and the matrices are the values used; quant_h: H is rounded to bf16 and quantised before the down product."""
    G = grouped(x, offsets, Wg)
    U = grouped(x, offsets, Wu) if Wu is not None else None
    H = G * _sigmoid(G) * U if U is not None else G * _phi(G)
    return G, U, H, grouped(quantised(bf16(H)) if quant_h else H, offsets, Wd)


def experts_bwd(dy, row_w, G, U, offsets, Wg, Wu, Wd, quant_g=True):
    """dX, dG and dU from the values dy [n, d] (times row_w), the saved G and U, and the matrices used."""
    t = [np.ascontiguousarray(w.T) for w in Wd]
    dH = grouped(dy, offsets, t) * (1 if row_w is None else row_w[:, None])
    if U is not None:
        s = _sigmoid(G)
        dU, dG = dH * G * s, dH * U * (s + G * s * (1 - s))
    else:
        dU, dG = None, dH * (_phi(G) + G * np.exp(-G * G / 2) / math.sqrt(2 * math.pi))
    if quant_g:
        dG, dU = bf16(dG), bf16(dU) if dU is not None else None
    use = quantised if quant_g else (lambda v: v)
    dX = grouped(use(dG), offsets, [w.T for w in Wg])
    if dU is not None:
        dX = dX + grouped(use(dU), offsets, [w.T for w in Wu])
    return dX, dG, dU


def clip(grads, max_norm):
    """The norm and the clipped values of a list of arrays, as (float, list)."""
    norm = math.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    f = min(1.0, max_norm / (norm + 1e-6))
    return norm, [g.astype(np.float64) * f for g in grads]
