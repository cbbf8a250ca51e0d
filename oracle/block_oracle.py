"""Plain definitions in 64 bits (numpy) of what stands around the experts: dropout from a counter, norms with their gradients, the sequences' balance
loss and z loss.  Written from the definitions in include/moe_hip.h; shares no code with the library."""
from __future__ import annotations

import numpy as np

_LOW = (1 << 32) - 1


def philox(counter, key):
    """Philox4x32-10: four words of a counter (whole numbers or arrays of them) and two of a key -> four words."""
    c = [np.asarray(x, dtype=object) for x in counter]
    k = list(key)
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & _LOW, (p >> 32) ^ c[3] ^ k[1], p & _LOW]
        k = [(k[0] + 0x9E3779B9) & _LOW, (k[1] + 0xBB67AE85) & _LOW]
    return c


def _philox_fast(c0, c1, c2, c3, k0, k1):
    """The same on arrays of uint64 (a product of 32-bit words fits)."""
    w, s = np.uint64(_LOW), np.uint64(32)
    c = [np.asarray(x, dtype=np.uint64) for x in (c0, c1, c2, c3)]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> s) ^ c[1] ^ np.uint64(k0), q & w, (p >> s) ^ c[3] ^ np.uint64(k1), p & w]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return c


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def keep(n_rows, cols, p, seed, step, site, row0=0):
    """The mask of rows row0 .. row0 + n_rows - 1."""
    blocks = (cols + 7) // 8
    shape = (n_rows, blocks)
    full = lambda x: np.broadcast_to(np.asarray(x, dtype=np.uint64), shape)  # noqa: E731
    words = _philox_fast(full(np.arange(blocks) + (site << 16)), full(row0 + np.arange(n_rows)[:, None]), full(step & _LOW), full(step >> 32 & _LOW), seed & _LOW,
                         seed >> 32 & _LOW)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 2)
    return halves.reshape(n_rows, 8 * blocks)[:, :cols] >= threshold(p)


def scale(p):
    return 65536.0 / (65536 - threshold(p))


def dropout(x, mask, p, r=None):
    y = np.where(mask, x, 0.0) * scale(p)
    return y if r is None else np.where(mask, y + r, r)


def norm_fwd(z, w, b, kind, eps):
    """y, mean, rstd, h."""
    d = z.shape[1]
    mean = z.sum(1) / d if kind == "layer" else np.zeros(len(z))
    c = z - mean[:, None]
    rstd = 1 / np.sqrt((c * c).sum(1) / d + eps)
    h = c * rstd[:, None]
    y = h * w if w is not None else h.copy()
    return (y if b is None else y + b), mean, rstd, h


def norm_bwd(dy, h, rstd, w, kind):
    """The gradient of z (without what reaches it otherwise), dw, db."""
    d = dy.shape[1]
    g = dy * w if w is not None else dy
    dz = g - h * ((g * h).sum(1) / d)[:, None]
    if kind == "layer":
        dz = dz - (g.sum(1) / d)[:, None]
    return dz * rstd[:, None], (dy * h).sum(0), dy.sum(0)


def shares(logits, gate):
    """Softmax, scores, shares and lse of every row; a row of nothing but -inf has zeros."""
    m = logits.max(1, keepdims=True)
    some = np.isfinite(m)
    e = np.where(some, np.exp(logits - np.where(some, m, 0.0)), 0.0)
    total = e.sum(1, keepdims=True)
    soft = np.where(some, e / np.where(some, total, 1.0), 0.0)
    lse = np.where(some, m + np.log(np.where(some, total, 1.0)), 0.0)[:, 0]
    if gate == "softmax":
        return soft, soft, soft, lse
    with np.errstate(over="ignore"):
        score = 1 / (1 + np.exp(-logits))
    total = score.sum(1, keepdims=True)
    return soft, score, np.where(total > 0, score / np.where(total > 0, total, 1.0), 0.0), lse


def seq_loss(logits, topk, ranges, k, gate, alpha, beta):
    """counts, P, (balance, z), dlogits of their sum, over the token ranges [(from, to)] of the sequences."""
    T, E = logits.shape
    S = len(ranges)
    filled, tokens = sum(b > a for a, b in ranges), sum(b - a for a, b in ranges)
    counts, P, dz = np.zeros((S, E), dtype=np.int64), np.zeros((S, E)), np.zeros((T, E))
    balance = z = 0.0
    for s, (a, b) in enumerate(ranges):
        if b <= a:
            continue
        n = b - a
        soft, score, share, lse = shares(logits[a:b], gate)
        ids = topk[a:b].reshape(-1)
        counts[s] = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
        P[s] = share.sum(0) / n
        f = counts[s] / (k * n)
        balance += alpha / filled * E * (f * P[s]).sum()
        z += beta / tokens * (lse ** 2).sum()
        up = alpha / filled * E * f / n
        inner = up - (share * up).sum(1, keepdims=True)
        dz[a:b] = share * inner * (1 - score if gate == "sigmoid" else 1.0) + 2 * beta / tokens * lse[:, None] * soft
    return counts, P, np.array([balance, z]), dz
