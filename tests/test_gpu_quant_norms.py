"""The backward pass of the block-scaled experts in the 2-norm, against bounds that a loss of accuracy by two would pass.

Rounding to bf16 is uniform in half a step: 2^-8 / sqrt(3) of the smallest value of a binade, so at most that of any tensor's norm (2.3e-3).  To it comes what the sums
of dH move: off by the deviation s = 1.5e-5 of their terms' 2-norm (calls of few values: 2^-22, a few roundings of fp32) times the derivative, a value of dG or dU
crosses the border of a rounding with the probability (2 / pi)^(1/2) s / step, and is then off by a step: the sum of probability times step^2 over all values is the
square that this adds, relative to that of the values, as random directions add up.  Values are few where they are large, so twice the root of it is allowed."""
import numpy as np
import pytest

from oracle import quant_oracle as qo

from .test_gpu_quant import EXPERTS, TALL, Layer, np_of, rel

pytestmark = pytest.mark.gpu
ROUNDING = 2.0 ** -8 / np.sqrt(3)


def added(parts):
    """The relative norm of what is moved: parts are (values, deviations, steps)."""
    moved = sum(float((np.minimum(np.sqrt(2 / np.pi) * s / step, 1) * step ** 2).sum()) for _, s, step in parts)
    return np.sqrt(moved / sum(float((v ** 2).sum()) for v, _, _ in parts))


def steps(v, bits, floor=0.0):
    return np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 1e-300))) - bits), np.maximum(floor, 1e-300))


def smallest(v):
    """2^-9 of the 2^e of each value's block of 128."""
    pad = np.pad(np.abs(v), ((0, 0), (0, -v.shape[1] % 128)))
    return pad.reshape(len(v), -1, 128).max(2).repeat(128, 1)[:, :v.shape[1]] * 2.0 ** -9 / 224


@pytest.mark.parametrize("case", [c for c in EXPERTS + TALL if c[0] * c[2] * min(c[3], c[4]) >= 1 << 13])
def test_backward(case):
    L = Layer(*case)
    L.forward()
    L.backward()
    G, U, H = (np_of(t) for t in (L.G, L.U, L.H))
    w = L.wr if L.gather else None
    dX, dG, dU = qo.experts_bwd(L.dyv, w, G, U if L.gated else None, L.bounds, *L.values)
    e = 2.0 ** -22 if L.n * L.shape.d_ff <= 1 << 16 else 1.5e-5
    t = e * np.sqrt(qo.grouped(L.dyv ** 2, L.bounds, [np.ascontiguousarray((x * x).T) for x in L.values[2]])) * (1 if w is None else np.abs(w)[:, None])
    if L.gated:
        s = 1 / (1 + np.exp(-G))
        pairs = [(dG, t * np.abs(U * (s + G * s * (1 - s)))), (dU, t * np.abs(G * s))]
    else:
        pairs = [(dG, t * np.abs(qo._phi(G) + G * np.exp(-G * G / 2) / np.sqrt(2 * np.pi)))]
    # (the hardware's exponential and reciprocal, and erf's approximation: 2^-18 of a value)
    pairs = [(v, np.hypot(d, 2.0 ** -18 * v)) for v, d in pairs]
    eight, sixteen = added([(v, d, steps(v, 3, smallest(v))) for v, d in pairs]), [added([(v, d, steps(v, 7))]) for v, d in pairs]
    assert rel(np_of(L.dX), dX) <= np.hypot(ROUNDING, 2 * eight)
    Xp, dYp = np_of(L.Xp), np_of(L.dYp)
    counts = np.diff(L.bounds)
    own = [np.concatenate([np_of(x[i]).ravel() for i in range(int((counts > 0).sum()))]) if x is not None else None for x in L.dW]
    product = lambda a, b: np.concatenate([(a[x:y].T @ b[x:y]).ravel() for x, y in zip(L.bounds, L.bounds[1:]) if y > x])
    assert rel(own[0], product(Xp, dG)) <= np.hypot(ROUNDING, 2 * sixteen[0])
    if L.gated:
        assert rel(own[1], product(Xp, dU)) <= np.hypot(ROUNDING, 2 * sixteen[1])
    assert rel(own[2], product(H, dYp)) <= ROUNDING
