"""The sequences' losses behind a sigmoid gate of confident logits, whose gradient has the factor 1 - score: against the 64-bit definition, relative to that factor.

Tolerances, u = 2^-24, |logit| up to 25: the exponential is off by 1.5 * 25 + 2 < 40 u of itself, the reciprocal by 2 u, so score and 1 - score (a product where the score is above
1/2, a difference without cancellation below) by 44 u of themselves; a share by 44 + 12 for the sum's additions + 44 for its terms + 4 for the division < 110 u.  dz = share (up -
sum share up) (1 - score): the bracket is off by (110 + 12 + 8) u of up + sum share up, the products by 110 + 44 + 4 u: 320 u of share (up + sum share up) (1 - score)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64
from tests.test_gpu_seq_nan import run

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("E,k", [(4, 1), (13, 2), (64, 6), (200, 8), (600, 4), (1000, 8)])
@pytest.mark.parametrize("low,high", [(12.0, 20.0), (16.0, 25.0), (-25.0, -12.0), (-25.0, 25.0)])
def test_confident_scores(E, k, low, high):
    T, alpha = 150, 0.01
    g = torch.Generator().manual_seed(E)
    x = low + (high - low) * torch.rand(T, E, generator=g)
    topk = torch.topk(x, k, dim=1).indices.int()
    start, length = [0, 40], [35, 110]
    ranges = [(0, 35), (40, 150)]
    counts, P, loss, coef, dlogits = run(x.cuda(), topk.cuda(), start, length, "sigmoid", alpha, 0.0)
    c64, P64, _, dz = ob.seq_loss(np64(x), topk.numpy(), ranges, k, "sigmoid", alpha, 0.0)
    assert np.array_equal(counts.cpu().numpy(), c64)
    x64 = np64(x)
    share = ob.shares(x64, "sigmoid")[2]
    up, rest = np.zeros((T, E)), np.exp(-x64) / (1 + np.exp(-x64))
    for s, (a, b) in enumerate(ranges):
        up[a:b] = alpha * E / 2 * c64[s] / (k * (b - a)) / (b - a)
    size = share * (up + (share * up).sum(1, keepdims=True)) * rest
    want = share * (up - (share * up).sum(1, keepdims=True)) * rest
    assert np.allclose(want[:35], dz[:35], rtol=1e-6, atol=1e-15)   # (the oracle's own difference keeps fewer digits)
    assert (np.abs(np64(dlogits) - want) <= 320 * U * size).all()
    assert np.abs(P64 - np64(P)).max() <= 1024 * U * P64.max()
