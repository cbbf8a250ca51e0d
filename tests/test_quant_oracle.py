"""The block-scaled operators' oracle against what is known by other means: torch's e4m3 conversion, hand-worked exponents, differences."""
import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo


def test_codes_are_those_of_torch():
    all_codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(all_codes.copy()).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(qo.decode(all_codes), ref, equal_nan=True)
    mid = 0.5 * (qo.VALUES[1:] + qo.VALUES[:-1])
    x = np.concatenate([qo.VALUES, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9)])
    x = np.concatenate([x, -x]).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(qo.encode(x.astype(np.float64)), ref)


@pytest.mark.parametrize("a,e", [(0.0, 0), (448.0, 0), (449.0, 1), (224.0, -1), (225.0, 0), (1.75, -8), (1.76, -7), (2.0 ** -126, -126),
                                 (2.0 ** -149, -126), (3.3895e38, 120)])
def test_exponents(a, e):
    assert qo.exponent(a) == e
    assert a == 0 or (a <= 448 * 2.0 ** e and (e == -126 or a > 448 * 2.0 ** (e - 1)))


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal(4096) * 10.0 ** np.arange(-8, 8).repeat(256)
    x[:256] = np.ldexp(257.0 + 2 * np.arange(256), -9)   # ties
    assert np.array_equal(qo.bf16(x), torch.from_numpy(x).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("gated", [True, False])
def test_gradients_are_those_of_differences(gated):
    rng = np.random.default_rng(1)
    off, d, F, n = [0, 3, 3, 7], 6, 5, 7
    x, dy, w = rng.standard_normal((n, d)), rng.standard_normal((n, d)), rng.random(n)
    Wg, Wu, Wd = ([rng.standard_normal(s) * 0.5 for _ in range(3)] for s in ((d, F), (d, F), (F, d)))
    Wu = Wu if gated else None
    G, U, _, _ = qo.experts_fwd(x, off, Wg, Wu, Wd, quant_h=False)
    dX, dG, dU = qo.experts_bwd(dy, w, G, U, off, Wg, Wu, Wd, quant_g=False)
    loss = lambda v: float((qo.experts_fwd(v, off, Wg, Wu, Wd, quant_h=False)[3] * dy * w[:, None]).sum())
    h = 1e-5
    for i in range(n):
        for j in range(d):
            a, b = x.copy(), x.copy()
            a[i, j] += h
            b[i, j] -= h
            assert math.isclose((loss(a) - loss(b)) / (2 * h), dX[i, j], rel_tol=1e-6, abs_tol=1e-8)
