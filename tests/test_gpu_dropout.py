"""moe_dropout against the generator's definition: the mask value for value, what is kept within one rounding."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def make(n, d, dtype, seed=0, pitch=0):
    g = torch.Generator().manual_seed(seed * 7919 + n * 13 + d)
    x = torch.randn(n, d, generator=g).to(dtype)
    x[x == 0] = 1
    wide = torch.full((n, d + pitch), float("nan"), dtype=dtype, device="cuda:0")
    view = wide[:, 1:1 + d] if pitch else wide
    view.copy_(x)
    return view


def check(out, X, R, mask, p):
    x, r = np64(X), np64(R) if R is not None else 0.0
    kept = x * ob.scale(p)
    want = np.where(mask, kept, 0.0) + r
    got = np64(out)
    # the scale is rounded once, the sum once
    assert (np.abs(got - want) <= 1.01 * (U * np.abs(kept) + HALF[out.dtype] * (np.abs(want) + U * np.abs(kept)))).all()
    assert np.array_equal(got[~mask], np.broadcast_to(r, x.shape)[~mask])
    if R is None:
        assert np.array_equal(got != 0, mask)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_r", [False, True])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 3), (700, 1), (5, 8), (64, 9), (129, 100), (31, 333), (300, 512), (2, 4097), (37, 7168), (1, 70001)])
def test_sizes(n, d, with_r, dtype):
    import paper_2502_02581_amd as moe

    seed, step, site, p = 0x1234567890ABCDE, (3 << 33) + 1, 65535, 0.1
    X, R = make(n, d, dtype), make(n, d, dtype, 1) if with_r else None
    drop = moe.MoEDropout(p, torch.tensor([seed, step], device="cuda:0"), site)
    out = torch.full((n, d), float("nan"), dtype=dtype, device="cuda:0")
    moe.moe_dropout(X, drop, out, R=R)
    check(out, X, R, ob.keep(n, d, p, seed, step, site), p)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 1e-5, 0.5, 0.9, 0.99998])
def test_probabilities(p):
    import paper_2502_02581_amd as moe

    X = make(50, 1000, torch.float32)
    out = torch.empty_like(X)
    moe.moe_dropout(X, moe.MoEDropout(p, torch.tensor([9, 8], device="cuda:0"), 1), out)
    check(out, X, None, ob.keep(50, 1000, p, 9, 8, 1), p)
    if p < 2.0 ** -17:
        moe.moe_dropout(X, moe.MoEDropout(p, None), out, R=X)   # nothing to draw
        assert torch.equal(out, X + X)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_rows_and_places(dtype):
    """Rows that are pieces of longer ones, into other such rows and in place: the mask goes by row and column alone."""
    import paper_2502_02581_amd as moe

    n, d, p = 40, 203, 0.3
    rng = torch.tensor([77, 5], device="cuda:0")
    drop = moe.MoEDropout(p, rng, 2)
    X, R, out = make(n, d, dtype, 0, 6), make(n, d, dtype, 1, 3), make(n, d, dtype, 2, 5)
    base = out._base if out._base is not None else out
    base.fill_(float("nan"))
    moe.moe_dropout(X, drop, out, R=R)
    check(out, X, R, ob.keep(n, d, p, 77, 5, 2), p)
    assert torch.isnan(base[:, :1]).all() and torch.isnan(base[:, 1 + d:]).all()
    a, b = X.clone(), R.clone()
    moe.moe_dropout(a, drop, a, R=R)
    moe.moe_dropout(X, drop, b, R=b)
    assert torch.equal(a, out) and torch.equal(b, out)


def test_what_is_dropped_adds_nothing():
    import paper_2502_02581_amd as moe

    X = torch.full((64, 72), float("inf"), device="cuda:0")
    X[::2] = float("nan")
    R = torch.ones_like(X)
    out = torch.empty_like(X)
    moe.moe_dropout(X, moe.MoEDropout(0.5, torch.tensor([3, 4], device="cuda:0")), out, R=R)
    mask = torch.from_numpy(ob.keep(64, 72, 0.5, 3, 4, 0)).cuda()
    assert (out[~mask] == 1).all() and not torch.isfinite(out[mask]).any()


def test_adjoint():
    """<drop(x), y> = <x, drop(y)>, and the mask of the norm's dropout is the same one."""
    import paper_2502_02581_amd as moe

    n, d = 30, 1001
    X, Y = make(n, d, torch.float32), make(n, d, torch.float32, 5)
    drop = moe.MoEDropout(0.2, torch.tensor([1 << 62, -1], device="cuda:0"), 9)
    a, b, z, y = (torch.empty_like(X) for _ in range(4))
    moe.moe_dropout(X, drop, a)
    moe.moe_dropout(Y, drop, b)
    left, right = (a.double() * Y.double()).sum(), (X.double() * b.double()).sum()
    assert abs(left - right) <= 2 * U * (a.double() * Y.double()).abs().sum()
    moe.moe_norm_fwd(moe.MoENorm(n, d, dtype="f32"), X, None, None, y, drop=drop, Z=z)
    assert torch.equal(z, a)


@pytest.mark.parametrize("dtype", [torch.bfloat16])
def test_beyond_two_to_the_31_values(dtype):
    """Row and column far behind: 2^31 + values; the last rows against the definition."""
    import paper_2502_02581_amd as moe

    d, n = 8200, (1 << 31) // 8200 + 300
    X = torch.ones(n, d, dtype=dtype, device="cuda:0")
    moe.moe_dropout(X, moe.MoEDropout(0.1, torch.tensor([21, 22], device="cuda:0"), 6), X)
    for r0 in (0, (1 << 31) // 8200 - 2, n - 4):
        got = X[r0:r0 + 4].float().cpu().numpy() != 0
        assert np.array_equal(got, ob.keep(4, d, 0.1, 21, 22, 6, r0))
