"""Layer norm of constant rows and of rows a few of their type's steps wide, whose squares around a rounded mean are that mean's error.

Tolerances, u = 2^-24.  Constant rows: the mean is exact, the deviation sqrt(eps) up to the roundings of a sum, a root and a division, and every value is its bias.  Others: the
squares around the mean taken are at most twice those around the true one, each sum is off by 48 u of itself and what is taken away by as much: (2 * 50 + 2 * 48) u of the
variance, 100 u of rstd (128 below).  z - mean is off by 48 u of the deviation around the mean taken, at most sqrt(2) of the true one: with rstd's 100 u, 128 u (1 + |h|) of y.  In the backward
pass a saved mean is off by a step, which is below a deviation here, so |z - mean| is at most (1 + |h|) deviations: twice the bound of ordinary rows with 2 + |h| for 1 + |h|."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64
from tests.test_gpu_norm import DT, EPS, U, close

pytestmark = pytest.mark.gpu

WIDTHS = [(9, 3), (300, 100), (40, 127), (37, 250), (20, 333), (25, 878), (700, 1000), (9, 1100), (1100, 2200), (5, 5001), (1030, 5000), (3, 7168), (3, 9001)]   # every team, short pieces among them


@pytest.mark.parametrize("n,d", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_constant_rows(n, d, dtype):
    import paper_2502_02581_amd as moe

    values = torch.tensor([0.0, 2.5, -97.3, 1.1e4, 3.3e8, 1e9, -7.7e9, 1.3e10, 6.1e11, -1e12, 9.9e14]).to(DT[dtype])
    g = torch.Generator().manual_seed(d)
    X = values[torch.arange(n) % len(values)][:, None].expand(n, d).contiguous().cuda()
    dY = torch.randn(n, d, generator=g).to(DT[dtype]).cuda()
    w, b = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    norm = moe.MoENorm(n, d, "layer", EPS, dtype, "f32")
    Y, dR, dw, db = torch.empty_like(X), torch.empty_like(X), torch.empty_like(w), torch.empty_like(w)
    mean, rstd = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(moe.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device="cuda:0")
    moe.moe_norm_fwd(norm, X, w, b, Y, mean, rstd)
    assert torch.equal(mean, X[:, 0].float())
    assert (np.abs(np64(rstd) * EPS ** 0.5 - 1) <= 4 * U).all()
    assert torch.equal(Y, b.to(DT[dtype]).expand(n, d))
    moe.moe_norm_bwd(norm, dY, X, w, mean, rstd, dR, dw, db, ws)
    dy, h = np64(dY), np.zeros((n, d))
    dz, dw64, db64 = ob.norm_bwd(dy, h, np64(rstd), np64(w), "layer")
    size = np.abs(dy * np64(w))
    close(dR, dz, 256 * U * np64(rstd)[:, None] * (size + size.mean(1)[:, None]), dtype)
    assert not dw.any()
    close(db, db64, 256 * U * np.abs(dy).sum(0), "f32")


@pytest.mark.parametrize("n,d", WIDTHS)
@pytest.mark.parametrize("base", [1.5e4, 1e9, -3e11])
def test_rows_of_a_few_steps(n, d, base):
    """Values of `base` and up to three steps of fp32 beside it, two in three of them others than it."""
    import paper_2502_02581_amd as moe

    g = torch.Generator().manual_seed(d + 1)
    one = torch.tensor(base)
    step = (torch.nextafter(one, one * 2) - one).abs()
    X = (one + step * torch.randint(-3, 4, (n, d), generator=g)).cuda()
    X[:, 0], X[:, -1] = base, base + 3 * float(step)
    w, b = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    dY = torch.randn(n, d, generator=g).cuda()
    norm = moe.MoENorm(n, d, "layer", EPS, "f32")
    Y, dR, mean, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    moe.moe_norm_fwd(norm, X, w, b, Y, mean, rstd)
    y, m64, r64, h = ob.norm_fwd(np64(X), np64(w), np64(b), "layer", EPS)
    close(rstd, r64, 128 * U * r64, "f32")
    close(mean, m64, U * np.abs(m64) + 128 * U / r64, "f32")
    close(Y, y, U * (128 * (1 + np.abs(h)) * np.abs(np64(w)) + 2 * np.abs(y)), "f32")
    moe.moe_norm_bwd(norm, dY, X, w, mean, rstd, dR, None, None, None)
    dy = np64(dY)
    dz = ob.norm_bwd(dy, h, r64, np64(w), "layer")[0]
    size = np.abs(dy * np64(w))
    tol = 512 * U * r64[:, None] * (size + size.mean(1)[:, None] + (2 + np.abs(h)) * (size * (2 + np.abs(h))).mean(1)[:, None])
    close(dR, dz, tol + 2 * U * np.abs(dz), "f32")
