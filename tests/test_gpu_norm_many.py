"""Norms of the largest row counts that are accepted: the rows at both ends against the 64-bit definitions, under the bounds of test_gpu_norm.py, and what lies in front of and
behind the tensors."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64
from tests.test_gpu_norm import EPS, U, close

pytestmark = pytest.mark.gpu

END = 1 << 16   # rows looked at, at either end: two steps of the launch's teams
GUARD = 1 << 16


def guarded(n, d):
    """[n, d] of zeros in bf16 between rows of NaN."""
    whole = torch.full((GUARD + n + GUARD, d), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    whole[GUARD:GUARD + n] = 0
    return whole, whole[GUARD:GUARD + n]


@pytest.mark.parametrize("d", [2, 3])
def test_two_to_the_31_rows(d):
    import paper_2502_02581_amd as moe

    n = 2 ** 31 - 2 ** 15 - 1
    g = torch.Generator().manual_seed(d)
    ends = lambda: [(torch.randn(END, d, generator=g) + 0.5).bfloat16().cuda() for _ in range(2)]  # noqa: E731
    (Xw, X), (Yw, Y), (dYw, dY) = (guarded(n, d) for _ in range(3))
    x, dy = ends(), ends()
    X[:END], X[-END:], dY[:END], dY[-END:] = x[0], x[1], dy[0], dy[1]
    w = torch.randn(d, generator=g).cuda()
    norm = moe.MoENorm(n, d, "rms", EPS, "bf16", "f32")
    rstd = torch.full((n,), float("nan"), device="cuda:0")
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(moe.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device="cuda:0")

    def around(whole):
        return bool(torch.isnan(whole[:GUARD]).all() and torch.isnan(whole[-GUARD:]).all())

    moe.moe_norm_fwd(norm, X, w, None, Y, None, rstd)
    want = [ob.norm_fwd(np64(t), np64(w), None, "rms", EPS) for t in x]
    for got, r, (y, _, r64, h) in zip((Y[:END], Y[-END:]), (rstd[:END], rstd[-END:]), want):
        close(got, y, U * (64 * (1 + np.abs(h)) * np.abs(np64(w)) + 2 * np.abs(y)), "bf16")
        close(r, r64, U * 40 * r64, "f32")
    assert around(Yw) and torch.isfinite(rstd).all() and not Y[END:1 << 24].any()
    moe.moe_norm_bwd(norm, dY, X, w, None, rstd, Y, dw, db, ws)
    sums, tol = np.zeros((2, d)), np.zeros((2, d))
    for got, t, (_, _, r64, h) in zip((Y[:END], Y[-END:]), dy, want):
        t = np64(t)
        dz, dw64, db64 = ob.norm_bwd(t, h, r64, np64(w), "rms")
        gg = np.abs(t * np64(w))
        close(got, dz, 256 * U * r64[:, None] * (gg + gg.mean(1)[:, None] + (1 + np.abs(h)) * (gg * (1 + np.abs(h))).mean(1)[:, None]) + 2 * U * np.abs(dz), "bf16")
        sums += dw64, db64
        tol += (np.abs(t) * (1 + np.abs(h))).sum(0), np.abs(t).sum(0)
    assert around(Yw)
    # (of the rows that hold anything, 2 END of them, each of 16384 teams has eight, which it adds in sequence)
    close(dw, sums[0], 256 * U * tol[0], "f32")
    close(db, sums[1], 256 * U * tol[1], "f32")
