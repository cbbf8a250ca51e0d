"""moe_norm_fwd and moe_norm_bwd against the 64-bit definitions, element by element.

Tolerances, u = 2^-24: a lane adds at most 32 values in sequence, then 10 sums of sums, so a sum of n terms is off by at most 42 u of the sum of their magnitudes (48 below).
With the mean's own error taken out, z - mean is off by u |z| / d-free terms: one rounding of the difference and 48 u of the mean |z - mean|, which is at most its deviation, 1 / rstd.
So h is off by (|h| (1 + 48 / 2 + 4) + 48) u < 64 u (1 + |h|), y by that times |w|, and two roundings.  dz = rstd (g - mean g - h mean(g h)) moves by rstd u (4 |g| + 52 mean|g| +
(52 + 64) mean|g h| |h| + 64 (1 + |h|) |mean(g h)| + ..): bounded by 256 rstd u (|g| + mean|g| + (1 + |h|) mean|g (1 + |h|)|).  A weight gradient's sum has at most 64 rows in sequence and 80
sums of sums, and each term the error of h: 256 u sum |dy| (1 + |h|).  A result in bf16 is rounded once more, by at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def rows(gen, n, d, dtype, offset=0.0, pitch=None):
    """Activations; with pitch, rows that are pieces of longer ones, at an odd place."""
    x = torch.randn(n, d, generator=gen) * torch.exp(0.5 * torch.randn(n, 1, generator=gen)) + 0.3 * torch.randn(d, generator=gen) + offset
    x = x.to(DT[dtype])
    if pitch is None:
        return x.to("cuda:0")
    wide = torch.full((n, d + pitch), float("nan"), dtype=DT[dtype], device="cuda:0")
    wide[:, 1:1 + d] = x.to("cuda:0")
    return wide[:, 1:1 + d]


def blank(n, d, dtype, pitch=None):
    """An output full of NaN, and what its surroundings must still be afterwards."""
    wide = torch.full((n, d + (pitch or 0)), float("nan"), dtype=DT[dtype], device="cuda:0")
    return wide, (wide[:, 1:1 + d] if pitch else wide)


def untouched(wide, view):
    n = wide.shape[1] - view.shape[1]
    return n == 0 or bool(torch.isnan(torch.cat([wide[:, :1], wide[:, 1 + view.shape[1]:]], 1)).all())


def close(got, want, tol, dtype):
    got, tol = np64(got), np.broadcast_to(tol, want.shape) + HALF[dtype] * np.abs(want) * (1 + 2.0 ** -7)
    assert got.shape == want.shape and np.isfinite(got).all()
    off = np.abs(got - want) / (tol + 1e-300)
    assert off.max() <= 1, (off.max(), np.unravel_index(off.argmax(), off.shape))


def run(n, d, dtype, wdtype, kind, mode, p=0.25, pitch=None, weights=True, bias=True, offset=0.0, seed=0, dz_in=True, grads=True):
    import paper_2502_02581_amd as moe

    g = torch.Generator().manual_seed(1000 * n + d + seed)
    X = rows(g, n, d, dtype, offset, pitch)
    R = rows(g, n, d, dtype, offset, pitch) if mode in ("add", "drop") else None
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(DT[wdtype]).to("cuda:0") if weights else None
    b = (0.1 * torch.randn(d, generator=g)).to(DT[wdtype]).to("cuda:0") if bias else None
    dY, dZ = rows(g, n, d, dtype, 0.0, pitch), rows(g, n, d, dtype, 0.0, pitch) if dz_in else None
    rng = torch.tensor([(5 << 40) + seed, (1 << 35) + 7], dtype=torch.int64, device="cuda:0")
    drop = moe.MoEDropout(p, rng, 3) if mode in ("drop", "drop_only") else None
    norm = moe.MoENorm(n, d, kind, EPS, dtype, wdtype)
    has_z = mode != "plain"
    (Zw, Z), (Yw, Y), (dRw, dR), (dXw, dX) = (blank(n, d, dtype, pitch) for _ in range(4))
    f32 = dict(dtype=torch.float32, device="cuda:0")
    mean, rstd = (torch.full((n,), float("nan"), **f32) for _ in range(2))
    dw, db = (torch.full((d,), float("nan"), dtype=DT[wdtype], device="cuda:0") for _ in range(2))
    ws = torch.full((moe.moe_norm_bwd_workspace_bytes(norm),), 255, dtype=torch.uint8, device="cuda:0")
    layer = kind == "layer"
    moe.moe_norm_fwd(norm, X, w, b, Y, mean if layer else None, rstd, R=R, drop=drop, Z=Z if has_z else None)
    moe.moe_norm_bwd(norm, dY, Z if has_z else X, w, mean if layer else None, rstd, dR, dw if grads else None, db if grads else None, ws if grads else None,
                     dZ=dZ, drop=drop, dX=dX if drop else None)
    torch.cuda.synchronize()
    assert untouched(Zw, Z) and untouched(Yw, Y) and untouched(dRw, dR) and untouched(dXw, dX)
    # ---- forward
    x, r = np64(X), np64(R) if R is not None else None
    mask = ob.keep(n, d, p, (5 << 40) + seed, (1 << 35) + 7, 3) if drop else np.ones((n, d), bool)
    scale = ob.scale(p) if drop else 1.0
    if has_z:
        want = np.where(mask, x * scale, 0.0) + (r if r is not None else 0.0)
        close(Z, want, U * np.abs(x * scale) * 1.01, dtype)
        dropped = np64(Z)[~mask]
        assert np.array_equal(dropped, np64(R)[~mask] if r is not None else np.zeros_like(dropped))
        x = np64(Z)   # the norm is of the values that are kept
    W, B = np64(w) if w is not None else None, np64(b) if b is not None else None
    y, m64, r64, h = ob.norm_fwd(x, W, B, kind, EPS)
    absw = np.abs(W) if W is not None else 1.0
    close(Y, y, U * (64 * (1 + np.abs(h)) * absw + 2 * np.abs(y)), dtype)
    close(rstd, r64, U * 40 * r64, "f32")
    if layer:
        close(mean, m64, U * (np.abs(m64) + 48 / r64), "f32")
    # ---- backward
    dy = np64(dY)
    dz, dw64, db64 = ob.norm_bwd(dy, h, r64, W, kind)
    g = np.abs(dy * absw)
    tol = 256 * U * r64[:, None] * (g + g.mean(1)[:, None] + (1 + np.abs(h)) * (g * (1 + np.abs(h))).mean(1)[:, None])
    total = dz + (np64(dZ) if dZ is not None else 0.0)
    tol = tol + 2 * U * np.abs(total)
    close(dR, total, tol, dtype)
    if drop:
        close(dX, np.where(mask, total * scale, 0.0), tol * scale + 2 * U * np.abs(total) * scale, dtype)
        assert not np64(dX)[~mask].any()
    if grads:
        close(dw, dw64, 256 * U * (np.abs(dy) * (1 + np.abs(h))).sum(0), wdtype)
        close(db, db64, 256 * U * np.abs(dy).sum(0), wdtype)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 2), (5, 7), (9, 8), (4, 9), (33, 64), (70, 333), (17, 512), (6, 513), (258, 1000), (40, 1025), (19, 2048), (7, 4100), (5, 7168), (3, 8200), (2, 16384)])
def test_sizes(n, d, dtype, wdtype, kind):
    run(n, d, dtype, wdtype, kind, "plain")


@pytest.mark.parametrize("mode", ["add", "drop", "drop_only"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 5), (37, 129), (300, 1000), (21, 2050), (4, 7168), (2, 16383)])
def test_residual(n, d, dtype, kind, mode):
    run(n, d, dtype, dtype, kind, mode)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch", [2, 9])
@pytest.mark.parametrize("n,d", [(5, 64), (12, 1001), (6, 3000)])
def test_strided_rows(n, d, pitch, dtype):
    """Rows that are pieces of longer ones and start on no boundary; what lies between them stays as it was."""
    run(n, d, dtype, dtype, "layer", "drop", pitch=pitch)


@pytest.mark.parametrize("n,d,dtype", [(512, 520, "bf16"), (513, 520, "bf16"), (1024, 72, "f32"), (1025, 72, "f32"), (1023, 4096, "bf16"), (1025, 4096, "bf16"), (3000, 1000, "bf16"), (5000, 64, "f32"), (2500, 2048, "bf16"), (1030, 7168, "f32"), (16384, 16, "bf16")])
def test_many_rows(n, d, dtype):
    """More rows than teams: every block adds several."""
    run(n, d, dtype, dtype, "layer", "plain")


@pytest.mark.parametrize("weights,bias,dz_in,grads", [(False, False, True, True), (True, False, False, True), (False, True, False, False)])
def test_absent_tensors(weights, bias, dz_in, grads):
    for d in (100, 3000):
        run(9, d, "bf16", "f32", "layer", "plain", weights=weights, bias=bias, dz_in=dz_in, grads=grads)


@pytest.mark.parametrize("d", [200, 4096])
def test_rows_far_from_zero(d):
    """Mean 1e4, deviation 1: the mean's rounding error would be 5e-4 of the deviation."""
    run(7, d, "f32", "f32", "layer", "plain", offset=1e4)


@pytest.mark.parametrize("offset", [2.0, 6.0, 12.0, 300.0])
@pytest.mark.parametrize("n,d", [(30, 500), (2500, 96)])
def test_means_around_the_lines(n, d, offset):
    """Means of a few deviations, on both sides of the lines from which on their rounding error is taken out, for both ways to the weights' gradients."""
    run(n, d, "f32", "f32", "layer", "plain", offset=offset)


@pytest.mark.parametrize("d", [48, 5000, 20, 200])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_that_are_not_finite_stay_alone(kind, d):
    """NaN and infinities reach their own row and no other; a constant row has the deviation sqrt(eps)."""
    import paper_2502_02581_amd as moe

    norm = moe.MoENorm(6, d, kind, EPS, "f32")
    X = torch.randn(6, d, device="cuda:0")
    clean = X.clone()
    X[1, d // 2], X[3, 0], X[4] = float("nan"), float("inf"), 2.5
    Y, Yc, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(6, device="cuda:0")
    moe.moe_norm_fwd(norm, X, None, None, Y, None, rstd)
    moe.moe_norm_fwd(norm, clean, None, None, Yc)
    assert torch.equal(Y[[0, 2, 5]], Yc[[0, 2, 5]])
    assert torch.isnan(Y[1]).all() and torch.isnan(Y[3]).any()
    if kind == "layer":
        assert torch.isnan(Y[3]).all() and not Y[4].any() and abs(float(rstd[4]) * EPS ** 0.5 - 1) < 1e-6


@pytest.mark.parametrize("mode", ["plain", "drop"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 6), (300, 7), (70, 15), (37, 127), (41, 128), (45, 130), (21, 255), (23, 256), (33, 257), (2100, 27), (2000, 203), (1500, 505), (1100, 1021), (1100, 1029),
                                 (1100, 2500), (1100, 3001), (1030, 8191), (20, 8199)])
def test_short_pieces(n, d, dtype, mode):
    """Rows that end inside a piece, for every size of team, with few rows and many."""
    run(n, d, dtype, "f32", "layer", mode)


@pytest.mark.parametrize("n,d", [(50, 96), (50, 7000), (700, 520), (9, 9000), (50, 97), (700, 15), (60, 1030), (1100, 3005)])
def test_outputs_that_are_inputs(n, d):
    """The residual stream updated in place, the gradient written over the one that came in, or over the saved rows: what it is into tensors of their own, the same bits (the
    weights' gradients, which then take another order: within fp32's rounding of their sums, and bf16's)."""
    import paper_2502_02581_amd as moe

    g = torch.Generator().manual_seed(d)
    X, R, dY, dZ = (rows(g, n, d, "bf16") for _ in range(4))
    w, b = torch.randn(d, generator=g).bfloat16().cuda(), torch.randn(d, generator=g).bfloat16().cuda()
    rng = torch.tensor([1, 2], device="cuda:0")
    norm, drop = moe.MoENorm(n, d), moe.MoEDropout(0.3, rng)
    mean, rstd = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(moe.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device="cuda:0")
    Z, Y, dR, dX = (torch.empty_like(X) for _ in range(4))
    dw, db = torch.empty_like(w), torch.empty_like(b)
    moe.moe_norm_fwd(norm, X, w, b, Y, mean, rstd, R=R, drop=drop, Z=Z)
    moe.moe_norm_bwd(norm, dY, Z, w, mean, rstd, dR, dw, db, ws, dZ=dZ, drop=drop, dX=dX)
    x, r = X.clone(), R.clone()
    moe.moe_norm_fwd(norm, x, w, b, x, mean, rstd, R=r, drop=drop, Z=r)
    assert torch.equal(x, Y) and torch.equal(r, Z)
    dy, dz = dY.clone(), dZ.clone()
    dw2, db2 = torch.empty_like(w), torch.empty_like(b)
    moe.moe_norm_bwd(norm, dy, Z, w, mean, rstd, dz, dw2, db2, ws, dZ=dz, drop=drop, dX=dy)
    assert torch.equal(dz, dR) and torch.equal(dy, dX)
    h = (Z.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for a, b2, terms in ((dw, dw2, dY.double() * h), (db, db2, dY.double())):
        assert ((a.double() - b2.double()).abs() <= 2 * (2.0 ** -8 * terms.sum(0).abs() + 256 * U * terms.abs().sum(0) * 3)).all()
    zz = Z.clone()
    moe.moe_norm_bwd(norm, dY, zz, w, mean, rstd, zz, dw2, db2, ws, dZ=dZ, drop=drop, dX=dX)
    assert torch.equal(zz, dR)


def test_beyond_two_to_the_31_values():
    """Rows whose values lie behind 2^31 others, forward and backward: the last rows against the definition."""
    import paper_2502_02581_amd as moe

    d = 16384
    n = (1 << 31) // d + 40
    g = torch.Generator().manual_seed(9)
    few = [rows(g, 8, d, "bf16") for _ in range(2)]
    X, dY, Y = (torch.zeros(n, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(3))
    X[-8:], dY[-8:] = few
    w = torch.randn(d, generator=g).cuda()
    norm = moe.MoENorm(n, d, "layer", EPS, "bf16", "f32")
    mean, rstd, dw, db = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0"), torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(moe.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device="cuda:0")
    moe.moe_norm_fwd(norm, X, w, None, Y, mean, rstd)
    x, dy = np64(few[0]), np64(few[1])
    y, m64, r64, h = ob.norm_fwd(x, np64(w), None, "layer", EPS)
    close(Y[-8:], y, U * (64 * (1 + np.abs(h)) * np.abs(np64(w)) + 2 * np.abs(y)), "bf16")
    assert not Y[:-8].any()
    moe.moe_norm_bwd(norm, dY, X, w, mean, rstd, Y, dw, db, ws)
    dz, dw64, db64 = ob.norm_bwd(dy, h, r64, np64(w), "layer")
    gg = np.abs(dy * np64(w))
    tol = 256 * U * r64[:, None] * (gg + gg.mean(1)[:, None] + (1 + np.abs(h)) * (gg * (1 + np.abs(h))).mean(1)[:, None]) + 2 * U * np.abs(dz)
    close(Y[-8:], dz, tol, "bf16")
    assert not Y[:-8].any()
    close(dw, dw64, 256 * U * (np.abs(dy) * (1 + np.abs(h))).sum(0), "f32")
    close(db, db64, 256 * U * np.abs(dy).sum(0), "f32")


def test_no_rows():
    import paper_2502_02581_amd as moe

    norm = moe.MoENorm(0, 40)
    e = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda:0")
    w = torch.ones(40, dtype=torch.bfloat16, device="cuda:0")
    dw, db = torch.full_like(w, 7), torch.full_like(w, 7)
    f = torch.empty(0, device="cuda:0")
    ws = torch.empty(moe.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device="cuda:0")
    moe.moe_norm_fwd(norm, e, w, None, e, f, f)
    moe.moe_norm_bwd(norm, e, e, w, f, f, e, dw, db, ws)
    assert not dw.any() and not db.any()


def test_gradient_by_differences():
    """The forward pass's own differences along one direction, in fp32 on values where they are exact enough: a step of 2^-6 of the input moves the sum of Y dY by the
    gradient's product with it up to the third derivative's (1/6 step^2 times values of a few) and the sums' rounding (1e-6 / step)."""
    import paper_2502_02581_amd as moe

    n, d = 5, 300
    g = torch.Generator().manual_seed(4)
    norm = moe.MoENorm(n, d, "layer", EPS, "f32")
    X, dY, along = (torch.randn(n, d, generator=g).cuda() for _ in range(3))
    w, b = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    Y, dR, mean, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    step, total = 2.0 ** -6, []
    for sign in (1, -1):
        moe.moe_norm_fwd(norm, X + sign * step * along, w, b, Y)
        total.append((Y.double() * dY.double()).sum(1))
    moe.moe_norm_fwd(norm, X, w, b, Y, mean, rstd)
    moe.moe_norm_bwd(norm, dY, X, w, mean, rstd, dR, None, None, None)
    slope = (total[0] - total[1]) / (2 * step)
    want = (dR.double() * along.double()).sum(1)
    assert ((slope - want).abs() <= 1e-2 * (dY.norm(dim=1) * along.norm(dim=1)).double() * step).all()
