"""The block-scaled 8-bit operators against their 64-bit definitions.

Bounds.  Codes and exponents are exact.  An element of a product is off by at most
  2^-8 |c|             its rounding to bf16 (half a step)
  2^-10 sum |a b|      the matrix instruction aligns eight neighbouring products to the largest one and drops what lies 13 bits below its leading
                       bit: less than 8 * 2^-13 of the largest, so of the sum of the eight
  (K / 8) 2^-24 sum |a b|   fp32 additions, one for eight products
"""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo

from .helpers import small_tiles

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def moe():
    import paper_2502_02581_amd as m

    return m


def u8(*shape, fill=0xA5):
    return torch.full(shape, fill, dtype=torch.uint8, device=DEV)


def np_of(t):
    return t.detach().cpu().double().numpy()


def same_codes(got, ref):
    """Equal bytes; NaN codes may differ in sign, and zeros of blocks that a sign bit survives in do not."""
    g, r = got.cpu().numpy(), np.asarray(ref)
    nan = (r & 127) == 127
    return np.array_equal((g & 127) == 127, nan) and np.array_equal(g[~nan], r[~nan])


def product_bound(a, b, c):
    """Per element, for c = a b in 64 bits."""
    K = a.shape[1]
    return 2.0 ** -8 * np.abs(c) + (2.0 ** -10 + max(K / 8, 1) * 2.0 ** -24) * (np.abs(a) @ np.abs(b)) + 1e-37


# ------------------------------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,cols,ld,shift", [(1, 1, 1, 0), (1, 128, 128, 0), (3, 127, 127, 0), (5, 129, 136, 0), (17, 1000, 1000, 0), (64, 2048, 2048, 0),
                                             (7, 264, 300, 4), (33, 136, 136, 1), (2, 7168, 7168, 0), (1025, 40, 40, 0)])
def test_rows(dtype, n, cols, ld, shift):
    m = moe()
    g = torch.Generator().manual_seed(n * 1000 + cols)
    base = torch.full((shift + n * ld,), float("nan"))
    X = base[shift:].view(n, ld)[:, :cols]   # neighbours of a strided matrix are NaN: not part of it
    X.copy_(torch.randn(n, cols, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g)))
    X = base.to(dtype).to(DEV)[shift:].view(n, ld)[:, :cols]
    Q, S = u8(n, m.moe_quant_row_bytes(cols)), u8(n, m.moe_quant_scale_bytes(cols))
    m.moe_quant_rows(X, Q, S)
    q, s = qo.quant_rows(np_of(X))
    assert np.array_equal(S.cpu().numpy(), s)
    assert same_codes(Q, q)


def test_rows_special_values():
    """Blocks of zeros, of one value, at the borders of the exponent, tiny and huge ones, with infinities and NaN."""
    m = moe()
    rows = [torch.zeros(256), torch.full((256,), 448.0), torch.full((256,), 449.0), torch.full((256,), -1.75), torch.full((256,), 1.7578125),
            torch.full((256,), 2.0 ** -126), torch.full((256,), 2.0 ** -149), torch.full((256,), 3.38e38),
            torch.linspace(-448, 448, 256), torch.linspace(0, 0.02, 256), torch.arange(256) * 2.0 ** -9]
    inf, nan, both = torch.linspace(-3, 3, 256), torch.linspace(-3, 3, 256), torch.full((256,), float("inf"))
    inf[5], inf[200], nan[130], both[128:] = float("inf"), -float("inf"), float("nan"), float("nan")
    X = torch.stack(rows + [inf, nan, both])
    n = X.shape[0]
    for dtype in (torch.float32, torch.bfloat16):
        x = X.to(dtype).to(DEV)
        Q, S = u8(n, 256), u8(n, 2)
        m.moe_quant_rows(x, Q, S)
        q, s = qo.quant_rows(np_of(x))
        assert np.array_equal(S.cpu().numpy(), s)
        assert same_codes(Q, q)
        assert int(S[0, 0]) == 127 and int(Q[0].max()) == 0


def test_rows_empty_and_other_stream():
    m = moe()
    m.moe_quant_rows(torch.empty(0, 64, device=DEV), u8(0, 128), u8(0, 1))
    X = torch.randn(50, 300, device=DEV)
    Q, S = u8(50, 384), u8(50, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m.moe_quant_rows(X, Q, S, stream=side)
    side.synchronize()
    q, s = qo.quant_rows(np_of(X))
    assert np.array_equal(S.cpu().numpy(), s) and same_codes(Q, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,K,N", [(1, 8, 8), (2, 128, 128), (3, 136, 264), (1, 1000, 72), (5, 256, 1408), (1, 64, 2048)])
def test_weights(dtype, E, K, N):
    m = moe()
    g = torch.Generator().manual_seed(K * 100 + N)
    W = (torch.randn(E, K, N, generator=g) * torch.exp(torch.randn(E, 1, 1, generator=g))).to(dtype).to(DEV)
    b, r = m.moe_quant_scale_bytes, m.moe_quant_row_bytes
    Q, S, Qt, St = u8(E, K, r(N)), u8(E, b(K), b(N)), u8(E, N, r(K)), u8(E, b(N), b(K))
    m.moe_quant_weights(W, Q, S, Qt, St)
    for e in range(E):
        w = np_of(W[e])
        q, s = qo.quant_matrix(w)
        assert np.array_equal(S[e].cpu().numpy(), s) and same_codes(Q[e], q)
        q, s = qo.quant_matrix(w.T)
        assert np.array_equal(St[e].cpu().numpy(), s) and same_codes(Qt[e], q)
    # one layout alone, rows as pieces of longer ones; the other pieces stay as they are
    wide, exps = u8(E, K, 2 * r(N)), u8(E, b(K), 2 * b(N))
    m.moe_quant_weights(W, wide[:, :, r(N):], exps[:, :, b(N):], None, None)
    assert torch.equal(wide[:, :, r(N):], Q) and torch.equal(exps[:, :, b(N):], S)
    assert int((wide[:, :, :r(N)] != 0xA5).sum()) == 0 and int((exps[:, :, :b(N)] != 0xA5).sum()) == 0
    only, e2 = u8(E, N, r(K)), u8(E, b(N), b(K))
    m.moe_quant_weights(W, None, None, only, e2)
    assert torch.equal(only, Qt) and torch.equal(e2, St)


# ------------------------------------------------------------------------------------------ products
def scaled_rows(g, n, K, std=1.0):
    x = torch.randn(n, K, generator=g, dtype=torch.float64).numpy() * std * np.exp(torch.randn(n, 1, generator=g, dtype=torch.float64).numpy())
    q, s = qo.quant_rows(x)
    return torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV), qo.values(q, s)[:, :K]


def scaled_matrices(g, E, K, N):
    """Codes of the transposed matrices, and their values [K, N]."""
    qs, ss, vs = [], [], []
    for _ in range(E):
        w = torch.randn(N, K, generator=g, dtype=torch.float64).numpy() / np.sqrt(K)
        w *= np.exp(torch.randn(-(-N // 128), generator=g, dtype=torch.float64).numpy()).repeat(128)[:N, None]   # exponents that differ
        q, s = qo.quant_matrix(w)
        qs.append(torch.from_numpy(q))
        ss.append(torch.from_numpy(s))
        vs.append(np.ascontiguousarray(qo.values(q, s, 128)[:, :K].T))
    return torch.stack(qs).to(DEV), torch.stack(ss).to(DEV), vs


GEMM_CASES = [
    ([1], 8, 8), ([1], 128, 16), ([16], 256, 64), ([17], 1000, 136), ([5, 0, 3], 136, 40), ([0, 0, 1], 128, 128), ([0, 0], 64, 64),
    ([64, 65, 63, 1, 0, 128], 384, 264), ([257, 3, 96], 512, 520), ([300, 200, 140, 33], 256, 256), ([513], 640, 384), ([700, 0, 130, 15, 16, 31], 200, 200),
    ([1] * 40, 256, 128), ([2, 0] * 30, 1408, 72), ([256, 512, 128], 128, 256), ([33], 4096, 48), ([1], 7168, 512), ([16], 7168, 256), ([100], 2304, 640),
    ([300], 7168, 256), ([5000], 128, 4096),            # one group: parts of tall tiles, a last round cut into low ones
    ([37 * i % 300 for i in range(60)], 128, 4096),     # four rounds of tiles: the order that mixes heights
]


@pytest.mark.parametrize("counts,K,N,dense", [(*c, False) for c in GEMM_CASES] + [(*c, True) for c in GEMM_CASES if len(c[0]) == 1])
def test_gemm(counts, K, N, dense):   # dense: without offsets, one group
    m = moe()
    g = torch.Generator().manual_seed(sum(counts) * 7 + K + N)
    E, before, behind = len(counts), (0 if dense else 2), (0 if dense else 5)   # rows of no group on both sides
    n = sum(counts) + before + behind
    off = np.concatenate([[before], before + np.cumsum(counts)]).astype(np.int32)
    A, As, a = scaled_rows(g, n, K)
    B, Bs, b = scaled_matrices(g, E, K, N)
    C = torch.full((n, N), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = u8(m.moe_quant_gemm_workspace_bytes(E, n, K, N))
    m.moe_quant_gemm(None if dense else torch.from_numpy(off).to(DEV), K, A, As, B, Bs, C, ws)
    got = np_of(C)
    for e in range(E):
        x, y = int(off[e]), int(off[e + 1])
        ref = a[x:y] @ b[e]
        assert (np.abs(got[x:y] - ref) <= product_bound(a[x:y], b[e], ref)).all(), e
    assert (got[:before] == 7).all() and (got[n - behind:] == 7).all()
    again = torch.full_like(C, 7.0)
    m.moe_quant_gemm(None if dense else torch.from_numpy(off).to(DEV), K, A, As, B, Bs, again, ws)
    assert torch.equal(C.view(torch.int16), again.view(torch.int16))


def test_gemm_exponents_at_the_ends():
    """Very large and very small blocks side by side; sums beyond the range become infinite, NaN codes reach their rows and columns alone."""
    m = moe()
    n, K, N = 40, 256, 128
    g = torch.Generator().manual_seed(3)
    x = torch.randn(n, K, generator=g, dtype=torch.float64).numpy()
    x[0] *= 2.0 ** 100
    x[1] *= 2.0 ** -100
    x[2, :128] *= 2.0 ** 60
    x[3] = 0
    q, s = qo.quant_rows(x)
    q[4, 7] = 127
    w = torch.randn(N, K, generator=g, dtype=torch.float64).numpy()
    qw, sw = qo.quant_matrix(w)
    qw[9, 200] = 255
    sw = sw + np.uint8(20)
    dev = lambda t: torch.from_numpy(t).to(DEV)
    C = torch.empty(n, N, dtype=torch.bfloat16, device=DEV)
    m.moe_quant_gemm(None, K, dev(q), dev(s), dev(qw)[None], dev(sw)[None], C, u8(m.moe_quant_gemm_workspace_bytes(1, n, K, N)))
    a, b = qo.values(q, s), qo.values(qw, sw, 128)
    got = np_of(C)
    nan = np.zeros((n, N), bool)
    nan[4], nan[:, 9] = True, True
    assert np.array_equal(np.isnan(got), nan)
    fine = np.nan_to_num(a), np.nan_to_num(b.T)
    ref = fine[0] @ fine[1]
    ok = ~nan
    assert (np.abs(got - ref)[ok] <= product_bound(*fine, ref)[ok]).all()
    s[0] += np.uint8(28)   # 2^128 and more
    m.moe_quant_gemm(None, K, dev(q), dev(s), dev(qw)[None], dev(sw)[None], C, u8(m.moe_quant_gemm_workspace_bytes(1, n, K, N)))
    big = np_of(C)[0]
    ref = (qo.values(q, s)[0] @ np.nan_to_num(b.T))
    sure = (np.abs(ref) > 2.0 ** 130) & ~nan[0]
    # (not of the sum's sign: a sum of terms beyond 2^128 stays at the infinity that its first partial sums reached, as in any fp32 arithmetic)
    assert sure.any() and np.isinf(big[sure]).all()


# ------------------------------------------------------------------------------------------- experts
# T, E, k, d, d_ff, gated, rows read in place
EXPERTS = [(1, 4, 1, 64, 64, True, True), (1, 8, 4, 128, 136, True, True), (16, 12, 4, 256, 192, True, True), (33, 3, 1, 136, 72, False, False),
           (300, 6, 3, 200, 264, True, True), (150, 2, 1, 1000, 328, False, True), (600, 5, 2, 256, 384, True, False), (1100, 3, 1, 384, 128, True, True),
           (64, 40, 2, 128, 256, True, True), (700, 2, 1, 128, 136, True, True), (520, 2, 1, 264, 648, False, False),
           (100, 12, 4, 264, 392, True, True), (200, 9, 2, 136, 200, False, True)]
# calls whose weight gradients take the tall tiles, in common launches with the input gradients, the weight gradients' tiles first (d up to 1024) or last
TALL = [(3500, 3, 1, 1000, 136, True, True), (3500, 3, 1, 1000, 136, False, False), (1700, 4, 1, 2056, 200, True, False), (1150, 5, 2, 2048, 128, False, True),
        (900, 70, 4, 1024, 64, True, True)]


def routed(T, E, k, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g) - 1.2 * torch.log(torch.arange(1, E + 1, dtype=torch.float32))
    idx = torch.topk(z, k, dim=1).indices.reshape(-1)
    counts = torch.bincount(idx, minlength=E)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32)
    return off, torch.sort(idx, stable=True).indices.to(torch.int32), torch.rand(T, k, generator=g) * 0.7 + 0.1, g


class Layer:
    """Inputs of one set of experts and what the quantised values stand for."""

    def __init__(self, T, E, k, d, F, gated, gather):
        m = moe()
        self.shape, self.E, self.n, self.gated, self.gather = m.MoEShape(T, d, E, k, F, "bf16"), E, T * k, gated, gather
        off, src, w, g = routed(T, E, k, T * 13 + d)
        self.off, self.src, self.src_np = off.to(DEV), src.to(DEV), src.numpy()
        self.bounds = off.numpy()
        bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).to(DEV)
        self.X, self.dY = bf(T, d), bf(T, d)
        self.W = [bf(E, d, F, std=d ** -0.5), bf(E, d, F, std=d ** -0.5) if gated else None, bf(E, F, d, std=F ** -0.5)]
        token = (self.src // k).long()
        self.Xp = self.X[token]
        self.row_w = w.to(DEV)
        self.wr = w.reshape(-1).numpy()[self.src_np].astype(np.float64)
        self.dYp = (self.dY[token].float() * self.row_w.view(-1)[self.src.long()][:, None]).to(torch.bfloat16)
        self.values = [None if t is None else [qo.quantised_matrix(np_of(t[e])) for e in range(E)] for t in self.W]
        self.weights = m.MoEQuantWeights(self.shape, E, gated=gated)
        self.weights.update(*self.W)
        rows = lambda x: (u8(x.shape[0], m.moe_quant_row_bytes(d)), u8(x.shape[0], m.moe_quant_scale_bytes(d)))
        # rows read in place: the tokens' own order; else grouped rows, and the weights of the combine are in dYp
        self.x, self.dy = (self.X, self.dY) if gather else (self.Xp, self.dYp)
        self.xq, self.dyq = rows(self.x), rows(self.dy)
        m.moe_quant_rows(self.x, *self.xq)
        m.moe_quant_rows(self.dy, *self.dyq)
        at = self.src_np // k if gather else slice(None)
        self.xv, self.dyv = (qo.quantised(np_of(t))[at] for t in (self.x, self.dy))
        self.ws = u8(max(m.moe_quant_expert_fwd_workspace_bytes(self.shape, E, self.n), m.moe_quant_expert_bwd_workspace_bytes(self.shape, E, self.n)))
        new = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device=DEV)
        self.G, self.U, self.H, self.Y, self.dX = new(self.n, F), new(self.n, F), new(self.n, F), new(self.n, d), new(self.n, d)
        self.ids, self.n_active = torch.full((E,), -7, dtype=torch.int32, device=DEV), torch.full((1,), -7, dtype=torch.int32, device=DEV)
        self.dW = [new(E, d, F), new(E, d, F) if gated else None, new(E, F, d)]

    def forward(self, keep=True, Y=None, plan=None, stream=None):
        g = (self.G, self.U if self.gated else None, self.H) if keep else (None, None, None)
        moe().moe_quant_expert_fwd(self.shape, self.E, self.off, self.n, self.src if self.gather else None, *self.xq, self.weights, *g,
                                   self.Y if Y is None else Y, self.ws, plan, stream)

    def backward(self, stream=None):
        moe().moe_quant_expert_bwd(self.shape, self.E, self.off, self.n, self.src if self.gather else None, self.row_w if self.gather else None,
                                   *self.dyq, self.Xp, self.weights, self.G, self.U if self.gated else None, self.H, self.dYp, self.dX, self.ids,
                                   self.n_active, *self.dW, self.ws, stream)


def group_bound(rows, off, mats, ref):
    out = np.zeros_like(ref)
    for e, w in enumerate(mats):
        x, y = off[e], off[e + 1]
        out[x:y] = product_bound(rows[x:y], w, ref[x:y])
    return out


def rel(got, ref):
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))


@pytest.mark.parametrize("case", EXPERTS)
def test_experts_forward(case):
    L = Layer(*case)
    L.forward()
    G, U, H, _ = qo.experts_fwd(L.xv, L.bounds, *L.values)
    got = {n: np_of(getattr(L, n)) for n in "GUHY"}
    eG = group_bound(L.xv, L.bounds, L.values[0], G)
    assert (np.abs(got["G"] - G) <= eG).all()
    if L.gated:
        eU = group_bound(L.xv, L.bounds, L.values[1], U)
        assert (np.abs(got["U"] - U) <= eU).all()
        # H comes from the unrounded sums: |silu'| <= 1.1, |silu(g)| <= |g|; 2^-18 |h| for the hardware's exponential and reciprocal
        fG, fU = eG - 2.0 ** -8 * np.abs(G), eU - 2.0 ** -8 * np.abs(U)
        eH = 1.1 * fG * (np.abs(U) + fU) + np.abs(G) * fU
    else:
        eH = 1.2 * (eG - 2.0 ** -8 * np.abs(G)) + 3e-7 * np.abs(G)   # |gelu'| <= 1.2; erf's approximation 1.5e-7
    # (a result below bf16's half step of the largest rounding: 2^-8 of what it may be)
    assert (np.abs(got["H"] - H) <= (2.0 ** -8 + 2.0 ** -17) * (np.abs(H) + eH) + eH + 1e-37).all()
    # the H that is kept is the one whose codes are used
    hq = qo.quantised(got["H"])
    ref = qo.grouped(hq, L.bounds, L.values[2])
    assert (np.abs(got["Y"] - ref) <= group_bound(hq, L.bounds, L.values[2], ref)).all()
    # a pass that keeps nothing gives the same bits
    Y = torch.full_like(L.Y, float("nan"))
    L.forward(keep=False, Y=Y)
    assert torch.equal(Y.view(torch.int16), L.Y.view(torch.int16))


@pytest.mark.parametrize("case", EXPERTS + TALL)
def test_experts_backward(case):
    """dX and the weight gradients in the 2-norm: their own rounding, 2^-8, and what becomes of dG and dU that lie near a border of bf16 or
    e4m3 and fall on its other side: fewer than one in 2^8 (the products' error is below 2^-12 of a value, a step of e4m3 at least 2^-4 of
    it), by one step of at most 2^-3: 2^-3 * 2^-4 = 2^-7.  The weight gradients see steps of bf16 only: 2^-8 in place of that."""
    L = Layer(*case)
    assert small_tiles(L.E, L.n, L.shape.d, L.shape.d_ff) == (case in EXPERTS)
    L.forward()
    L.backward()
    G, U, H = (np_of(t) for t in (L.G, L.U, L.H))
    w = L.wr if L.gather else None
    dX, dG, dU = qo.experts_bwd(L.dyv, w, G, U if L.gated else None, L.bounds, *L.values)
    assert rel(np_of(L.dX), dX) <= 2.0 ** -8 + 2.0 ** -7
    counts = np.diff(L.bounds)
    active = np.nonzero(counts)[0]
    n = int(L.n_active.item())
    assert n == len(active) and np.array_equal(L.ids.cpu().numpy(), np.concatenate([active, -np.ones(L.E - n)]))
    Xp, dYp = np_of(L.Xp), np_of(L.dYp)
    for slot, e in enumerate(active):
        x, y = L.bounds[e], L.bounds[e + 1]
        pairs = [(L.dW[0], Xp, dG), (L.dW[1], Xp, dU), (L.dW[2], H, dYp)]
        for t, a, b in pairs:
            if t is not None:
                assert rel(np_of(t[slot]), a[x:y].T @ b[x:y]) <= 2.0 ** -7
    for t in L.dW:
        assert t is None or bool(torch.isnan(t[n:].float()).all())   # slots of no expert are not written


@pytest.mark.parametrize("gated", [True, False])
def test_infinities_stay_in_their_rows(gated):
    """A token with an infinity and one with NaN: their own rows come out as NaN, all others with the bits they have without them."""
    L = Layer(40, 3, 1, 136, 72, gated, False)
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    outs = (L.G, L.U, L.H, L.Y, L.dX) if gated else (L.G, L.H, L.Y, L.dX)
    ref = [t.clone() for t in outs]
    m = moe()
    L.x[7, 5], L.x[20, 100] = float("inf"), float("nan")
    L.dy[31, 3] = float("nan")
    m.moe_quant_rows(L.x, *L.xq)
    m.moe_quant_rows(L.dy, *L.dyq)
    L.forward()
    L.backward()
    for t, r in zip(outs, ref):
        bad = [7, 20, 31] if t is L.dX else [7, 20]
        good = [i for i in range(40) if i not in bad]
        assert torch.equal(t[good].view(torch.int16), r[good].view(torch.int16)) and bool(torch.isnan(t[bad].float()).all())


def test_gradient_against_differences():
    """The directional derivative of a loss through the same matrices without rounding: an operand is off by at most 2^-4 of itself, and three
    quantised ones lie between the loss and dX."""
    L = Layer(40, 3, 2, 128, 192, True, False)
    L.forward()
    L.backward()
    dX, dYp = np_of(L.dX), L.dyv
    loss = lambda x: float((qo.experts_fwd(x, L.bounds, *L.values, quant_h=False)[3] * dYp).sum())
    h = 1e-4 / np.abs(dX).max()
    diff = (loss(L.xv + h * dX) - loss(L.xv - h * dX)) / (2 * h)
    assert abs(diff - (dX * dX).sum()) <= 3 * 2.0 ** -4 * (dX * dX).sum()


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,E,k,d,F", [(1, 1, 1, 256, 136), (3, 2, 1, 1000, 64), (20, 1, 1, 264, 200), (50, 1, 1, 136, 136), (90, 2, 2, 256, 256)])
def test_few_values_are_computed_without_alignment(T, E, k, d, F, gated):
    """What is quantised behind a product of up to 2^16 values: every row and column holds two products of 448^2 that cancel, the other ones are 1, 0 or -1.
    All partial sums are whole numbers below 2^24, and what is left, of K products of variance 4/9, one of up to 256: exact in fp32 and in bf16.  An
    instruction that drops what lies 13 bits below the largest of eight products loses it.  g = 32, whose sigmoid is 1 in fp32, scales dU by 32."""
    L = Layer(T, E, k, d, F, gated, True)
    assert L.n * F <= 1 << 16
    g = torch.Generator().manual_seed(T + d)
    small = lambda *s: torch.randint(-1, 2, s, generator=g).float()
    x, dy, wg, wd = small(T, d), small(T, d), small(E, d, F), small(E, F, d)
    for t, at, sign in ((x, 5, 1), (dy, 17, 1)):
        t[:, at], t[:, at + 1] = 448, 448 * sign
    wg[:, 5], wg[:, 6] = 448, -448
    wd[:, :, 17], wd[:, :, 18] = 448, -448
    to = lambda t: t.to(torch.bfloat16).to(DEV)
    L.X, L.dY, L.row_w = to(x), to(dy), torch.ones(T, k, device=DEV)
    L.weights.update(to(wg), to(wg) if gated else None, to(wd))
    moe().moe_quant_rows(L.X, *L.xq)
    moe().moe_quant_rows(L.dY, *L.dyq)
    token = L.src_np // k
    G = qo.grouped(np_of(x)[token], L.bounds, [np_of(w) for w in wg])
    dH = qo.grouped(np_of(dy)[token], L.bounds, [np.ascontiguousarray(np_of(w).T) for w in wd])
    assert max(np.abs(G).max(), np.abs(dH).max()) <= 256
    L.forward()
    assert np.array_equal(np_of(L.G), G)
    if gated:
        assert np.array_equal(np_of(L.U), G)
    # the gradient of each row by itself: the weight gradient of an operand that has a one in a column of that row's own
    L.G.fill_(32)
    if gated:
        L.U.zero_()
    L.Xp = torch.zeros(L.n, d, dtype=torch.bfloat16, device=DEV)
    L.Xp[torch.arange(L.n), torch.arange(L.n) % d] = 1
    assert L.n <= d
    L.backward()
    got, scale = (L.dW[1], 32) if gated else (L.dW[0], 1)   # (gelu'(32) is 1)
    slot = 0
    for e in range(E):
        a, b = L.bounds[e], L.bounds[e + 1]
        if b > a:
            assert np.array_equal(np_of(got[slot])[a:b], scale * dH[a:b])
            slot += 1


def test_experts_without_rows():
    L = Layer(20, 4, 2, 64, 64, True, False)
    m = moe()
    off = torch.zeros(5, dtype=torch.int32, device=DEV)
    none = lambda c: torch.empty(0, c, dtype=torch.bfloat16, device=DEV)
    q = (u8(0, 128), u8(0, 1))
    m.moe_quant_expert_fwd(L.shape, 4, off, 0, None, *q, L.weights, none(64), none(64), none(64), none(64), L.ws)
    m.moe_quant_expert_bwd(L.shape, 4, off, 0, None, None, *q, none(64), L.weights, none(64), none(64), none(64), none(64), none(64), L.ids,
                           L.n_active, *L.dW, L.ws)
    assert int(L.n_active.item()) == 0 and L.ids.tolist() == [-1] * 4
    # all groups empty although there are rows: nothing is touched
    L.off = off
    L.forward()
    L.backward()
    assert bool(torch.isnan(L.Y.float()).all()) and bool(torch.isnan(L.dX.float()).all()) and bool(torch.isnan(L.dW[0].float()).all())
    assert int(L.n_active.item()) == 0


def test_experts_in_a_graph_and_on_another_stream():
    """Captured and replayed between eager calls, and on a side stream: the same bits."""
    L = Layer(200, 5, 2, 256, 136, True, True)
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    outs = [L.G, L.U, L.H, L.Y, L.dX, L.dW[0], L.dW[1], L.dW[2]]
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    L.forward(stream=side)
    L.backward(stream=side)
    side.synchronize()
    same = lambda: all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(outs, ref))
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.forward()
        L.backward()
    for i in range(3):
        for t in outs[:5]:
            t.fill_(float(i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(), i
        L.forward(keep=False, Y=torch.empty_like(L.Y))   # eager work between replays, on the same workspace
        torch.cuda.synchronize()


def test_refusals_of_the_binding(monkeypatch):
    m = moe()
    L = Layer(20, 4, 2, 64, 64, True, True)
    with monkeypatch.context() as other:   # as if another GPU were the current one
        other.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(m.MoEError, match="current device"):
            m.moe_quant_rows(L.X, *L.xq)
        with pytest.raises(m.MoEError, match="current device"):
            L.weights.update(*L.W)
        with pytest.raises(m.MoEError, match="current device"):
            L.forward()
        with pytest.raises(m.MoEError, match="current device"):
            m.moe_grad_norm([], torch.zeros(1, device=DEV), L.ws)
    with pytest.raises(m.MoEError, match="shape"):
        m.moe_quant_rows(torch.randn(4, 64, device=DEV), u8(4, 64), u8(4, 1))
    with pytest.raises(m.MoEError, match="float32 or bfloat16"):
        m.moe_quant_rows(torch.zeros(4, 64, device=DEV, dtype=torch.float16), u8(4, 128), u8(4, 1))
    with pytest.raises(m.MoEError, match="adjacent"):
        m.moe_quant_rows(torch.randn(64, 4, device=DEV).t(), u8(4, 128), u8(4, 1))
    with pytest.raises(m.MoEError, match="overlap"):
        m.moe_quant_rows(torch.randn(64, device=DEV).expand(4, 64), u8(4, 128), u8(4, 1))
    with pytest.raises(m.MoEError, match="experts of"):
        m.moe_quant_expert_fwd(m.MoEShape(20, 64, 4, 2, 72, "bf16"), 4, L.off, L.n, L.src, *L.xq, L.weights, L.G, L.U, L.H, L.Y, L.ws)
    with pytest.raises(m.MoEError, match="backward"):
        W = m.MoEQuantWeights(L.shape, 4, backward=False)
        m.moe_quant_expert_bwd(L.shape, 4, L.off, L.n, L.src, L.row_w, *L.dyq, L.Xp, W, L.G, L.U, L.H, L.dYp, L.dX, L.ids, L.n_active, *L.dW, L.ws)
    with pytest.raises(m.MoEError, match="Wu goes with"):
        L.weights.update(L.W[0], None, L.W[2])
    with pytest.raises(m.MoEError, match="workspace"):
        m.moe_quant_expert_fwd(L.shape, 4, L.off, L.n, L.src, *L.xq, L.weights, L.G, L.U, L.H, L.Y, L.ws[:16])


# --------------------------------------------------------------------------------------------- layer
@pytest.mark.parametrize("T,E,k,d,F,S,Fs,overlap,fused,gated,gated_s", [
    (1, 8, 2, 128, 64, 0, 0, False, True, True, True), (130, 6, 2, 256, 200, 0, 0, False, True, True, True),
    (300, 5, 3, 136, 264, 2, 72, False, True, True, True), (257, 4, 2, 128, 128, 1, 64, True, True, True, False),
    (200, 6, 2, 200, 136, 1, 128, True, False, False, True), (0, 4, 2, 64, 64, 1, 64, False, True, True, True),
    (1800, 4, 2, 1024, 128, 1, 64, False, True, True, True)])
def test_layer(T, E, k, d, F, S, Fs, overlap, fused, gated, gated_s):
    """MoEHotPath with quant: the routed experts are the separate calls bit for bit, the shared ones those of the layer without; then the clipping
    of its gradients against their 64-bit norm."""
    m = moe()
    shape = m.MoEShape(T, d, E, k, F, "bf16", "softmax", True)
    g = torch.Generator().manual_seed(T + d)
    bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).to(DEV)
    X, dY, logits = bf(T, d), bf(T, d), torch.randn(T, E, generator=g).to(DEV)
    W = [bf(E, d, F, std=d ** -0.5), bf(E, d, F, std=d ** -0.5) if gated else None, bf(E, F, d, std=F ** -0.5)]
    Ws = [bf(S, d, Fs, std=d ** -0.5), bf(S, d, Fs, std=d ** -0.5) if gated_s else None, bf(S, Fs, d, std=Fs ** -0.5)] if S else [None] * 3
    weights = m.MoEQuantWeights(shape, E, gated=gated)
    weights.update(*W)
    hp = m.MoEHotPath(shape, S, Fs, DEV, overlap_shared=overlap, aux_alpha=0.001, fused=fused, quant=True)
    for t in hp.b.values():
        if t.dtype == torch.bfloat16:
            t.zero_()
    hp.forward(logits, X, weights, None, None, *Ws)
    hp.backward(dY, X, weights, None, None, *Ws)
    torch.cuda.synchronize()
    b, A = hp.b, T * k
    ref = m.MoEHotPath(shape, S, Fs, DEV, aux_alpha=0.001, fused=fused)
    ref.forward(logits, X, *W, *Ws)
    ref.backward(dY, X, *W, *Ws)
    same = lambda x, y: torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y)
    for n in ("topk_idx", "topk_w", "counts", "offsets", "src_of", "Xp", "active_ids", "n_active"):
        assert same(b[n], ref.b[n]), n
    if S:   # (common launches of bf16 sets may sum in other parts)
        for n in ("Ysh", "dXsh", "dWsg", "dWsd"):
            assert T == 0 or rel(np_of(b[n]), np_of(ref.b[n])) <= 2.0 ** -7, n
    if T:
        new = {n: torch.zeros_like(b[n]) for n in ("G", "U", "H", "Yp", "dXp", "dWg_c", "dWu_c", "dWd_c", "active_ids", "n_active")}
        xq, dq = ((u8(T, m.moe_quant_row_bytes(d)), u8(T, m.moe_quant_scale_bytes(d))) for _ in range(2))
        ws = u8(max(m.moe_quant_expert_fwd_workspace_bytes(shape, E, A), m.moe_quant_expert_bwd_workspace_bytes(shape, E, A)))
        m.moe_quant_rows(X, *xq)
        m.moe_quant_rows(dY, *dq)
        U = new["U"] if gated else None
        m.moe_quant_expert_fwd(shape, E, b["offsets"], A, b["src_of"], *xq, weights, new["G"], U, new["H"], new["Yp"], ws)
        m.moe_quant_expert_bwd(shape, E, b["offsets"], A, b["src_of"], b["topk_w"], *dq, b["Xp"], weights, b["G"], b["U"] if gated else None, b["H"],
                               b["dYp"], new["dXp"], new["active_ids"], new["n_active"], new["dWg_c"], new["dWu_c"] if gated else None, new["dWd_c"], ws)
        for n in new:
            assert same(new[n], b[n]), n
        # and near the layer in bf16: an operand of e4m3 is off by at most 2^-4 of itself, three lie one behind the other on the longest way
        for n in ("Y", "dX"):
            assert rel(np_of(b[n]), np_of(ref.b[n])) <= 3 * 2.0 ** -4, n
    grads = hp.gradients(gated, gated_s)
    n = int(b["n_active"].item())
    flat = [np_of(t[0][:n]) if isinstance(t, tuple) else np_of(t) for t in grads]
    total = float(np.sqrt(sum((x ** 2).sum() for x in flat)))
    norm, nws = torch.zeros(1, device=DEV), u8(m.moe_grad_norm_workspace_bytes())
    m.moe_grad_norm(grads, norm, nws)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    m.moe_grad_clip(grads, norm, 0.5 * total)
    m.moe_grad_norm(grads, norm, nws)
    assert abs(float(norm) - 0.5 * total) <= 2.0 ** -8 * total + 1e-6   # every value rounded to bf16 again
    with pytest.raises(m.MoEError, match="MoEQuantWeights"):
        hp.forward(logits, X, *W, *Ws)
    with pytest.raises(m.MoEError, match="MoEQuantWeights"):
        ref.backward(dY, X, weights, None, None, *Ws)


def test_layer_in_a_graph():
    """A captured forward and backward pass of the layer between eager ones, the weights quantised anew in between."""
    m = moe()
    T, E, k, d, F = 150, 6, 2, 256, 136
    shape = m.MoEShape(T, d, E, k, F, "bf16", "softmax", True)
    g = torch.Generator().manual_seed(9)
    bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).to(DEV)
    X, dY, logits = bf(T, d), bf(T, d), torch.randn(T, E, generator=g).to(DEV)
    W = [bf(E, d, F, std=d ** -0.5), bf(E, d, F, std=d ** -0.5), bf(E, F, d, std=F ** -0.5)]
    weights = m.MoEQuantWeights(shape, E)
    hp = m.MoEHotPath(shape, 0, 0, DEV, quant=True)
    step = lambda: (weights.update(*W), hp.forward(logits, X, weights), hp.backward(dY, X, weights))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    names = ("Y", "dX", "dlogits", "dWg_c", "dWu_c", "dWd_c")
    n = int(hp.b["n_active"].item())
    pick = lambda: [hp.b[x][:n].clone() if x.endswith("_c") else hp.b[x].clone() for x in names]
    for i in range(3):
        W[0].mul_(0.9)
        X.mul_(1.1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = pick()
        for x in names:
            hp.b[x].zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, pick())), i


def test_layer_refuses_fp32():
    m = moe()
    with pytest.raises(m.MoEError, match="bf16"):
        m.MoEHotPath(m.MoEShape(8, 64, 4, 2, 64, "f32"), quant=True)


@pytest.mark.parametrize("case", [(60, 3, 2, 256, 136, True, False), (100, 12, 4, 264, 392, True, False), (600, 5, 2, 256, 384, False, False),
                                  (1700, 4, 1, 2056, 200, True, False)])
@pytest.mark.parametrize("graph", [False, True])
def test_rows_of_no_group(case, graph):
    """Rows ahead of the first and behind the last group, of NaN codes, exponents of 255 and NaN: their outputs stay as they were, and nothing of them
    reaches another row or a weight gradient, whichever tiles the call takes; eager and in a graph."""
    L = Layer(*case)
    off = L.bounds.copy()
    off[:] = np.clip(off, 5, L.n - 37)
    L.off = torch.from_numpy(off).to(DEV)

    def run():
        L.forward()
        L.backward()

    outs = [L.G, L.H, L.Y, L.dX] + ([L.U] if L.gated else [])
    grads = [t for t in L.dW if t is not None]
    run()
    inside = slice(5, L.n - 37)
    n = int(L.n_active.item())
    ref = [t[inside].clone() for t in outs] + [t[:n].clone() for t in grads]
    for rows in (slice(0, 5), slice(L.n - 37, L.n)):
        for t in (*L.xq, *L.dyq):
            t[rows] = 255
        for t in (L.Xp, L.dYp):
            t[rows] = float("nan")
        for t in outs:
            t[rows] = 7
    L.ws.fill_(255)
    for t in grads:
        t.fill_(7)
    if graph:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            run()
    for _ in range(3 if graph else 1):
        for t in outs:
            t[inside] = 0 if t is L.Y or t is L.dX else t[inside]
        g.replay() if graph else run()
        torch.cuda.synchronize()
        got = [t[inside] for t in outs] + [t[:n] for t in grads]
        assert int(L.n_active.item()) == n and all(bool(torch.isfinite(t.float()).all()) for t in got)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, ref))
        for t in outs:
            assert bool((t[:5] == 7).all()) and bool((t[L.n - 37:] == 7).all())
        assert all(bool((t[n:] == 7).all()) for t in grads)
