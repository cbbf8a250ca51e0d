"""Block-scaled tensors of more than 4 GiB, and of more values than 32 bits count: the last rows and matrices against calls of those alone; as many groups as there may be;
infinities and NaN inside tall tiles."""
import pytest
import torch

from oracle import quant_oracle as qo

from .test_gpu_quant import DEV, Layer, moe, np_of, product_bound, same_codes, u8

pytestmark = pytest.mark.gpu
bf16 = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)
i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("160 GiB of device memory")
    yield
    torch.cuda.empty_cache()


def codes(g, rows, cols):
    """Finite codes of either sign, padded."""
    q = torch.randint(0, 120, (rows, -(-cols // 128) * 128), dtype=torch.uint8, device=DEV, generator=g)
    q[:, cols:] = 0
    q[::2] |= 128   # (rows of one sign: sums that are far from zero)
    return q


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_rows():
    m = moe()
    n, cols = 36001, 60000
    assert n * cols * 2 > 1 << 32
    X = bf16(n, cols).normal_()
    Q, S = u8(n, m.moe_quant_row_bytes(cols)), u8(n, m.moe_quant_scale_bytes(cols))
    m.moe_quant_rows(X, Q, S)
    rows = [0, 17895, 17896, 35791, 35792, n - 1]   # on both sides of 2^30 and 2^31 values
    q, s = qo.quant_rows(np_of(X[rows]))
    assert (S[rows].cpu().numpy() == s).all() and same_codes(Q[rows], q)


def test_matrices():
    m = moe()
    E, K, N = 131, 4096, 4104
    assert E * K * N * 2 > 1 << 32 and E * K * N > 1 << 31
    b, r = m.moe_quant_scale_bytes, m.moe_quant_row_bytes
    W = bf16(E, K, N).normal_()
    Q, S, Qt, St = u8(E, K, r(N)), u8(E, b(K), b(N)), u8(E, N, r(K)), u8(E, b(N), b(K))
    m.moe_quant_weights(W, Q, S, Qt, St)
    for e in (0, 63, 127, E - 1):
        alone = u8(1, K, r(N)), u8(1, b(K), b(N)), u8(1, N, r(K)), u8(1, b(N), b(K))
        m.moe_quant_weights(W[e:e + 1], *alone)
        for whole, one in zip((Q, S, Qt, St), alone):
            assert torch.equal(whole[e], one[0])
    q, s = qo.quant_matrix(np_of(W[E - 1, :128]))
    assert (S[E - 1, :1].cpu().numpy() == s).all() and same_codes(Q[E - 1, :128], q)


def test_products():
    """A, the matrices and C beyond 4 GiB each; the last group against a call of its own, a few of its rows against the definition."""
    m = moe()
    n, K, N, E = 530000, 8192, 4104, 130
    assert min(n * K, n * N * 2, E * N * K) > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(3)
    A, B = codes(g, n, K), codes(g, E * N, K).view(E, N, K)
    exps = lambda *s: torch.randint(108, 112, s, dtype=torch.uint8, device=DEV, generator=g)
    As, Bs = exps(n, K // 128), exps(E, -(-N // 128), K // 128)
    first = n - 700
    off = [first * i // (E - 1) for i in range(E)] + [n]
    C, ws = bf16(n, N), u8(m.moe_quant_gemm_workspace_bytes(E, n, K, N))
    m.moe_quant_gemm(i32(*off), K, A, As, B, Bs, C, ws)
    one = bf16(700, N)
    m.moe_quant_gemm(i32(0, 700), K, A[first:], As[first:], B[E - 1:], Bs[E - 1:], one, ws)
    assert same(one, C[first:])
    whole = bf16(n, N)   # one group, no offsets: the last matrix for all rows
    m.moe_quant_gemm(None, K, A, As, B[E - 1:], Bs[E - 1:], whole, u8(m.moe_quant_gemm_workspace_bytes(1, n, K, N)))
    assert same(whole[first:], C[first:])
    del whole
    rows = [first, first + 255, first + 256, n - 1]
    a, b = qo.values(A[rows].cpu().numpy(), As[rows].cpu().numpy()), qo.values(B[E - 1].cpu().numpy(), Bs[E - 1].cpu().numpy(), 128).T
    ref = a @ b
    assert (abs(np_of(C[rows]) - ref) <= product_bound(a, b, ref)).all()


@pytest.mark.parametrize("gather", [False, True])
def test_experts(gather):
    """Saved tensors and outputs beyond 4 GiB, codes of the tokens up to there; the last group against a call of its own."""
    m = moe()
    T, k, d, F, E = (530000, 1, 4096, 4360, 3) if not gather else (524000, 1, 8192, 4360, 3)
    n, last = T * k, 800
    assert n * F * 2 > 1 << 32 and n * d * 2 > 1 << 32 and T * d < (1 << 32) - 4096
    shape = m.MoEShape(T, d, E, k, F, "bf16")
    g = torch.Generator(device=DEV).manual_seed(4)
    normal = lambda *s, std=1.0: bf16(*s).normal_(0, std, generator=g)
    W = [normal(E, d, F, std=d ** -0.5), normal(E, d, F, std=d ** -0.5), normal(E, F, d, std=F ** -0.5)]
    weights = m.MoEQuantWeights(shape, E)
    weights.update(*W)
    X = normal(T if gather else n, d)
    q = u8(X.shape[0], d), u8(X.shape[0], d // 128)
    m.moe_quant_rows(X, *q)
    src = torch.randperm(n, device=DEV, generator=g).to(torch.int32) if gather else None
    rw = torch.rand(T, k, device=DEV, generator=g) + 0.1 if gather else None
    at = (src // k).long() if gather else slice(None)
    Xp = X[at]
    dYp = Xp if rw is None else (X[at].float() * rw.view(-1)[src.long()][:, None]).to(torch.bfloat16)
    del X
    off = i32(0, n // 2, n - last, n)
    G, U, H, Y, dX = bf16(n, F), bf16(n, F), bf16(n, F), bf16(n, d), bf16(n, d)
    ids, na = i32(0, 0, 0), i32(0)
    dW = [bf16(E, d, F), bf16(E, d, F), bf16(E, F, d)]
    ws = u8(max(m.moe_quant_expert_fwd_workspace_bytes(shape, E, n), m.moe_quant_expert_bwd_workspace_bytes(shape, E, n)))
    m.moe_quant_expert_fwd(shape, E, off, n, src, *q, weights, G, U, H, Y, ws)
    m.moe_quant_expert_bwd(shape, E, off, n, src, rw, *q, Xp, weights, G, U, H, dYp, dX, ids, na, *dW, ws)
    assert ids.tolist() == [0, 1, 2] and int(na) == 3
    tail = slice(n - last, n)
    one = m.MoEShape(last, d, 1, 1, F, "bf16")
    w1 = m.MoEQuantWeights(one, 1)
    w1.update(*[w[E - 1:] for w in W])
    q1 = tuple(t[at][tail].contiguous() for t in q)
    ident, rw1 = (torch.arange(last, dtype=torch.int32, device=DEV), rw.view(-1)[src[tail].long()].contiguous()) if gather else (None, None)
    g1, u1, h1, y1, x1 = bf16(last, F), bf16(last, F), bf16(last, F), bf16(last, d), bf16(last, d)
    dw1 = [bf16(1, d, F), bf16(1, d, F), bf16(1, F, d)]
    m.moe_quant_expert_fwd(one, 1, i32(0, last), last, None, *q1, w1, g1, u1, h1, y1, ws)
    m.moe_quant_expert_bwd(one, 1, i32(0, last), last, ident, rw1, *q1, Xp[tail], w1, g1, u1, h1, dYp[tail], x1, i32(0), i32(0), *dw1, ws)
    for a, b in ((g1, G), (u1, U), (h1, H), (y1, Y), (x1, dX)):
        assert same(a, b[tail])
    for a, b in zip(dw1, dW):   # (bf16 products, whose sums may be in other parts)
        assert float((a[0].double() - b[2].double()).norm()) <= 2.0 ** -7 * float(b[2].double().norm())
    assert all(bool(torch.isfinite(t.float().sum())) for t in (Y[:100], dX[:100], Y[n // 2 - 50:n // 2 + 50], dX[n // 2 - 50:n // 2 + 50]))


@pytest.mark.parametrize("case", [(1700, 4, 1, 2056, 200, True, False), (3500, 3, 1, 1000, 136, False, False), (600, 5, 2, 256, 384, True, False)])
def test_infinities_stay_in_their_rows(case):
    """Beyond the calls of few values: rows of an infinity or NaN come out as NaN, all others with the bits that they have without them."""
    m, L = moe(), Layer(*case)
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    outs = [t for t in (L.G, L.U if L.gated else None, L.H, L.Y, L.dX) if t is not None]
    ref = [t.clone() for t in outs]
    bad, bad_dy = [0, 7, 255, 256, L.n - 1], [31, 129, 300]
    L.x[bad[:3], 5], L.x[bad[3:], 100] = float("inf"), float("nan")
    L.dy[bad_dy, 3] = float("nan")
    m.moe_quant_rows(L.x, *L.xq)
    m.moe_quant_rows(L.dy, *L.dyq)
    L.forward()
    L.backward()
    for t, r in zip(outs, ref):
        rows = bad + bad_dy if t is L.dX else bad
        good = torch.ones(L.n, dtype=torch.bool, device=DEV)
        good[rows] = False
        assert same(t[good], r[good]) and bool(torch.isnan(t[rows].float()).all())


@pytest.mark.parametrize("rows", [1, 3])
def test_as_many_groups_as_there_may_be(rows):
    """1024 groups, each third one empty: found in the offsets by the blocks themselves (up to 1024 rows), and with a plan."""
    m = moe()
    E, K, N = 1024, 264, 136
    counts = [0 if i % 3 == 1 else rows for i in range(E)]
    n = sum(counts)
    assert (n <= 1024) == (rows == 1)
    g = torch.Generator(device=DEV).manual_seed(5)
    A, B = codes(g, n, K), codes(g, E * N, K).view(E, N, -1)
    exps = lambda *s: torch.randint(108, 112, s, dtype=torch.uint8, device=DEV, generator=g)
    As, Bs = exps(n, 3), exps(E, 2, 3)
    off = torch.tensor([0] + counts).cumsum(0).to(torch.int32)
    C = torch.full((n, N), 7.0, dtype=torch.bfloat16, device=DEV)
    m.moe_quant_gemm(off.to(DEV), K, A, As, B, Bs, C, u8(m.moe_quant_gemm_workspace_bytes(E, n, K, N)))
    a, got = qo.values(A.cpu().numpy(), As.cpu().numpy()), np_of(C)
    Bn, Bsn = B.cpu().numpy(), Bs.cpu().numpy()
    for e in range(E):
        x, y = int(off[e]), int(off[e + 1])
        if y > x:
            b = qo.values(Bn[e], Bsn[e], 128).T
            assert (abs(got[x:y] - a[x:y] @ b) <= product_bound(a[x:y], b, a[x:y] @ b)).all(), e
