"""Launches of many rounds of tiles: seven and more, where XCDs get long runs of them, and four and more, where bands come from both ends, of every kind
of block-scaled launch.  The elements against 64-bit products of the same values, on the device."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo

from .helpers import small_tiles
from .test_gpu_quant import DEV, Layer, moe, np_of, product_bound, u8

pytestmark = pytest.mark.gpu


def rounds(counts, cols, width):
    """Rounds of 256 tiles of the plan's heights (256, and what is left in tiles of 128, 64 and 32) times column tiles."""
    n = 0
    for c in counts:
        eighths = -(-(c % 256) * 8 // 256)
        n += c // 256 + (eighths > 0) + (eighths in (3, 5, 6))
    return n * -(-cols // width) / 256


def block_scaled(g, shape, cols):
    """Codes of normal values and exponents that differ from block to block, [.., cols] padded, and the 64-bit values they stand for."""
    kb = -(-cols // 128)
    q = torch.zeros(*shape, kb * 128, dtype=torch.uint8)
    q[..., :cols] = (torch.randn(*shape, cols, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return q


def values(q, s, per=1):
    """(on the device: test_quant_oracle.py holds torch's conversion against the definition)"""
    e = (s.double() - 127).repeat_interleave(128, -1).repeat_interleave(per, -2)[..., :q.shape[-2], :]
    return q.view(torch.float8_e4m3fn).double() * torch.exp2(e)


def check(C, a, b, rows):
    """|error| <= 2^-8 |c| + (2^-10 + max(K / 8, 1) 2^-24) |a||b| an element (see test_gpu_quant.py), and in the 2-norm the rounding to bf16 alone: uniform
    in half a step, 2^-8 / sqrt(3) of the smallest value of a binade, so of any; the instruction's 1.5e-5 and the sums' do not count beside it."""
    ref = a[rows] @ b
    err = (C[rows].double() - ref).abs()
    K = a.shape[1]
    assert bool((err <= 2.0 ** -8 * ref.abs() + (2.0 ** -10 + max(K / 8, 1) * 2.0 ** -24) * (a[rows].abs() @ b.abs()) + 1e-37).all())
    assert float(err.norm() / ref.norm()) <= 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("counts,K,N", [([37 * i % 300 for i in range(64)], 128, 6400), ([1] * 20 + [3000, 0, 700, 257, 130] + [65] * 30, 256, 8200),
                                        ([9000, 1, 5000], 136, 8192)])
def test_grouped_products(counts, K, N):
    m = moe()
    assert rounds(counts, N, 256) >= 7
    g = torch.Generator().manual_seed(sum(counts))
    E, n = len(counts), sum(counts)
    off = torch.tensor([0] + counts).cumsum(0).to(torch.int32)
    A, B = block_scaled(g, (n,), K).to(DEV), block_scaled(g, (E, N), K).to(DEV)
    kb = -(-K // 128)
    As, Bs = torch.randint(118, 122, (n, kb), generator=g).to(torch.uint8).to(DEV), torch.randint(116, 120, (E, -(-N // 128), kb), generator=g).to(torch.uint8).to(DEV)
    C = torch.full((n + 3, N), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = u8(m.moe_quant_gemm_workspace_bytes(E, n, K, N))
    m.moe_quant_gemm(off.to(DEV), K, A, As, B, Bs, C[:n], ws)
    a = values(A, As)
    for e in range(E):
        x, y = int(off[e]), int(off[e + 1])
        if y > x:
            check(C, a, values(B[e], Bs[e], 128).t().contiguous(), slice(x, y))
    assert bool((C[n:] == 7).all())


@pytest.mark.parametrize("n,K,N", [(15000, 128, 8192), (9001, 264, 14080), (70000, 136, 2056)])
def test_one_group(n, K, N):
    """Whole rounds of tall tiles, and a last one whose tiles are cut or not."""
    m = moe()
    assert -(-n // 256) * -(-N // 256) >= 7 * 256
    g = torch.Generator().manual_seed(n)
    kb = -(-K // 128)
    A, B = block_scaled(g, (n,), K).to(DEV), block_scaled(g, (1, N), K).to(DEV)
    As, Bs = torch.randint(118, 122, (n, kb), generator=g).to(torch.uint8).to(DEV), torch.randint(116, 120, (1, -(-N // 128), kb), generator=g).to(torch.uint8).to(DEV)
    C = torch.full((n + 3, N), 7.0, dtype=torch.bfloat16, device=DEV)
    m.moe_quant_gemm(None, K, A, As, B, Bs, C[:n], u8(m.moe_quant_gemm_workspace_bytes(1, n, K, N)))
    a, b = values(A, As), values(B[0], Bs[0], 128).t().contiguous()
    for x in range(0, n, 8192):
        check(C, a, b, slice(x, min(x + 8192, n)))
    assert bool((C[n:] == 7).all())


@pytest.mark.parametrize("case,least", [((14000, 20, 2, 128, 2816, True, True), 7), ((12000, 4, 1, 400, 6400, False, False), 4),
                                        ((11000, 12, 2, 256, 2816, True, False), 4), ((8000, 3, 2, 1032, 4104, True, True), 4)])
def test_experts(monkeypatch, case, least):
    """Gate and up, and dH with its quantised outputs beside the weight gradients, in launches of that many rounds.  Every row of a group has the bits that a call of
    that group's rows alone gives it, whose launch has few; some rows, and all of groups so small that such a call takes another instruction, against the oracle."""
    m = moe()
    T, E, k, d, F, gated, gather = case
    with monkeypatch.context() as c:   # (quantised below, where they are looked at)
        c.setattr(qo, "quantised_matrix", lambda w: w)
        c.setattr(qo, "quantised", lambda x: x)
        L = Layer(*case)
    counts = np.diff(L.bounds)
    assert not small_tiles(E, L.n, d, F)
    assert rounds(counts, F, 128 if gated else 256) >= least and rounds(counts, F, 256) >= 4
    L.forward()
    L.backward()
    outs = [t for t in (L.G, L.U if gated else None, L.H, L.Y, L.dX) if t is not None]
    assert all(bool(torch.isfinite(t.float()).all()) for t in outs)
    ids = {int(e): i for i, e in enumerate(L.ids[:int(L.n_active.item())].tolist())}
    assert sorted(ids) == list(np.nonzero(counts)[0])
    bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    looked_at = sorted(ids)[:1] + sorted(ids)[len(ids) // 2:][:1] + sorted(ids)[-1:]
    alone = 0
    for e in ids:
        x, y = int(L.bounds[e]), int(L.bounds[e + 1])
        r = y - x
        if r * F > 1 << 16:
            alone += r
            shape = m.MoEShape(r, d, 1, 1, F, "bf16")
            W = m.MoEQuantWeights(shape, 1, gated=gated)
            W.update(*[None if w is None else w[e:e + 1].contiguous() for w in L.W])
            # rows in place: these rows' tokens in their order, and their weights
            src = L.src[x:y].long()
            at = src // k if gather else torch.arange(x, y, device=DEV)
            ident, rw = (torch.arange(r, dtype=torch.int32, device=DEV), L.row_w.view(-1)[src].contiguous()) if gather else (None, None)
            G, U, H, Y, dX = bf(r, F), bf(r, F) if gated else None, bf(r, F), bf(r, d), bf(r, d)
            new = [bf(1, d, F), bf(1, d, F) if gated else None, bf(1, F, d)]
            ws = u8(max(m.moe_quant_expert_fwd_workspace_bytes(shape, 1, r), m.moe_quant_expert_bwd_workspace_bytes(shape, 1, r)))
            m.moe_quant_expert_fwd(shape, 1, i32(0, r), r, None, *(t[at] for t in L.xq), W, G, U, H, Y, ws)
            m.moe_quant_expert_bwd(shape, 1, i32(0, r), r, ident, rw, *(t[at] for t in L.dyq), L.Xp[x:y].contiguous(), W, G, U, H, L.dYp[x:y].contiguous(), dX,
                                   i32(0), i32(0), *new, ws)
            for a, b in zip([t for t in (G, U, H, Y, dX) if t is not None], outs):
                assert torch.equal(a.view(torch.int16), b[x:y].view(torch.int16)), e
            for a, b in zip(new, L.dW):   # (bf16 products, whose sums may be in other parts: two roundings to bf16)
                if a is not None:
                    ref = b[ids[e]].double()
                    assert float((a[0].double() - ref).norm()) <= 2.0 ** -7 * float(ref.norm()), e
        elif e not in looked_at:
            looked_at.append(e)
    assert alone > 0.9 * L.n
    for e in looked_at:
        x, y = int(L.bounds[e]), int(L.bounds[e + 1])
        rows = list(range(x, y)) if (y - x) * F <= 1 << 16 else sorted({x, x + 1, (x + y) // 2, y - 2, y - 1})
        wg, wd = (qo.quantised_matrix(L.values[i][e]) for i in (0, 2))
        xv = qo.quantised(L.xv[rows])
        for got, a, b in ((L.G, xv, wg), (L.Y, qo.quantised(np_of(L.H[rows])), wd)):
            assert (np.abs(np_of(got[rows]) - a @ b) <= product_bound(a, b, a @ b)).all(), e
