"""moe_seq_loss and moe_seq_loss_bwd against the 64-bit definitions.

Tolerances, u = 2^-24, logits within 12 of each other: an exponential is off by 4 u and by the rounding of its argument, 12 u; a row's sum by 12 u more; so a share by 40 u.  P adds at most 256 shares in
sequence and 400 sums of sums of positive terms: 40 + 656 < 1024 u of itself, and so (its terms are positive) is the balance.  lse is off by 16 u + u |lse|, its squares' sum by
(2 (16 + |lse|) + 700) u: 1024 u (1 + z).  dz = share (up - sum share up) (..) + c lse soft: 128 u of share (|up| + sum share |up|) + c soft (|lse| + 1)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as ob
from tests.helpers import np64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def ranges_of(start, length, T):
    """The sequences' token ranges as the header says: not beyond the next start, nor T."""
    out = []
    for s, a in enumerate(start):
        end = a + length[s] if length is not None else T
        nxt = start[s + 1] if s + 1 < len(start) else T
        out.append((a, max(a, min(end, nxt, T))))
    return out


def run(T, E, k, gate, start=None, length=None, alpha=0.01, beta=0.002, seed=0, accumulate=False, spoil=True, dloss=1.0, logits=None):
    """start, length: lists; start alone: n + 1 offsets."""
    import paper_2502_02581_amd as moe

    g = torch.Generator().manual_seed(seed + T * 31 + E)
    x = torch.randn(T, E, generator=g) + torch.randn(E, generator=g) if logits is None else logits
    topk = torch.topk(x, k, dim=1).indices.to(torch.int32) if T else torch.zeros(0, k, dtype=torch.int32)
    if start is None:
        ranges = [(0, T)]
    elif length is None:
        ranges = [(a, max(a, b)) for a, b in zip(start[:-1], start[1:])]
    else:
        ranges = ranges_of(start, length, T)
    inside = np.zeros(T, bool)
    for a, b in ranges:
        inside[a:b] = True
    lg, tk = x.clone(), topk.clone()
    if spoil and not inside.all():   # padding holds anything
        lg[torch.from_numpy(~inside)] = float("nan")
        tk[torch.from_numpy(~inside)] = 1 << 30
    n = len(ranges)
    shape = moe.MoEShape(T, 8, E, k, 8, "f32", gate)
    dev = "cuda:0"
    dl = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    st, ln = dl(start), dl(length)
    lg, tk = lg.to(dev), tk.to(dev)
    counts = torch.full((n, E), -5, dtype=torch.int32, device=dev)
    P, loss, coef = (torch.full(s, float("nan"), device=dev) for s in ((n, E), (2,), (n + 1,)))
    old = torch.randn(T, E, generator=g).to(dev)
    dlogits = old.clone() if accumulate else torch.full((T, E), float("nan"), device=dev)
    ws = torch.full((moe.moe_seq_loss_workspace_bytes(shape, n),), 255, dtype=torch.uint8, device=dev)
    moe.moe_seq_loss(shape, lg, tk, st, ln, alpha, beta, counts, P, loss, coef, ws)
    moe.moe_seq_loss_bwd(shape, lg, st, ln, counts, coef, dloss, accumulate, dlogits)
    torch.cuda.synchronize()
    x64 = np64(x)
    c64, P64, loss64, dz = ob.seq_loss(x64, topk.numpy(), ranges, k, gate, alpha, beta)
    assert np.array_equal(counts.cpu().numpy(), c64)
    assert (np.abs(np64(P) - P64) <= 1024 * U * P64).all()
    got = np64(loss)
    assert abs(got[0] - loss64[0]) <= 1024 * U * abs(loss64[0]) and abs(got[1] - loss64[1]) <= 1024 * U * (beta + loss64[1])
    soft, score, share, lse = ob.shares(x64, gate) if T else (np.zeros((0, E)),) * 3 + (np.zeros(0),)
    up = np.zeros((T, E))
    filled, tokens = max(1, sum(b > a for a, b in ranges)), max(1, sum(b - a for a, b in ranges))
    for s, (a, b) in enumerate(ranges):
        if b > a:
            up[a:b] = alpha * E / filled * c64[s] / (k * (b - a)) / (b - a)
    tol = share * (up + (share * up).sum(1, keepdims=True)) + 2 * beta / tokens * soft * (np.abs(lse) + 1)[:, None]
    tol = abs(dloss) * 128 * U * tol * inside[:, None]
    want = dloss * dz
    if accumulate:
        want = want + np64(old)
        tol = tol + U * np.abs(want)
        assert torch.equal(dlogits[torch.from_numpy(~inside).to(dev)], old[torch.from_numpy(~inside).to(dev)])
    assert (np.abs(np64(dlogits) - want) <= tol + 1e-37).all()
    return counts, P, loss, dlogits


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(1, 1), (3, 2), (4, 4), (7, 2), (8, 2), (13, 3), (16, 1), (32, 8), (60, 4), (64, 2), (100, 6), (128, 64), (256, 8), (300, 3), (512, 8), (777, 5), (1024, 8)])
def test_experts(E, k, gate):
    """Every number of lanes a row, one sequence and several, none of them on a chunk's border."""
    run(50, E, k, gate)
    run(333, E, k, gate, start=[0, 7, 90, 91, 200], length=[5, 83, 1, 60, 133])


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,S", [(16, 1024, 8, 1), (31, 513, 4, 1), (10, 1000, 64, 1), (32, 512, 2, 2), (16384, 1, 1, 5), (4096, 4, 2, 64), (4097, 4, 2, 64), (4096, 4, 2, 65), (130, 126, 3, 8)])
def test_around_the_line_of_small_calls(T, E, k, S, gate):
    """One launch or two: 16384 logits, 64 jobs of 16 experts; as many experts as its counters have room for."""
    start = [T * i // S for i in range(S)]
    run(T, E, k, gate, start=start, length=[max(0, T // S - i % 3) for i in range(S)])


def test_mixed_lengths():
    """One long sequence among hundreds of short ones: those of many pieces are joined by a wavefront, the others by four lanes."""
    start = list(range(0, 600, 2)) + [600, 30000, 30001]
    length = [1 + i % 2 for i in range(300)] + [29400, 1, 5]
    run(30010, 64, 2, "softmax", start=start, length=length)
    run(30010, 64, 2, "sigmoid", start=[0, 100] + [30000 + i for i in range(10)], length=[90, 29800] + [1] * 10)


def test_beyond_two_to_the_31_values():
    """Logits behind 2^31 others: the last of three sequences against the definition (the others: nothing, and all alike)."""
    import paper_2502_02581_amd as moe

    E, k, tail = 1024, 4, 70
    T = (1 << 31) // E + 100
    g = torch.Generator().manual_seed(2)
    x = torch.zeros(T, E, device="cuda:0")
    last = torch.randn(tail, E, generator=g)
    x[-tail:] = last.cuda()
    topk = torch.zeros(T, k, dtype=torch.int32, device="cuda:0")
    ids = torch.topk(last, k, dim=1).indices.to(torch.int32)
    topk[-tail:] = ids.cuda()
    st = torch.tensor([0, 5, T - tail, T], dtype=torch.int32, device="cuda:0")
    st[1] = 0
    shape = moe.MoEShape(T, 8, E, k, 8, "f32")
    f = dict(device="cuda:0")
    counts, P, loss, coef = torch.empty(3, E, dtype=torch.int32, **f), torch.empty(3, E, **f), torch.empty(2, **f), torch.empty(4, **f)
    ws = torch.empty(moe.moe_seq_loss_workspace_bytes(shape, 3), dtype=torch.uint8, **f)
    moe.moe_seq_loss(shape, x, topk, st, None, 0.01, 0.0, counts, P, loss, coef, ws)
    moe.moe_seq_loss_bwd(shape, x, st, None, counts, coef, 1.0, False, x)   # (over the logits: each is read before its gradient is written)
    c64, P64, _, dz = ob.seq_loss(np64(last), ids.numpy(), [(0, tail)], k, "softmax", 0.01 / 2, 0.0)
    assert np.array_equal(counts[2].cpu().numpy(), c64[0]) and int(counts[1, 0]) == k * (T - tail) and not counts[0].any()
    assert (np.abs(np64(P[2]) - P64[0]) <= 1024 * U * P64[0]).all()
    share = ob.shares(np64(last), "softmax")[0]
    up = 0.005 * E * c64[0] / (k * tail) / tail
    assert (np.abs(np64(x[-tail:]) - dz) <= 128 * U * share * (up + (share * up).sum(1, keepdims=True))).all()


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_sequences(gate):
    """Offsets without lengths, empty sequences at every place, tokens before the first and behind the last, lengths that reach beyond."""
    run(100, 16, 2, gate, start=[0, 40, 40, 100])
    run(100, 16, 2, gate, start=[0, 0, 0, 0, 100])
    run(100, 16, 2, gate, start=[10, 20, 30], length=[10, 0, 5])
    run(100, 16, 2, gate, start=[10, 20, 30], length=[50, 50, 5000])
    run(100, 16, 2, gate, start=[10, 20, 30], length=[-3, 4, 2 ** 31 - 1])
    run(100, 16, 2, gate, start=[100, 100], length=[5, 5])
    run(64, 8, 1, gate, start=[3], length=[0])


@pytest.mark.parametrize("T,E,S", [(1, 5, 1), (1000, 8, 1000), (700, 64, 350), (2000, 256, 130), (20000, 8, 3), (9000, 60, 1)])
def test_lengths(T, E, S):
    """From one token a sequence to many chunks, more sequences than a chunk's search asks for at once."""
    start = [T * i // S for i in range(S)]
    r = np.random.RandomState(T)
    length = [int(r.randint(0, 2 + T // S)) for _ in range(S)]
    run(T, E, min(2, E), "softmax", start=start, length=length)


def test_many_empty_sequences():
    start = sorted(np.random.RandomState(3).randint(0, 40, 5000).tolist())
    run(40, 12, 2, "sigmoid", start=start, length=[1] * 5000)


@pytest.mark.parametrize("alpha,beta", [(0.0, 0.1), (0.1, 0.0), (0.0, 0.0)])
@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_weights_of_the_losses(gate, alpha, beta):
    run(77, 24, 3, gate, start=[0, 30], length=[20, 47], alpha=alpha, beta=beta)


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_accumulating(gate):
    run(150, 40, 2, gate, start=[3, 60], length=[20, 80], accumulate=True, dloss=0.5)
    run(150, 41, 2, gate, start=[3, 60], length=[20, 80], dloss=-3.0)


def test_no_tokens():
    import paper_2502_02581_amd as moe

    shape = moe.MoEShape(0, 8, 6, 2, 8, "f32")
    dev = "cuda:0"
    e = torch.empty(0, 6, device=dev)
    counts, P, loss, coef = torch.full((2, 6), 3, dtype=torch.int32, device=dev), torch.ones(2, 6, device=dev), torch.ones(2, device=dev), torch.ones(3, device=dev)
    st = torch.zeros(3, dtype=torch.int32, device=dev)
    ws = torch.empty(moe.moe_seq_loss_workspace_bytes(shape, 2), dtype=torch.uint8, device=dev)
    moe.moe_seq_loss(shape, e, torch.empty(0, 2, dtype=torch.int32, device=dev), st, None, 0.1, 0.1, counts, P, loss, coef, ws)
    moe.moe_seq_loss_bwd(shape, e, st, None, counts, coef, 1.0, False, e)
    assert not counts.any() and not P.any() and not loss.any() and not coef.any()


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_masked_experts(gate):
    """Logits of -inf (experts that a token may not use), rows of nothing else, the type's lowest value, large ones."""
    x = torch.randn(60, 20, generator=torch.Generator().manual_seed(1))
    x[:, 3] = float("-inf")
    x[5] = x[59] = float("-inf")
    x[7, 4:] = torch.finfo(torch.float32).min
    if gate == "softmax":
        x[9, 0], x[10, 2] = 100.0, -1e30
    with np.errstate(over="ignore"):
        run(60, 20, 2, gate, start=[0, 20], length=[20, 40], logits=x, beta=0.0)
    run(60, 20, 2, gate, start=[0, 20], length=[5, 30], logits=torch.where(x < -1e20, torch.full_like(x, float("-inf")), x).clamp(max=10))


def test_same_bits():
    """Sums in a fixed order: another call gives the same bits, whatever the workspace held."""
    a = run(5000, 64, 2, "softmax", start=[0, 1500, 1600], length=[1490, 90, 3000])
    b = run(5000, 64, 2, "softmax", start=[0, 1500, 1600], length=[1490, 90, 3000])
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_agrees_with_the_batch_loss():
    """One sequence of all tokens and no z loss: moe_aux_loss, whose sums have another order."""
    import paper_2502_02581_amd as moe

    T, E, k = 500, 60, 4
    counts, P, loss, dl = run(T, E, k, "softmax", alpha=0.01, beta=0.0)
    g = torch.Generator().manual_seed(T * 31 + E)
    x = (torch.randn(T, E, generator=g) + torch.randn(E, generator=g)).cuda()
    shape = moe.MoEShape(T, 8, E, k, 8, "f32")
    P2, loss2, ws = torch.empty(E, device="cuda:0"), torch.empty(1, device="cuda:0"), torch.empty(moe.moe_aux_loss_workspace_bytes(shape), dtype=torch.uint8, device="cuda:0")
    d2 = torch.empty(T, E, device="cuda:0")
    moe.moe_aux_loss(shape, x, counts[0].contiguous(), 0.01, P2, loss2, ws)
    moe.moe_aux_loss_bwd(shape, x, counts[0].contiguous(), 0.01, 1.0, False, d2)
    assert torch.allclose(P2, P[0], rtol=2048 * U, atol=0) and torch.allclose(loss2, loss[:1], rtol=2048 * U, atol=0)
    assert (d2 - dl).abs().max() <= 256 * U * 2 * d2.abs().max() * E
