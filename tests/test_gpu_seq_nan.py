"""NaN among the logits of the sequences' losses: it reaches its token's gradient, its sequence's shares and both losses, and nothing else."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def run(x, topk, start, length, gate, alpha=0.01, beta=0.002):
    import paper_2502_02581_amd as moe

    (T, E), k, n = x.shape, topk.shape[1], len(start)
    dev = "cuda:0"
    shape = moe.MoEShape(T, 8, E, k, 8, "f32", gate)
    st, ln = (torch.tensor(v, dtype=torch.int32, device=dev) for v in (start, length))
    counts = torch.empty(n, E, dtype=torch.int32, device=dev)
    P, loss, coef, dlogits = torch.empty(n, E, device=dev), torch.empty(2, device=dev), torch.empty(n + 1, device=dev), torch.empty(T, E, device=dev)
    ws = torch.empty(moe.moe_seq_loss_workspace_bytes(shape, n), dtype=torch.uint8, device=dev)
    moe.moe_seq_loss(shape, x, topk, st, ln, alpha, beta, counts, P, loss, coef, ws)
    moe.moe_seq_loss_bwd(shape, x, st, ln, counts, coef, 1.0, False, dlogits)
    return counts, P, loss, coef, dlogits


def spoil(row, how):
    if how == "one":
        row[row.shape[0] // 2] = float("nan")
    elif how == "all":
        row[:] = float("nan")
    else:   # NaN beside nothing but -inf
        row[:] = float("-inf")
        row[-1] = float("nan")


# rows of every number of lanes; calls of one launch, of chunks of a wavefront and of a block
@pytest.mark.parametrize("T,E,S", [(40, 1, 2), (60, 7, 3), (50, 16, 2), (64, 100, 3), (30, 300, 2), (20, 700, 2), (3000, 8, 900), (2000, 30, 700), (6000, 64, 3), (900, 256, 2), (600, 1000, 2)])
@pytest.mark.parametrize("how", ["one", "all", "beside -inf"])
@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_nan_of_a_token(T, E, S, how, gate):
    g = torch.Generator().manual_seed(T + E)
    x = torch.randn(T, E, generator=g)
    topk = torch.topk(x, min(2, E), dim=1).indices.int().cuda()
    start = [T * i // S for i in range(S)]
    length = [T * (i + 1) // S - T * i // S for i in range(S)]
    clean = run(x.cuda(), topk, start, length, gate)
    token = start[-1] + length[-1] // 2
    spoil(x[token], how)
    counts, P, loss, coef, dlogits = run(x.cuda(), topk, start, length, gate)
    assert torch.equal(counts, clean[0]) and torch.equal(coef, clean[3])
    assert torch.isnan(P[-1]).all() and torch.equal(P[:-1], clean[1][:-1])
    assert torch.isnan(loss).all() and torch.isfinite(clean[2]).all()
    assert torch.isnan(dlogits[token]).all()
    others = torch.arange(T, device="cuda:0") != token
    assert torch.equal(dlogits[others], clean[4][others])


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_rows_of_minus_infinity_alone(gate):
    """They add nothing, as before."""
    x = torch.randn(50, 20, generator=torch.Generator().manual_seed(1))
    topk = torch.topk(x, 2, dim=1).indices.int().cuda()
    x[7] = x[49] = float("-inf")
    counts, P, loss, coef, dlogits = run(x.cuda(), topk, [0, 20], [20, 30], gate)
    assert torch.isfinite(P).all() and torch.isfinite(loss).all() and torch.isfinite(dlogits).all() and not dlogits[[7, 49]].any()
