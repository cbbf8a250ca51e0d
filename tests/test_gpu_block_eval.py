"""A block evaluated through the object that trains it: forward(training=False) takes no mask and keeps no statistics, bit for bit what a block without dropout computes."""
import pytest
import torch

from tests.test_gpu_block import Block

pytestmark = pytest.mark.gpu

NAMES = ("Xn", "logits", "Y", "Out", "topk_idx", "seq_loss", "seq_counts", "seq_P")


def results(B):
    return {n: B.hp.b[n].clone() for n in NAMES + (("Z",) if B.R is not None else ())}


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_evaluation(dtype, residual, kind):
    kw = dict(T=90, dtype=dtype, kind=kind, residual=residual, seqs=([0, 40], [35, 50]))
    B, plain = Block(p=0.3, **kw), Block(p=0.0, **kw)
    B.forward()
    B.backward()
    trained, step = results(B), B.outputs()
    statistics = B.hp.b["mean"].clone(), B.hp.b["rstd"].clone()
    assert B.forward(training=False) is B.hp.b["Out"]
    plain.forward()
    for (n, a), b in zip(results(B).items(), results(plain).values()):
        assert torch.equal(a, b), n
    assert not torch.equal(B.hp.b["Out"], trained["Out"])
    assert torch.equal(B.hp.b["mean"], statistics[0]) and torch.equal(B.hp.b["rstd"], statistics[1])
    B.forward()   # the same step's masks again
    B.backward()
    for now, then in ((results(B), trained), (B.outputs(), step)):
        assert all(torch.equal(now[n], then[n]) for n in then)
    B.check()


def test_no_backward_pass_follows():
    import paper_2502_02581_amd as moe

    B = Block()
    B.forward(training=False)
    with pytest.raises(moe.MoEError, match="without training"):
        B.backward()
    B.forward()
    B.backward()
    B.check()


def test_evaluation_in_a_graph():
    B = Block(T=60, dtype="bf16")
    B.forward(training=False)
    want = results(B)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.forward(training=False)
    for _ in range(3):
        B.forward()   # training passes between the replays
        B.backward()
        B.rng[1] += 1
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in want.items():
            assert torch.equal(B.hp.b[n], t), n
