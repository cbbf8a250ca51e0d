"""The block-scaled experts on another stream and in graphs, every output cleared ahead of every run: each run has to write all of them."""
import numpy as np
import pytest
import torch

from .test_gpu_quant import Layer, moe

pytestmark = pytest.mark.gpu
# calls of few values, on small tiles with a plan, in common launches with the weight gradients first and last; gated or not; rows in place or grouped
CASES = [(60, 3, 2, 256, 136, True, True), (100, 12, 4, 264, 392, False, True), (700, 5, 2, 256, 384, True, False), (1700, 4, 1, 2056, 200, True, True),
         (3500, 3, 1, 1000, 136, False, True)]


class Bits:
    """The outputs of a layer: cleared, and compared with those of its first run."""

    def __init__(self, L):
        self.L = L
        self.outs = [t for t in (L.G, L.U if L.gated else None, L.H, L.Y, L.dX, *L.dW, L.ids, L.n_active) if t is not None]
        self.n = int(L.n_active.item())
        self.ref = [self.part(t).clone() for t in self.outs]

    def part(self, t):   # (slots of no expert are not written)
        return t[:self.n] if any(t is x for x in self.L.dW) else t

    def clear(self, value):
        for t in self.outs:
            t.fill_(value)
        torch.cuda.synchronize()

    def check(self, what):
        torch.cuda.synchronize()
        for t, r in zip(self.outs, self.ref):
            assert np.array_equal(self.part(t).cpu().view(torch.uint8).numpy(), r.cpu().view(torch.uint8).numpy()), what


@pytest.mark.parametrize("case", CASES)
def test_every_run_writes_every_output(case):
    L = Layer(*case)
    L.forward()
    L.backward()
    b = Bits(L)
    side = torch.cuda.Stream()
    b.clear(3)
    L.forward(stream=side)
    L.backward(stream=side)
    side.synchronize()
    b.check("another stream, by argument")
    b.clear(4)
    with torch.cuda.stream(side):
        L.forward()
        L.backward()
    b.check("another stream, the current one")
    both, fwd, bwd = (torch.cuda.CUDAGraph() for _ in range(3))
    with torch.cuda.graph(both):
        L.forward()
        L.backward()
    with torch.cuda.graph(fwd):   # two graphs on one workspace, replayed one behind the other
        L.forward()
    with torch.cuda.graph(bwd):
        L.backward()
    for i in range(3):
        b.clear(5 + i)
        both.replay()
        b.check(f"replay {i}")
        L.ws.fill_(255)
        b.clear(9 + i)
        fwd.replay()
        bwd.replay()
        b.check(f"replay {i} in two graphs")
        L.forward(keep=False, Y=torch.empty_like(L.Y))   # eager work between replays, on the same workspace
    torch.cuda.synchronize()


@pytest.mark.parametrize("case", [(60, 3, 2, 256, 136, True, False), (100, 12, 4, 264, 392, True, False), (600, 5, 2, 256, 384, False, False),
                                  (1700, 4, 1, 2056, 200, True, False)])
@pytest.mark.parametrize("graph", [False, True])
def test_rows_of_no_group_stay_and_all_others_are_written(case, graph):
    """Rows ahead of the first and behind the last group hold NaN codes and NaN; every other row of every output is cleared ahead of every run."""
    L = Layer(*case)
    off = np.clip(L.bounds, 5, L.n - 37)
    L.off = torch.from_numpy(off).to(L.off.device)
    L.forward()
    L.backward()
    inside, n = slice(5, L.n - 37), int(L.n_active.item())
    outs = [t for t in (L.G, L.U if L.gated else None, L.H, L.Y, L.dX) if t is not None]
    grads = [t for t in L.dW if t is not None]
    ref = [t[inside].clone() for t in outs] + [t[:n].clone() for t in grads]
    for rows in (slice(0, 5), slice(L.n - 37, L.n)):
        for t in (*L.xq, *L.dyq):
            t[rows] = 255
        for t in (L.Xp, L.dYp):
            t[rows] = float("nan")

    def run():
        L.forward()
        L.backward()

    g = torch.cuda.CUDAGraph()
    if graph:
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            run()
    for i in range(3):
        for t in outs + grads:
            t.fill_(7 + i)
        L.n_active.fill_(-1)
        L.ws.fill_(255)
        torch.cuda.synchronize()
        g.replay() if graph else run()
        torch.cuda.synchronize()
        assert int(L.n_active.item()) == n
        got = [t[inside] for t in outs] + [t[:n] for t in grads]
        for a, r in zip(got, ref):
            assert torch.equal(a.view(torch.int16), r.view(torch.int16)), i
        for t in outs:
            assert bool((t[:5] == 7 + i).all()) and bool((t[L.n - 37:] == 7 + i).all())
        assert all(bool((t[n:] == 7 + i).all()) for t in grads)


def test_two_passes_at_once():
    """Two layers and a clipping on three streams, each on its own workspace, give the bits that they give alone."""
    m = moe()
    layers = [Layer(700, 5, 2, 256, 384, True, True), Layer(1700, 4, 1, 2056, 200, True, False)]
    for L in layers:
        L.forward()
        L.backward()
    grads = [torch.randn(100003, device=layers[0].X.device), torch.randn(1 << 20, device=layers[0].X.device).to(torch.bfloat16)]
    out = [torch.empty_like(t) for t in grads]
    norm, ws = torch.zeros(1, device=grads[0].device), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=grads[0].device)

    def clip(stream=None):
        m.moe_grad_norm(grads, norm, ws, stream)
        m.moe_grad_clip(grads, norm, 1.0, out, stream)

    clip()
    torch.cuda.synchronize()
    bits, ref = [Bits(L) for L in layers], [norm.clone(), *[t.clone() for t in out]]
    streams = [torch.cuda.Stream() for _ in range(3)]
    for i in range(4):
        for b in bits:
            b.clear(i)
        for t in (norm, *out):
            t.fill_(-1)
        torch.cuda.synchronize()
        for _ in range(3):
            for L, s in zip(layers, streams):
                L.forward(stream=s)
                L.backward(stream=s)
            clip(streams[2])
        torch.cuda.synchronize()
        for b in bits:
            b.check(i)
        assert all(torch.equal(a, r) for a, r in zip((norm, *out), ref))
