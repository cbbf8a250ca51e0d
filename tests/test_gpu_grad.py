"""moe_grad_norm and moe_grad_clip against 64-bit sums.

The norm is summed in 64 bits and rounded to fp32: half a step, 2^-24, and the square root's.  The factor is off by the rounding of the norm, of the sum
with 1e-6 and of the quotient, each at most 2^-24 (hardware division: one step, 2^-23), a value then by its own rounding."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FACTOR = 4 * 2.0 ** -23


def moe():
    import paper_2502_02581_amd as m

    return m


def calls(grads, max_norm, out=None):
    m = moe()
    norm = torch.full((1,), -1.0, device=DEV)
    ws = torch.full((m.moe_grad_norm_workspace_bytes(),), 255, dtype=torch.uint8, device=DEV)
    m.moe_grad_norm(grads, norm, ws)
    m.moe_grad_clip(grads, norm, max_norm, out)
    return float(norm.item())


def np_of(t):
    return t.detach().cpu().double().numpy()


SIZES = [[1], [7, 0, 9], [16384, 16383, 16385, 3], [1000003], [5] * 130, [8, 1 << 20, 24577]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("ratio", [0.3, 3.0])
@pytest.mark.parametrize("in_place", [False, True])
def test_norm_and_clip(dtype, sizes, ratio, in_place):
    g = torch.Generator().manual_seed(sum(sizes))
    grads = [(torch.randn(n, generator=g) * 10.0 ** (i % 5 - 2)).to(dtype).to(DEV) for i, n in enumerate(sizes)]
    ref = [np_of(t) for t in grads]
    total, _ = qo.clip(ref, 1.0)
    norm, want = qo.clip(ref, ratio * total)
    out = None if in_place else [torch.full_like(t, 7) for t in grads]
    keep = [t.clone() for t in grads]
    got = calls(grads, ratio * total, out)
    assert abs(got - norm) <= 2.0 ** -23 * norm
    half = torch.finfo(dtype).eps / 2
    for t, w, k in zip(grads if in_place else out, want, keep):
        # (values below the type's normal range are rounded to steps of its smallest one)
        assert (np.abs(np_of(t) - w) <= (half + 2 * FACTOR) * np.abs(w) + 1e-38).all()
        if ratio > 1:
            assert torch.equal(t, k)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    assert got == calls([k.clone() for k in keep], 1.0)   # the same bits again


def test_compacted_gradients():
    """Only the slots that n_active names count and are written; a device number that is larger than the tensor, or below zero, is held to it."""
    g = torch.Generator().manual_seed(5)
    for n, used in ((0, 0), (1, 1), (5, 5), (9, 9), (12, 9), (-3, 0)):
        big = torch.randn(9, 40, 33, generator=g)
        big[used:] = float("nan")
        small = torch.randn(300, generator=g)
        grads = [(big.to(torch.bfloat16).to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV)), small.to(DEV)]
        ref = [np_of(grads[0][0][:used]), np_of(grads[1])]
        norm, want = qo.clip(ref, 0.5)
        out = [torch.full_like(grads[0][0], 7), torch.full_like(grads[1], 7)]
        got = calls(grads, 0.5, out)
        assert abs(got - norm) <= 2.0 ** -23 * norm
        assert (np.abs(np_of(out[0][:used]) - want[0]) <= (2.0 ** -8 + 2 * FACTOR) * np.abs(want[0])).all()
        assert bool((out[0][used:] == 7).all())
        assert (np.abs(np_of(out[1]) - want[1]) <= (2.0 ** -24 + 2 * FACTOR) * np.abs(want[1])).all()


def test_values_at_the_ends_of_the_range():
    """Squares neither overflow nor vanish; no gradients, zeros, infinities and NaN."""
    t = lambda *v: torch.tensor(v, device=DEV)
    for scale in (1e30, 1e-30):
        x = t(3.0, 4.0) * scale
        assert abs(calls([x.clone()], 1.0) - 5 * scale) <= 1e-6 * 5 * scale
    assert calls([], 1.0) == 0.0 and calls([torch.empty(0, device=DEV)], 1.0) == 0.0
    z = torch.zeros(100, device=DEV)
    assert calls([z], 1.0) == 0.0 and bool((z == 0).all())
    x, o = t(1.0, float("inf")), t(9.0, 9.0)
    assert calls([x], 1.0, [o]) == float("inf") and o[0] == 0 and torch.isnan(o[1])
    x, y = t(1.0, float("nan")), torch.ones(5, device=DEV, dtype=torch.bfloat16)
    assert np.isnan(calls([x, y], 1.0)) and bool(torch.isnan(y.float()).all())
    y = torch.ones(4, device=DEV)
    assert calls([y], 0.0) == 2.0 and bool((y == 0).all())


def test_captured_and_replayed():
    m = moe()
    g = torch.Generator().manual_seed(1)
    grads = [torch.randn(5000, generator=g).to(DEV), (torch.randn(4, 64, generator=g).to(torch.bfloat16).to(DEV), torch.tensor([3], dtype=torch.int32, device=DEV))]
    out = [torch.zeros(5000, device=DEV), torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)]
    norm, ws = torch.zeros(1, device=DEV), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.moe_grad_norm(grads, norm, ws)
        m.moe_grad_clip(grads, norm, 1.0, out)
    for i in range(3):
        grads[0].mul_(1.5)
        grads[1][1].fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b, c = norm.clone(), out[0].clone(), out[1].clone()
        fresh = [torch.zeros_like(t) for t in out]
        n = calls(grads, 1.0, fresh)
        assert n == float(a) and torch.equal(b, fresh[0]) and torch.equal(c[:i], fresh[1][:i])


def test_refusals():
    m = moe()
    norm, ws = torch.zeros(1, device=DEV), torch.empty(16, dtype=torch.uint8, device=DEV)
    x = torch.ones(8, device=DEV)
    with pytest.raises(m.MoEError, match="workspace"):
        m.moe_grad_norm([x], norm, ws)
    with pytest.raises(m.MoEError, match="outputs"):
        m.moe_grad_clip([x], norm, 1.0, [])
    with pytest.raises(m.MoEError, match="shape"):
        m.moe_grad_clip([x], norm, 1.0, [x[:4]])
    with pytest.raises(m.MoEError, match="contiguous"):
        m.moe_grad_clip([torch.ones(4, 4, device=DEV).t()], norm, 1.0)
    with pytest.raises(m.MoEError, match="aligned"):
        m.moe_grad_clip([x[1:]], norm, 1.0)
    with pytest.raises(m.MoEError, match="float32 or bfloat16"):
        m.moe_grad_clip([x.half()], norm, 1.0)
    with pytest.raises(m.MoEError, match="twice"):
        m.moe_grad_clip([x, x], norm, 1.0)
    with pytest.raises(m.MoEError, match="twice"):
        m.moe_grad_clip([x, x.clone()], norm, 1.0, [x, x])
    with pytest.raises(m.MoEError, match="slots"):
        m.moe_grad_norm([(x[0], torch.ones(1, dtype=torch.int32, device=DEV))], norm, torch.empty(1 << 14, dtype=torch.uint8, device=DEV))
    with pytest.raises(m.MoEError, match="GPU"):
        m.moe_grad_norm([torch.ones(3)], norm, ws)


def test_clip_refuses_an_output_that_is_another_gradient():
    m = moe()
    x, y, norm = torch.ones(8, device=DEV), torch.ones(8, device=DEV), torch.ones(1, device=DEV)
    with pytest.raises(m.MoEError, match="another gradient"):
        m.moe_grad_clip([x, y], norm, 0.5, [y, torch.empty_like(x)])
    with pytest.raises(m.MoEError, match="another gradient"):
        m.moe_grad_clip([x, y], norm, 0.5, [y, x])
    m.moe_grad_clip([x, y], norm, 0.5, [x, torch.empty_like(y)])   # the first in place, the second not
    assert abs(float(x[0]) - 0.5) <= 1e-6 and float(y[0]) == 1.0   # (0.5 / (1 + 1e-6))


def test_calls_go_to_the_current_stream():
    from paper_2502_02581_amd.binding import _stream

    side = torch.cuda.Stream()
    assert _stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert _stream(None) == side.cuda_stream == _stream(side)
    graph = torch.cuda.CUDAGraph()
    x = torch.zeros(8, device=DEV)
    with torch.cuda.graph(graph):
        assert _stream(None) == torch.cuda.current_stream().cuda_stream
        x.add_(1)
    torch.cuda.synchronize()
