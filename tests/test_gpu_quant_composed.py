"""The block-scaled forward pass against the calls it consists of, and what the 8-bit instruction's sums do to the values that are quantised behind them."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo

from .test_gpu_quant import DEV, Layer, moe, np_of, rel, u8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [(300, 6, 3, 200, 264, True, False), (520, 2, 1, 264, 648, False, False), (1700, 4, 1, 2056, 200, True, False),
                                  (512, 40, 2, 128, 72, True, False), (3500, 3, 1, 1000, 136, True, False)])
def test_forward_is_the_public_calls_bit_for_bit(case):
    """Above 2^16 values of H, with offsets: G and U are moe_quant_gemm's, Y that of moe_quant_rows of H; whichever tiles each of the calls takes."""
    L = Layer(*case)
    m, d, F = moe(), L.shape.d, L.shape.d_ff
    assert L.n * F > 1 << 16
    L.forward()
    ws = u8(max(m.moe_quant_gemm_workspace_bytes(L.E, L.n, d, F), m.moe_quant_gemm_workspace_bytes(L.E, L.n, F, d)))

    def product(K, N, a, w):
        C = torch.full((L.n, N), 7.0, dtype=torch.bfloat16, device=DEV)
        m.moe_quant_gemm(L.off, K, *a, *w, C, ws)
        return C

    hq = u8(L.n, m.moe_quant_row_bytes(F)), u8(L.n, m.moe_quant_scale_bytes(F))
    m.moe_quant_rows(L.H, *hq)
    pairs = [(L.G, product(d, F, L.xq, L.weights.WgT)), (L.Y, product(F, d, hq, L.weights.WdT))]
    if L.gated:
        pairs.append((L.U, product(d, F, L.xq, L.weights.WuT)))
    for a, b in pairs:
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("case", [(1100, 3, 1, 384, 64, True, False), (300, 6, 3, 200, 264, True, True), (100, 2, 1, 2048, 704, False, False),
                                  (2100, 4, 2, 256, 136, True, True), (64, 8, 4, 1000, 328, True, False)])
def test_values_that_the_instruction_moves(case):
    """Just above 2^16 values of H and beyond.  A sum of the instruction is off by e = 1.5e-5 of its terms' 2-norm t, so a value of H by the standard deviation
    s = e t (f_G^2 + f_U^2)^(1/2) of its two sums (f: the derivatives of H), and the hardware's exponential and reciprocal add 2^-18 of it.  It becomes another e4m3 value
    where a border lies between: borders are a step of e4m3 apart, 2^-3 of the value's power of two and at least 2^-9 of the block's 2^e, and a normal error of
    deviation s << step crosses one with the probability E|error| / step = (2 / pi)^(1/2) s / step.  The number of moved values is that sum over all values, held
    to half as much again and six of its standard deviations (for normal products 1.6e-3 of the values of silu(G) U and 1.0e-3 of gelu(G), small ones most of all).
    (Values next to zero whose deviation is more than a step are counted with probability 1.)  Where two values differ by x, their codes' values differ by at most x, half a
    step for each rounding to e4m3 and half a step of bf16, 2^-4 of those, for each to bf16: by six deviations and 17/16 of a step, which is 2^-3 of the smaller value or
    the block's smallest.  Y is then off by its rounding, 2^-8 / sqrt(3) in the 2-norm, and by the moved
    values' share of H, as random directions add up (a fifth for the spread of that)."""
    L = Layer(*case)
    assert L.n * L.shape.d_ff > 1 << 16
    L.forward()
    G, U, H, Y = qo.experts_fwd(L.xv, L.bounds, *L.values)
    own, ref = qo.quantised(np_of(L.H)), qo.quantised(qo.bf16(H))
    square = lambda ws: [w * w for w in ws]
    tG = qo.grouped(L.xv ** 2, L.bounds, square(L.values[0]))
    if L.gated:
        tU = qo.grouped(L.xv ** 2, L.bounds, square(L.values[1]))
        sig = 1 / (1 + np.exp(-G))
        var = tG * (U * (sig + G * sig * (1 - sig))) ** 2 + tU * (G * sig) ** 2
    else:
        var = tG * (qo._phi(G) + G * np.exp(-G * G / 2) / np.sqrt(2 * np.pi)) ** 2
    deviation = np.sqrt(1.5e-5 ** 2 * var + (2.0 ** -18 * H) ** 2)
    pad = -ref.shape[1] % 128
    blocks = np.pad(np.maximum(np.abs(own), np.abs(ref)), ((0, 0), (0, pad))).reshape(len(ref), -1, 128).max(2).repeat(128, 1)[:, :ref.shape[1]]
    smallest = 2.0 ** -9 / 224 * blocks   # (a block's maximum is above 224 2^e; half of it or more)
    step = np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(H), 1e-300))) - 3), smallest / 2)
    expected = np.minimum(np.sqrt(2 / np.pi) * deviation / step, 1).sum()
    moved = own != ref
    assert moved.sum() <= 1.5 * expected + 6 * np.sqrt(expected)
    apart = np.abs(own - ref) - 6 * deviation - 17 / 16 * np.maximum(2.0 ** -3 * np.minimum(np.abs(own), np.abs(ref)), smallest)
    assert float(apart.max()) <= 0
    share = rel(own, ref)
    assert rel(np_of(L.Y), Y) <= np.sqrt(2.0 ** -16 / 3 + (1.2 * share) ** 2)
