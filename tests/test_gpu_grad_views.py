"""Clipping of gradients that are pieces of one buffer, of a norm that fp32 does not hold, and of more values than 32 bits count."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_pieces_of_one_buffer():
    """Adjacent pieces are clipped as the whole is; pieces that share values are refused, and one gradient may be read for two outputs."""
    import paper_2502_02581_amd as m

    g = torch.Generator().manual_seed(2)
    whole = torch.randn(40000, generator=g).to(DEV)
    norm, ws = torch.zeros(1, device=DEV), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    m.moe_grad_norm([whole], norm, ws)
    limit = 0.5 * float(norm)
    want = torch.empty_like(whole)
    m.moe_grad_clip([whole], norm, limit, [want])
    cuts = [0, 4, 16384, 16400, 39996, 40000]
    pieces = [whole[a:b] for a, b in zip(cuts, cuts[1:])]
    out = torch.empty_like(whole)
    m.moe_grad_clip(pieces, norm, limit, [out[a:b] for a, b in zip(cuts, cuts[1:])])
    assert torch.equal(out, want)
    keep = whole.clone()
    for bad, outs in (([whole, whole[16:32]], None), ([whole[:64], whole[60:128]], None), ([whole[:64]], [whole[4:68]]),
                      ([whole[:64], whole[64:128]], [whole[64:128], out[:64]]), ([whole[:8], whole[8:16]], [out[:8], out[4:12]])):
        with pytest.raises(m.MoEError, match="twice|another gradient|overlaps"):
            m.moe_grad_clip(bad, norm, limit, outs)
    torch.cuda.synchronize()
    assert torch.equal(whole, keep)
    a, b = torch.empty_like(whole), torch.empty_like(whole)
    m.moe_grad_clip([whole, whole], norm, limit, [a, b])
    assert torch.equal(a, want) and torch.equal(b, want)
    m.moe_grad_clip(pieces, norm, limit)
    assert torch.equal(whole, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_beyond_fp32(dtype):
    """Below 2^128 the norm is a number and the factor scales by it; from there on it is infinite and clips to zero, infinities to NaN."""
    import paper_2502_02581_amd as m

    norm, ws = torch.zeros(1, device=DEV), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    big = 2.0 ** 127
    x, out = torch.tensor([big, big, -big], dtype=dtype, device=DEV), torch.ones(3, dtype=dtype, device=DEV)
    m.moe_grad_norm([x], norm, ws)
    assert abs(float(norm) / (big * 3 ** 0.5) - 1) <= 2.0 ** -23
    m.moe_grad_clip([x], norm, 1.0, [out])
    assert float((out.double().abs() - 3 ** -0.5).abs().max()) <= 3 ** -0.5 * (torch.finfo(dtype).eps / 2 + 2.0 ** -21)
    x = torch.tensor([big, big, -big, big, 1.0], dtype=dtype, device=DEV)
    out = torch.ones(5, dtype=dtype, device=DEV)
    m.moe_grad_norm([x], norm, ws)
    assert float(norm) == float("inf")   # 2^128 and a little more
    m.moe_grad_clip([x], norm, 1.0, [out])
    assert bool((out == 0).all())
    x[1] = float("inf")
    m.moe_grad_clip([x], norm, 1.0, [out])
    assert bool(torch.isnan(out[1])) and bool((out[[0, 2, 3, 4]] == 0).all())


def test_more_values_than_32_bits_count():
    import paper_2502_02581_amd as m

    torch.cuda.empty_cache()
    n = (1 << 32) + 24
    if torch.cuda.mem_get_info()[0] < 32 << 30:
        pytest.skip("32 GiB of device memory")
    x = torch.ones(4, n // 4, dtype=torch.bfloat16, device=DEV)   # slots of 2^30 + 6 values, three of which count
    used = torch.tensor([3], dtype=torch.int32, device=DEV)
    norm, ws = torch.zeros(1, device=DEV), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    for grads, values in (([x], n), ([(x, used)], n // 4 * 3)):
        x.fill_(1)
        x.view(-1)[-1] = 2
        m.moe_grad_norm(grads, norm, ws)
        want = (values + (3 if values == n else 0)) ** 0.5
        assert abs(float(norm) - want) <= 2.0 ** -23 * want
        m.moe_grad_clip(grads, norm, 0.5 * float(norm))
        flat = x.view(-1)
        for i in (0, 1 << 31, (1 << 32) - 8, values - 2):
            assert float(flat[min(i, values - 2)]) == 0.5
        assert bool((flat[n // 4 * 3:n // 4 * 3 + 100] == (0.5 if values == n else 1)).all()) and float(flat[-1]) == (1 if values == n else 2)
    del x
    torch.cuda.empty_cache()
