"""Clipping of gradients that are pieces of one buffer."""
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
