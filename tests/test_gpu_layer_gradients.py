"""Clipping the gradients of layers of two-matrix experts: buffers that no such pass writes are no part of the norm."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("gated,gated_shared", [(False, False), (False, True), (True, False)])
def test_norm_of_a_layer_with_two_matrix_experts(quant, gated, gated_shared):
    import paper_2502_02581_amd as m

    T, E, k, d, F, S, Fs = 130, 6, 2, 256, 200, 2, 72
    shape = m.MoEShape(T, d, E, k, F, "bf16", "softmax", True)
    g = torch.Generator().manual_seed(17)
    bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).to(DEV)
    X, dY, logits = bf(T, d), bf(T, d), torch.randn(T, E, generator=g).to(DEV)
    W = [bf(E, d, F, std=d ** -0.5), bf(E, d, F, std=d ** -0.5) if gated else None, bf(E, F, d, std=F ** -0.5)]
    Ws = [bf(S, d, Fs, std=d ** -0.5), bf(S, d, Fs, std=d ** -0.5) if gated_shared else None, bf(S, Fs, d, std=Fs ** -0.5)]
    hp = m.MoEHotPath(shape, S, Fs, DEV, quant=quant)
    for n, t in hp.b.items():
        if n.startswith("dW"):
            t.fill_(float("nan"))
    if quant:
        weights = m.MoEQuantWeights(shape, E, gated=gated)
        weights.update(*W)
        W = [weights, None, None]
    hp.forward(logits, X, *W, *Ws)
    hp.backward(dY, X, *W, *Ws)
    grads = hp.gradients()
    n = int(hp.b["n_active"].item())
    flat = [x[0][:n] if isinstance(x, tuple) else x for x in grads]
    assert len(flat) == 4 + gated + gated_shared and all(bool(torch.isfinite(x.float()).all()) for x in flat)
    total = float(np.sqrt(sum(float(x.double().square().sum()) for x in flat)))
    norm, ws = torch.zeros(1, device=DEV), torch.empty(m.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    m.moe_grad_norm(grads, norm, ws)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total   # (rounded to fp32, behind a square root)
    m.moe_grad_clip(grads, norm, 0.25 * total)
    assert all(bool(torch.isfinite(x.float()).all()) for x in flat)
    m.moe_grad_norm(grads, norm, ws)
    assert abs(float(norm) - 0.25 * total) <= (2.0 ** -8 + 2.0 ** -21) * 0.25 * total + 1e-6   # every value rounded to bf16 again
