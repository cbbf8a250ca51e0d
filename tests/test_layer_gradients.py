"""Which weight gradients a layer lists after a backward pass (the calls that launch are left out: no GPU needed)."""
import pytest
import torch

import paper_2502_02581_amd as moe
from paper_2502_02581_amd import binding

LAUNCHES = ("moe_combine_bwd", "moe_experts_bwd", "moe_expert_bwd", "moe_quant_rows", "moe_quant_expert_bwd", "moe_combine", "moe_route_bwd",
            "moe_route_aux_bwd", "moe_aux_loss_bwd")


@pytest.fixture
def layer(monkeypatch):
    for name in LAUNCHES:
        monkeypatch.setattr(binding, name, lambda *a, **k: None)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    monkeypatch.setattr(binding.MoEQuantWeights, "_seal", lambda self: None)

    def make(S, quant):
        hp = moe.MoEHotPath(moe.MoEShape(8, 64, 4, 2, 64, "bf16"), S, 32 if S else 0, "cpu", quant=quant)
        hp._logits = None
        return hp

    return make


def listed(hp, *a, **k):
    names = {t.data_ptr(): n for n, t in hp.b.items()}
    return [names[(x[0] if isinstance(x, tuple) else x).data_ptr()] for x in hp.gradients(*a, **k)]


def backward(hp, gated, gated_shared):
    shape = hp.shape
    W = moe.MoEQuantWeights(shape, shape.E, gated=gated, device="cpu") if hp.quant else torch.empty(1)
    hp.backward(None, None, W, None if hp.quant or not gated else torch.empty(1), None if hp.quant else torch.empty(1), torch.empty(1),
                torch.empty(1) if gated_shared else None, torch.empty(1))


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gated_shared", [False, True])
def test_gradients_are_those_of_the_last_pass(layer, quant, S, gated, gated_shared):
    hp = layer(S, quant)
    backward(hp, not gated, not gated_shared)
    backward(hp, gated, gated_shared)
    want = ["dWg_c"] + ["dWu_c"] * gated + ["dWd_c"] + (["dWsg"] + ["dWsu"] * gated_shared + ["dWsd"] if S else [])
    assert listed(hp) == want
    assert listed(hp, gated, gated_shared) == want
    with pytest.raises(moe.MoEError, match="agree"):
        hp.gradients(not gated)
    if S:
        with pytest.raises(moe.MoEError, match="agree"):
            hp.gradients(gated, not gated_shared)


def test_before_the_first_pass(layer):
    hp = layer(1, False)
    for a in ((), (True,), (None, True)):
        with pytest.raises(moe.MoEError, match="no backward pass"):
            hp.gradients(*a)
    assert listed(hp, True, False) == ["dWg_c", "dWu_c", "dWd_c", "dWsg", "dWsd"]
    assert listed(layer(0, True), False) == ["dWg_c", "dWd_c"]
