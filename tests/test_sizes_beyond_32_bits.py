"""Sizes that the library's 32-bit arguments do not hold are refused, not cut off (no GPU needed: tensors without memory, and a library that only notes that it was reached)."""
import numpy as np
import pytest
import torch

import paper_2502_02581_amd as moe
from paper_2502_02581_amd import binding
from tests.test_other_device import Library, on

BIG = (1 << 32) + 5
SHAPE = moe.MoEShape(8, 128, 4, 2, 64)


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    monkeypatch.setattr(binding, "_current", lambda s: (0, 0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return lib


def t(*shape, dtype=torch.bfloat16):
    return on(torch.empty(*shape, dtype=dtype, device="meta"))


u8, i32, f32 = torch.uint8, torch.int32, torch.float32
DROP = lambda: moe.MoEDropout(0.0, None)  # noqa: E731
CALLS = {
    "shape": lambda: moe.MoEShape(BIG, 128, 4, 2, 64),
    "shape d": lambda: moe.MoEShape(8, 1 << 31, 4, 2, 64),
    "shape below": lambda: moe.MoEShape(8, 128, 4 - (1 << 32), 2, 64),
    "norm": lambda: moe.MoENorm(BIG, 64),
    "norm d": lambda: moe.MoENorm(4, BIG),
    "dropout rows": lambda: moe.moe_dropout(t(BIG, 1), DROP(), t(BIG, 1)),
    "dropout columns": lambda: moe.moe_dropout(t(1, BIG + 59), DROP(), t(1, BIG + 59)),
    "sequences": lambda: moe.moe_seq_loss(SHAPE, t(8, 4, dtype=f32), t(8, 2, dtype=i32), t(BIG, dtype=i32), t(BIG, dtype=i32), 0.1, 0.1, t(BIG, 4, dtype=i32),
                                          t(BIG, 4, dtype=f32), t(2, dtype=f32), t(BIG + 1, dtype=f32), t(1 << 20, dtype=u8)),
    "sequences backward": lambda: moe.moe_seq_loss_bwd(SHAPE, t(8, 4, dtype=f32), t(BIG, dtype=i32), t(BIG, dtype=i32), t(BIG, 4, dtype=i32), t(BIG + 1, dtype=f32), 1.0,
                                                       False, t(8, 4, dtype=f32)),
    "sequences workspace": lambda: moe.moe_seq_loss_workspace_bytes(SHAPE, BIG),
    "quant rows": lambda: moe.moe_quant_rows(t(BIG, 64), t(BIG, 128, dtype=u8), t(BIG, 1, dtype=u8)),
    "quant columns": lambda: moe.moe_quant_rows(t(1, BIG), t(1, BIG + 123, dtype=u8), t(1, (BIG + 123) // 128, dtype=u8)),
    "quant weights": lambda: moe.moe_quant_weights(t(1, BIG, 8), None, None, None, None),
    "quant product": lambda: moe.moe_quant_gemm(None, 64, t(BIG, 128, dtype=u8), t(BIG, 1, dtype=u8), t(1, 64, 128, dtype=u8), t(1, 1, 1, dtype=u8), t(BIG, 64), t(1, dtype=u8)),
    "quant product workspace": lambda: moe.moe_quant_gemm_workspace_bytes(1, BIG, 64, 64),
    "quant experts workspace": lambda: moe.moe_quant_expert_fwd_workspace_bytes(SHAPE, 4, BIG) + moe.moe_quant_expert_bwd_workspace_bytes(SHAPE, 4, BIG),
    "experts": lambda: moe.moe_expert_fwd(SHAPE, 4, t(5, dtype=i32), BIG, *[None] * 7, None, t(1, dtype=u8)),
    "experts backward": lambda: moe.moe_expert_bwd(SHAPE, 4, t(5, dtype=i32), BIG, *[None] * 14, t(1, dtype=u8)),
    "experts workspace": lambda: moe.moe_expert_fwd_workspace_bytes(SHAPE, BIG, 16, False),
    "experts workspace backward": lambda: moe.moe_expert_bwd_workspace_bytes(SHAPE, 4, BIG, False),
    "expert sets": lambda: moe.moe_experts_fwd(SHAPE, dict(d_ff=64, n_groups=4, n_rows=BIG, ws=None, ws_bytes=0), None),
    "load": lambda: moe.moe_plan_predict_load(np.zeros((3, 4)), BIG),
    "materialize": lambda: moe.moe_plan_materialize(np.zeros((4, 2)), np.zeros(4), BIG, 1, 1),
    "dispatch plan": lambda: moe.moe_plan_dispatch(np.zeros((4, 2)), np.zeros((4, 2)), BIG),
}


@pytest.mark.parametrize("name", CALLS)
def test_refused(lib, name):
    with pytest.raises(moe.MoEError, match="beyond 32 bits"):
        CALLS[name]()
    assert lib.reached == 0


def test_what_fits_is_taken(lib):
    """The largest values of 32 bits reach the library, whose own checks refuse or take them."""
    top = (1 << 31) - 1
    assert moe.MoEShape(top, 128, 4, 2, 64).c().T == top and moe.MoENorm(top, 64).c.n_rows == top
    moe.moe_dropout(t(top, 1), DROP(), t(top, 1))
    assert lib.reached == 1
