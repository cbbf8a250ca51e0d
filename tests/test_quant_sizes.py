"""The block-scaled expert calls of the binding refuse tensors of fewer values than they read or write (no GPU needed: see test_other_device.py)."""
import pytest
import torch

import paper_2502_02581_amd as moe

from .test_other_device import CALLS, SHAPE, E, T, lib, on, u8  # noqa: F401

NAMES = {"forward": ("offsets", "src_of", "q", "s", "G", "U", "H", "Y", "plan"),
         "backward": ("offsets", "src_of", "q", "s", "row_w", "X", "G", "U", "H", "dY", "dX", "ids", "n", "dWg", "dWu", "dWd")}


@pytest.mark.parametrize("name,short", [(n, a) for n in NAMES for a in NAMES[n]])
def test_one_value_short(lib, name, short):  # noqa: F811
    args, call = CALLS[name]
    if short == "plan":
        args = dict(args, plan=u8(1 << 12))
    call({n: on(t) for n, t in args.items()})
    assert lib.reached == 1
    # (slots of weight gradients: as many as there are groups or rows, whichever are fewer)
    with pytest.raises(moe.MoEError, match="values, the call takes|must have shape"):
        call({n: on(t.reshape(-1)[:t.numel() - 1] if n == short else t) for n, t in args.items()})
    assert lib.reached == 1


def test_slots_of_fewer_rows_than_groups(lib):  # noqa: F811
    """Two rows cannot activate more than two of five groups."""
    shape = moe.MoEShape(2, 128, 5, 1, 64, "bf16")
    bf = lambda *s: on(torch.zeros(*s, dtype=torch.bfloat16))
    i32 = lambda n: on(torch.zeros(n, dtype=torch.int32))
    b = lambda *s: on(u8(*s))
    W = moe.MoEQuantWeights.of_codes(shape, 5, (b(5, 64, 128), b(5, 1, 1)), None, (b(5, 128, 128), b(5, 1, 1)))
    W.Wgu, W.Wd = (b(5, 128, 128), b(5, 1, 1)), (b(5, 64, 128), b(5, 1, 1))
    W._seal()
    run = lambda slots: moe.moe_quant_expert_bwd(shape, 5, i32(6), 2, None, None, b(2, 128), b(2, 1), bf(2, 128), W, bf(2, 64), None, bf(2, 64), bf(2, 128),
                                                 bf(2, 128), i32(5), i32(1), bf(slots, 128, 64), None, bf(slots, 64, 128), b(1 << 16))
    run(2)
    assert lib.reached == 1
    with pytest.raises(moe.MoEError, match="dWg_c has"):
        run(1)
