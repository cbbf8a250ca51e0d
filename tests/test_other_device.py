"""The block-scaled calls and the clipping refuse every tensor of another GPU than the current one, whichever argument it is (no GPU needed: tensors that
say of themselves where they are, and a library that only notes that it was reached)."""
import pytest
import torch

import paper_2502_02581_amd as moe
from paper_2502_02581_amd import binding


class On(torch.Tensor):
    """A host tensor that takes itself for one of a GPU."""

    __torch_function__ = torch._C._disabled_torch_function_impl
    at = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.at))

    def get_device(self):
        return self.at


def on(t, at=0):
    t = t.as_subclass(On)
    t.at = at
    return t


class Library:
    reached = 0

    def moe_expert_plan_bytes(self, shape):   # (asked for, not a call)
        return 1 << 12

    def __getattr__(self, name):
        def call(*a):
            self.reached += 1
            return 0

        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return lib


u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
T, E, d, F = 4, 2, 128, 64
SHAPE = moe.MoEShape(T, d, E, 1, F, "bf16")


def expert_args():
    return dict(offsets=i32(E + 1), src_of=i32(T), q=u8(T, 128), s=u8(T, 1), G=bf(T, F), U=bf(T, F), H=bf(T, F), ws=u8(1 << 16))


def weights(t):
    return {n: t(x) for n, x in dict(WgT=u8(E, F, 128), WgT_s=u8(E, 1, 1), WuT=u8(E, F, 128), WuT_s=u8(E, 1, 1), WdT=u8(E, d, 128), WdT_s=u8(E, 1, 1),
                                     Wgu=u8(E, d, 256), Wgu_s=u8(E, 1, 2), Wd=u8(E, F, 128), Wd_s=u8(E, 1, 1)).items()}


def quant_weights(a):
    W = moe.MoEQuantWeights.of_codes(SHAPE, E, (a["WgT"], a["WgT_s"]), (a["WuT"], a["WuT_s"]), (a["WdT"], a["WdT_s"]))
    W.Wgu, W.Wd, W.backward = (a["Wgu"], a["Wgu_s"]), (a["Wd"], a["Wd_s"]), True
    W._seal()
    return W


def fwd(a):
    moe.moe_quant_expert_fwd(SHAPE, E, a["offsets"], T, a["src_of"], a["q"], a["s"], quant_weights(a), a["G"], a["U"], a["H"], a["Y"], a["ws"], a["plan"])


def bwd(a):
    moe.moe_quant_expert_bwd(SHAPE, E, a["offsets"], T, a["src_of"], a["row_w"], a["q"], a["s"], a["X"], quant_weights(a), a["G"], a["U"], a["H"], a["dY"],
                             a["dX"], a["ids"], a["n"], a["dWg"], a["dWu"], a["dWd"], a["ws"])


CALLS = {
    "rows": (dict(X=bf(T, d), Q=u8(T, 128), S=u8(T, 1)), lambda a: moe.moe_quant_rows(a["X"], a["Q"], a["S"])),
    "weights": (dict(W=bf(E, d, F), Q=u8(E, d, 128), S=u8(E, 1, 1), Qt=u8(E, F, 128), St=u8(E, 1, 1)),
                lambda a: moe.moe_quant_weights(a["W"], a["Q"], a["S"], a["Qt"], a["St"])),
    "gemm": (dict(offsets=i32(E + 1), A=u8(T, 128), As=u8(T, 1), B=u8(E, F, 128), Bs=u8(E, 1, 1), C=bf(T, F), ws=u8(1 << 16)),
             lambda a: moe.moe_quant_gemm(a["offsets"], d, a["A"], a["As"], a["B"], a["Bs"], a["C"], a["ws"])),
    "forward": (dict(expert_args(), Y=bf(T, d), plan=u8(1 << 16), **weights(lambda t: t)), fwd),
    "backward": (dict(expert_args(), row_w=torch.zeros(T, 1), X=bf(T, d), dY=bf(T, d), dX=bf(T, d), ids=i32(E), n=i32(1), dWg=bf(E, d, F),
                      dWu=bf(E, d, F), dWd=bf(E, F, d), **weights(lambda t: t)), bwd),
    "norm": (dict(g=bf(8), h=bf(2, 8), n=i32(1), norm=torch.zeros(1), ws=u8(1 << 15)),
             lambda a: moe.moe_grad_norm([a["g"], (a["h"], a["n"])], a["norm"], a["ws"])),
    "clip": (dict(g=bf(8), h=bf(2, 8), n=i32(1), norm=torch.zeros(1), o=bf(8), p=bf(2, 8)),
             lambda a: moe.moe_grad_clip([a["g"], (a["h"], a["n"])], a["norm"], 1.0, [a["o"], a["p"]])),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_the_current_device(lib, name):
    args, call = CALLS[name]
    call({n: on(t) for n, t in args.items()})
    assert lib.reached == 1


@pytest.mark.parametrize("name,other", [(n, a) for n in CALLS for a in CALLS[n][0]])
def test_one_tensor_of_another_device(lib, name, other):
    args, call = CALLS[name]
    with pytest.raises(moe.MoEError, match="cuda:1, the current device is cuda:0|one device"):
        call({n: on(t.clone(), int(n == other)) for n, t in args.items()})
    assert lib.reached == 0


@pytest.mark.parametrize("name", ["forward", "backward"])
def test_weights_of_another_device(lib, name):
    args, call = CALLS[name]
    with pytest.raises(moe.MoEError, match="cuda:1, the current device is cuda:0"):
        call({n: on(t.clone(), int(n.startswith(("Wg", "Wu", "Wd")))) for n, t in args.items()})
    assert lib.reached == 0


@pytest.mark.parametrize("name", ["norm", "clip"])
def test_empty_counter(lib, name):
    """A counter without a value has no address, which would mean that every slot counts."""
    args, call = CALLS[name]
    with pytest.raises(moe.MoEError, match="empty"):
        call({n: on(i32(0) if n == "n" else t) for n, t in args.items()})
    assert lib.reached == 0
