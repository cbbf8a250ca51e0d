"""What the norms, the dropout and the sequences' losses refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2502_02581_amd as moe
from paper_2502_02581_amd import binding
from paper_2502_02581_amd.binding import _CDrop, _CNorm, _CShape
from tests.test_other_device import on

OK16 = ctypes.c_void_p(4096)   # never dereferenced: every call below fails before a launch
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


def text(lib):
    return lib.moe_last_error().decode()


def drop(p=0.1, site=0, rng=4096):
    return ctypes.byref(_CDrop(p, site, rng))


def test_dropout(lib):
    def f(X=OK16, ldx=100, R=OK16, ldr=100, dt=1, n=4, cols=100, d=None, out=OK16, ldo=100):
        return lib.moe_dropout(X, ldx, R, ldr, dt, n, cols, d or drop(), out, ldo, None)

    assert f(dt=2) == -3 and "dtype" in text(lib)
    assert lib.moe_dropout(OK16, 8, None, 0, 1, 4, 8, None, OK16, 8, None) == -1 and "NULL" in text(lib)
    for p in (-0.1, 1.0, 1 - 2.0 ** -18, 7.0, float("nan"), float("inf")):
        assert f(d=drop(p)) == -1 and "probability" in text(lib), p
    assert f(d=drop(site=65536)) == -1 and "site" in text(lib)
    for rng in (None, 4100):
        assert f(d=drop(rng=rng)) == -1 and "rng" in text(lib)
    for kw in (dict(n=-1), dict(cols=0), dict(cols=(1 << 18) + 1)):
        assert f(**kw) == -1 and "bad" in text(lib)
    for kw in (dict(X=None), dict(out=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    for kw in (dict(ldx=99), dict(ldr=99), dict(ldo=99), dict(ldx=1 << 40), dict(ldx=-100)):
        assert f(**kw) == -1 and "stride" in text(lib)
    for kw in (dict(X=ODD), dict(R=ODD), dict(out=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib)
    assert f(n=0, X=None, R=None, out=None) == 0
    assert f(X=OK16, out=OK16, ldo=101) == -1 and "stride" in text(lib)
    assert f(n=1 << 30, cols=1 << 10, ldx=1 << 10, ldr=1 << 10, ldo=1 << 10) == -1 and "too many" in text(lib)


def norm(**kw):
    base = dict(n_rows=4, d=100, dtype=1, wdtype=0, kind=0, eps=1e-5)
    base.update(kw)
    return _CNorm(*[base[n] for n in ("n_rows", "d", "dtype", "wdtype", "kind", "eps")])


def test_norm_fwd(lib):
    def f(nm=None, X=OK16, ldx=100, R=OK16, ldr=100, d=None, w=OK16, b=OK16, Z=OK16, ldz=100, Y=ctypes.c_void_p(12288), ldy=100, mean=OK16, rstd=OK16):
        return lib.moe_norm_fwd(ctypes.byref(nm or norm()), X, ldx, R, ldr, d, w, b, Z, ldz, Y, ldy, mean, rstd, None)

    for kw in (dict(dtype=2), dict(wdtype=-1), dict(kind=2)):
        assert f(norm(**kw)) == -3 and "unknown" in text(lib)
    for kw in (dict(n_rows=-1), dict(n_rows=2 ** 31 - 2 ** 14, d=1), dict(d=0), dict(d=16385), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert f(norm(**kw)) == -1 and "bad" in text(lib)
        assert moe.load_library().moe_norm_bwd_workspace_bytes(ctypes.byref(norm(**kw))) == 0
    for kw in (dict(X=None), dict(Y=None), dict(Z=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    for kw in (dict(ldx=99), dict(ldr=99), dict(ldz=99), dict(ldy=99)):
        assert f(**kw) == -1 and "stride" in text(lib)
    for kw in (dict(X=ODD), dict(R=ODD), dict(Z=ODD), dict(Y=ODD), dict(w=ODD), dict(b=ODD), dict(mean=ODD), dict(rstd=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib)
    assert f(R=None) == -1 and "Z goes with" in text(lib)
    assert f(norm(kind=1)) == -1 and "no mean" in text(lib)
    assert f(d=drop(2.0)) == -1 and "probability" in text(lib)
    assert lib.moe_norm_fwd(None, OK16, 8, None, 0, None, None, None, None, 0, OK16, 8, None, None, None) == -1
    assert f(norm(n_rows=0), X=None, R=None, Z=None, Y=None) == 0
    there = ctypes.c_void_p(8192)
    assert f(Y=OK16) == -1 and "overlap" in text(lib)
    assert f(X=there, Z=there, ldz=101) == -1 and f(R=there, Z=there, ldz=101) == -1 and f(X=there, Y=there, ldy=101) == -1 and "stride" in text(lib)


def test_norm_bwd(lib):
    need = lib.moe_norm_bwd_workspace_bytes(ctypes.byref(norm()))
    assert need >= 2 * 100 * 4

    def f(nm=None, dY=OK16, lddy=100, Z=OK16, ldz=100, w=OK16, mean=OK16, rstd=OK16, dZ=OK16, lddz=100, d=None, dR=OK16, lddr=100, dX=None, lddx=0, dw=OK16,
          db=OK16, ws=OK16, nb=need):
        return lib.moe_norm_bwd(ctypes.byref(nm or norm()), dY, lddy, Z, ldz, w, mean, rstd, dZ, lddz, d, dR, lddr, dX, lddx, dw, db, ws, nb, None)

    for kw in (dict(dY=None), dict(Z=None), dict(mean=None), dict(rstd=None), dict(dR=None), dict(ws=None), dict(d=drop())):
        assert f(**kw) == -1 and "null" in text(lib), kw
    for kw in (dict(lddy=99), dict(ldz=99), dict(lddz=99), dict(lddr=99), dict(d=drop(), dX=OK16, lddx=99)):
        assert f(**kw) == -1 and "stride" in text(lib)
    for kw in (dict(dY=ODD), dict(Z=ODD), dict(dZ=ODD), dict(dR=ODD), dict(w=ODD), dict(dw=ODD), dict(db=ODD), dict(mean=ODD), dict(rstd=ODD), dict(ws=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib)
    assert f(dX=OK16, lddx=100) == -1 and "dX goes with" in text(lib)
    assert f(nb=need - 1) == -2 and "workspace" in text(lib)
    assert f(norm(dtype=9)) == -3
    assert f(d=drop(), dX=OK16, lddx=100) == -1 and "overlap" in text(lib)
    there = ctypes.c_void_p(8192)
    for kw in (dict(dY=there), dict(dZ=there), dict(Z=there)):
        assert f(dR=there, lddr=101, **kw) == -1 and "stride" in text(lib)
        assert f(d=drop(), dX=there, lddx=101, **kw) == -1 and "stride" in text(lib)
    assert f(norm(n_rows=0), dY=None, Z=None, mean=None, rstd=None, dZ=None, dR=None, dw=None, db=None, ws=None, nb=0) == 0


def shape(**kw):
    base = dict(T=16, d=64, E=8, k=2, d_ff=64, dtype=1, gate=0, renorm=1)
    base.update(kw)
    return _CShape(*[base[n] for n in ("T", "d", "E", "k", "d_ff", "dtype", "gate", "renorm")])


def test_seq_loss(lib):
    need = lib.moe_seq_loss_workspace_bytes(ctypes.byref(shape()), 3)
    assert need > 0 and lib.moe_seq_loss_workspace_bytes(ctypes.byref(shape()), 0) == 0 and lib.moe_seq_loss_workspace_bytes(ctypes.byref(shape(E=2000)), 1) == 0

    def f(s=None, lg=OK16, tk=OK16, n=3, st=OK16, ln=OK16, counts=OK16, P=OK16, loss=OK16, coef=OK16, ws=OK16, nb=need):
        return lib.moe_seq_loss(ctypes.byref(s or shape()), lg, tk, n, st, ln, 0.1, 0.1, counts, P, loss, coef, ws, nb, None)

    def g(s=None, lg=OK16, n=3, st=OK16, ln=OK16, counts=OK16, coef=OK16, dl=OK16):
        return lib.moe_seq_loss_bwd(ctypes.byref(s or shape()), lg, n, st, ln, counts, coef, 1.0, 0, dl, None)

    for call in (f, g):
        assert call(shape(gate=3)) == -3 and call(shape(k=9)) == -1 and call(shape(T=-1)) == -1
        for kw in (dict(n=0), dict(n=-1), dict(n=(1 << 24) + 1), dict(st=None), dict(st=None, ln=None), dict(n=1, st=None)):
            assert call(**kw) == -1 and "sequences" in text(lib), kw
        assert call(shape(T=2 ** 31 - 5, k=1, E=1)) == -1 and "index range" in text(lib)
    for kw in (dict(lg=None), dict(tk=None), dict(counts=None), dict(P=None), dict(loss=None), dict(coef=None), dict(ws=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    for kw in (dict(lg=None), dict(counts=None), dict(coef=None), dict(dl=None)):
        assert g(**kw) == -1 and "null" in text(lib)
    assert f(ws=ctypes.c_void_p(4104)) == -1 and "aligned" in text(lib)
    for kw in (dict(lg=ODD), dict(tk=ODD), dict(counts=ODD), dict(P=ODD), dict(loss=ODD), dict(coef=ODD), dict(st=ODD), dict(ln=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib), kw
    for kw in (dict(lg=ODD), dict(counts=ODD), dict(coef=ODD), dict(dl=ODD), dict(st=ODD), dict(ln=ODD)):
        assert g(**kw) == -1 and "aligned" in text(lib), kw
    assert f(nb=need - 1) == -2 and "workspace" in text(lib)
    assert g(shape(T=0), lg=None, counts=None, coef=None, dl=None) == 0


# ---- the binding: tensors that say of themselves where they are, and a library that only notes that it was reached
class Library:
    reached = 0

    def __getattr__(self, name):
        def call(*a):
            self.reached += 1
            return 0

        return call


@pytest.fixture
def noted(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_current", lambda stream: (0, 0))
    return lib


bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
f32 = lambda *s: torch.zeros(*s)  # noqa: E731
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
N, D, T, E, S = 4, 24, 6, 8, 3
NORM = moe.MoENorm(N, D, "layer", 1e-5, "bf16", "f32")
SHAPE = moe.MoEShape(T, 64, E, 2, 64)
ROWS = lambda *names: {n: bf(N, D) for n in names}  # noqa: E731
CALLS = {
    "dropout": (dict(ROWS("X", "R", "out"), rng=torch.zeros(2, dtype=torch.int64)),
                lambda a: moe.moe_dropout(a["X"], moe.MoEDropout(0.1, a["rng"]), a["out"], R=a["R"])),
    "norm_fwd": (dict(ROWS("X", "R", "Z", "Y"), w=f32(D), b=f32(D), mean=f32(N), rstd=f32(N), rng=torch.zeros(2, dtype=torch.int64)),
                 lambda a: moe.moe_norm_fwd(NORM, a["X"], a["w"], a["b"], a["Y"], a["mean"], a["rstd"], R=a["R"], drop=moe.MoEDropout(0.1, a["rng"]), Z=a["Z"])),
    "norm_bwd": (dict(ROWS("dY", "Z", "dZ", "dR", "dX"), w=f32(D), mean=f32(N), rstd=f32(N), dw=f32(D), db=f32(D), ws=f32(100),
                      rng=torch.zeros(2, dtype=torch.int64)),
                 lambda a: moe.moe_norm_bwd(NORM, a["dY"], a["Z"], a["w"], a["mean"], a["rstd"], a["dR"], a["dw"], a["db"], a["ws"], dZ=a["dZ"],
                                            drop=moe.MoEDropout(0.1, a["rng"]), dX=a["dX"])),
    "seq_loss": (dict(logits=f32(T, E), topk=i32(T, 2), start=i32(S), length=i32(S), counts=i32(S, E), P=f32(S, E), loss=f32(2), coef=f32(S + 1), ws=f32(100)),
                 lambda a: moe.moe_seq_loss(SHAPE, a["logits"], a["topk"], a["start"], a["length"], 0.1, 0.1, a["counts"], a["P"], a["loss"], a["coef"], a["ws"])),
    "seq_loss_bwd": (dict(logits=f32(T, E), start=i32(S), length=i32(S), counts=i32(S, E), coef=f32(S + 1), dlogits=f32(T, E)),
                     lambda a: moe.moe_seq_loss_bwd(SHAPE, a["logits"], a["start"], a["length"], a["counts"], a["coef"], 1.0, False, a["dlogits"])),
}


@pytest.mark.parametrize("name", CALLS)
def test_accepted(noted, name):
    args, call = CALLS[name]
    call({n: on(t.clone()) for n, t in args.items()})
    assert noted.reached == 1


@pytest.mark.parametrize("name,other", [(n, a) for n in CALLS for a in CALLS[n][0]])
def test_one_tensor_is_wrong(noted, name, other):
    """On another device, on none, of another type, one value short, with a hole between its values."""
    args, call = CALLS[name]
    t = args[other]
    wrong = [on(t.clone(), 1), t.clone(), on(t.to(torch.float16))]
    if other != "ws":
        wrong.append(on(t[..., :-1].clone()))
        wrong.append(on(torch.zeros(*t.shape, 2, dtype=t.dtype)[..., 0]))
    else:
        wrong.pop()   # (of any type)
    for x in wrong:
        with pytest.raises(moe.MoEError):
            call({n: x if n == other else on(v.clone()) for n, v in args.items()})
    assert noted.reached == 0


def test_rows_with_strides(noted):
    """Rows may be pieces of longer ones; they may not overlap or run across."""
    args, call = CALLS["norm_fwd"]
    a = {n: on(t.clone()) for n, t in args.items()}
    call(dict(a, X=on(torch.zeros(N, D + 5, dtype=torch.bfloat16)[:, 2:2 + D])))
    assert noted.reached == 1
    for x in (torch.zeros(D, dtype=torch.bfloat16).expand(N, D), torch.zeros(D, N, dtype=torch.bfloat16).t()):
        with pytest.raises(moe.MoEError, match="adjacent"):
            call(dict(a, X=on(x)))
    assert noted.reached == 1


def test_objects():
    for kw in (dict(kind="batch"), dict(dtype="f16"), dict(wdtype="int8")):
        with pytest.raises(moe.MoEError, match="none of"):
            moe.MoENorm(4, 8, **kw)
    for site in (-1, 65536):
        with pytest.raises(moe.MoEError, match="site"):
            moe.MoEDropout(0.1, None, site)
    with pytest.raises(moe.MoEError, match="shape"):
        moe.MoEDropout(0.1, on(torch.zeros(3, dtype=torch.int64)))
    with pytest.raises(moe.MoEError):
        moe.MoEDropout(0.1, torch.zeros(2, dtype=torch.int64))
    a, b = moe.MoENorm(4, 8), moe.MoENorm(4, 8)
    assert a == b and a.c.n_rows == 4 and a.weight_dtype is torch.bfloat16
