"""What the block-scaled calls and the clipping refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2502_02581_amd as moe
from paper_2502_02581_amd.binding import _CGrad, _CQuantWeights, _CShape

OK16 = ctypes.c_void_p(4096)   # never dereferenced: every call below fails before a launch
ODD = ctypes.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


def text(lib):
    return lib.moe_last_error().decode()


def test_sizes(lib):
    assert [moe.moe_quant_row_bytes(n) for n in (1, 127, 128, 129, 1000)] == [128, 128, 128, 256, 1024]
    assert [moe.moe_quant_scale_bytes(n) for n in (1, 127, 128, 129, 1000)] == [1, 1, 1, 2, 8]
    for n in list(range(1, 300)) + [4096, 4097, 1 << 22]:   # the binding's arithmetic is the library's
        assert (moe.moe_quant_row_bytes(n), moe.moe_quant_scale_bytes(n)) == (lib.moe_quant_row_bytes(n), lib.moe_quant_scale_bytes(n))
    assert ctypes.sizeof(_CGrad) == 48   # whole 64-bit words, as the binding packs them
    assert lib.moe_quant_row_bytes(0) == 0 and lib.moe_quant_scale_bytes(-3) == 0
    assert moe.moe_quant_gemm_workspace_bytes(0, 10, 8, 8) == 0 and moe.moe_quant_gemm_workspace_bytes(4, 10, 128, 128) > 0


def test_rows(lib):
    f = lambda X=OK16, dt=1, n=4, cols=100, ld=100, Q=OK16, S=OK16: lib.moe_quant_rows(X, dt, n, cols, ld, Q, S, None)
    assert f(dt=2) == -3 and "dtype" in text(lib)
    for kw in (dict(n=-1), dict(cols=0), dict(ld=99), dict(n=1 << 30, cols=1 << 20, ld=1 << 20)):
        assert f(**kw) == -1 and "bad" in text(lib)
    for kw in (dict(X=None), dict(Q=None), dict(S=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    assert f(Q=ODD) == -1 and f(X=ctypes.c_void_p(4097)) == -1 and "aligned" in text(lib)
    assert f(X=None, n=0, Q=None, S=None) == 0


def test_weights(lib):
    def f(W=OK16, dt=1, g=2, K=64, N=72, Q=OK16, ldq=128, S=OK16, lds=1, Qt=OK16, ldqt=128, St=OK16, ldst=1):
        return lib.moe_quant_weights(W, dt, g, K, N, Q, ldq, S, lds, Qt, ldqt, St, ldst, None)

    assert f(dt=9) == -3
    for kw in (dict(g=0), dict(g=2000), dict(K=60), dict(N=0), dict(N=73)):
        assert f(**kw) == -1 and "bad" in text(lib)
    for kw in (dict(W=None), dict(S=None), dict(Qt=None), dict(Q=None, S=None, Qt=None, St=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    for kw in (dict(ldq=120), dict(ldq=136), dict(lds=0), dict(ldqt=64), dict(ldst=0)):
        assert f(**kw) == -1 and "rows of" in text(lib)
    for kw in (dict(W=ODD), dict(Q=ODD), dict(Qt=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib)


def test_gemm(lib):
    need = moe.moe_quant_gemm_workspace_bytes(3, 50, 96, 64)

    def f(g=3, off=OK16, n=50, K=96, N=64, A=OK16, As=OK16, B=OK16, Bs=OK16, C=OK16, ws=OK16, nb=need):
        return lib.moe_quant_gemm(g, off, n, K, N, A, As, B, Bs, C, ws, nb, None)

    for kw in (dict(g=0), dict(g=1025), dict(n=-1), dict(K=0), dict(N=60), dict(N=0), dict(off=None), dict(K=1 << 25), dict(N=1 << 25)):
        assert f(**kw) == -1 and "bad" in text(lib)
    for kw in (dict(A=None), dict(As=None), dict(B=None), dict(Bs=None), dict(C=None), dict(ws=None)):
        assert f(**kw) == -1 and "null" in text(lib)
    for kw in (dict(A=ODD), dict(B=ODD), dict(C=ODD), dict(ws=ODD)):
        assert f(**kw) == -1 and "aligned" in text(lib)
    assert f(nb=need - 1) == -2 and "workspace" in text(lib)
    assert f(n=0, A=None, As=None, C=None) == 0


def shape(**kw):
    base = dict(T=16, d=64, E=8, k=2, d_ff=72, dtype=1, gate=0, renorm=1)
    base.update(kw)
    return _CShape(*[base[n] for n in ("T", "d", "E", "k", "d_ff", "dtype", "gate", "renorm")])


def weights(gated=1, **kw):
    return _CQuantWeights(**{**{n: 4096 for n, _ in _CQuantWeights._fields_}, "gated": gated, **kw})


def fwd(lib, s=None, g=8, off=OK16, n=32, src=None, XQ=OK16, XS=OK16, W=None, G=OK16, U=OK16, H=OK16, Y=OK16, plan=None, ws=OK16, nb=None):
    s = s or shape()
    nb = lib.moe_quant_expert_fwd_workspace_bytes(ctypes.byref(s), g, n) if nb is None else nb
    return lib.moe_quant_expert_fwd(ctypes.byref(s), g, off, n, src, XQ, XS, ctypes.byref(W or weights()), G, U, H, Y, plan, ws, nb, None)


def test_expert_fwd(lib):
    assert fwd(lib, shape(dtype=0)) == -3 and "bf16" in text(lib)
    assert fwd(lib, shape(d=60)) == -1 and fwd(lib, g=0, nb=1 << 20) == -1 and fwd(lib, n=-1, nb=1 << 20) == -1
    assert fwd(lib, shape(d_ff=1 << 24), nb=1 << 40) == -1 and "too long" in text(lib)
    for kw in (dict(off=None), dict(XQ=None), dict(XS=None), dict(Y=None), dict(ws=None), dict(H=None), dict(U=None), dict(G=None)):
        assert fwd(lib, **kw) == -1 and "null" in text(lib), kw
    for n in ("WgT", "WgT_s", "WuT", "WuT_s", "WdT", "WdT_s"):
        assert fwd(lib, W=weights(**{n: None})) == -1 and "null" in text(lib), n
    assert fwd(lib, W=weights(WdT=4100)) == -1 and "aligned" in text(lib)
    for kw in (dict(XQ=ODD), dict(G=ODD), dict(U=ODD), dict(H=ODD), dict(Y=ODD), dict(plan=ODD), dict(ws=ODD)):
        assert fwd(lib, **kw) == -1 and "aligned" in text(lib), kw
    assert fwd(lib, src=OK16, n=31) == -1 and "T*k" in text(lib)
    assert fwd(lib, shape(T=1 << 23, d=512, k=1), src=OK16, n=1 << 23) == -1 and "4 GiB" in text(lib)
    assert fwd(lib, plan=OK16, n=31) == -1 and fwd(lib, plan=OK16, g=7) == -1 and "plan" in text(lib)
    assert fwd(lib, nb=16) == -2 and "workspace" in text(lib)
    assert fwd(lib, n=0, XQ=None, XS=None, G=None, U=None, H=None, Y=None) == 0


def bwd(lib, s=None, g=8, off=OK16, n=32, src=OK16, rw=OK16, dYQ=OK16, dYS=OK16, X=OK16, W=None, G=OK16, U=OK16, H=OK16, dY=OK16, dX=OK16, ids=OK16,
        na=OK16, dWg=OK16, dWu=OK16, dWd=OK16, ws=OK16, nb=None):
    s = s or shape()
    nb = lib.moe_quant_expert_bwd_workspace_bytes(ctypes.byref(s), g, n) if nb is None else nb
    return lib.moe_quant_expert_bwd(ctypes.byref(s), g, off, n, src, rw, dYQ, dYS, X, ctypes.byref(W or weights()), G, U, H, dY, dX, ids, na, dWg,
                                    dWu, dWd, ws, nb, None)


def test_expert_bwd(lib):
    for kw in (dict(off=None), dict(src=None), dict(rw=None), dict(dYQ=None), dict(dYS=None), dict(X=None), dict(G=None), dict(U=None), dict(H=None),
               dict(dY=None), dict(dX=None), dict(ids=None), dict(na=None), dict(dWg=None), dict(dWu=None), dict(dWd=None), dict(ws=None)):
        assert bwd(lib, **kw) == -1 and "null" in text(lib), kw
    for n in ("Wgu", "Wgu_s", "Wd", "Wd_s"):
        assert bwd(lib, W=weights(**{n: None})) == -1 and "null" in text(lib), n
    for kw in (dict(dYQ=ODD), dict(X=ODD), dict(G=ODD), dict(dX=ODD), dict(dWg=ODD), dict(dWu=ODD), dict(dWd=ODD), dict(ws=ODD)):
        assert bwd(lib, **kw) == -1 and "aligned" in text(lib), kw
    assert bwd(lib, nb=16) == -2 and bwd(lib, shape(dtype=0)) == -3


def test_grads(lib):
    def g(**kw):
        return (_CGrad * 1)(_CGrad(**{**dict(g=4096, out=8192, n=10, n_active=None, slot=0, dtype=1), **kw}))

    norm = lambda l, n=1, out=OK16, ws=OK16, nb=1 << 20: lib.moe_grad_norm(l, n, out, ws, nb, None)
    clip = lambda l, n=1, out=OK16, m=1.0: lib.moe_grad_clip(l, n, out, m, None)
    assert norm(g(dtype=5)) == -3 and clip(g(dtype=5)) == -3
    for l in (g(g=None), g(n=-1), g(n_active=4096, slot=0), g(n=1 << 41)):
        assert norm(l) == -1 and clip(l) == -1 and "gradient 0" in text(lib)
    assert clip(g(out=None)) == -1 and norm(g(g=4104)) == -1 and clip(g(out=8200)) == -1 and "aligned" in text(lib)
    assert norm(g(), n=-1) == -1 and norm(None, n=1) == -1
    assert norm(g(), out=None) == -1 and norm(g(), ws=None) == -1 and norm(g(), nb=8) == -2
    assert clip(g(), out=None) == -1 and clip(g(), m=-1.0) == -1 and clip(g(), m=float("nan")) == -1
    assert clip(g(n=0, g=None, out=None)) == 0 and clip(g(), n=0) == 0
