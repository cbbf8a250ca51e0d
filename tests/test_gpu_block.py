"""The whole pre-norm block through MoEHotPath against the 64-bit definitions chained by hand: norm, router, experts, dropout, residual stream, the sequences' losses, and
every gradient; on other streams, in graphs whose step advances, beside a plain layer.

Tolerances are the layer tests' own, relative to each tensor's largest value: 1e-4 in fp32 (a chain of four products; each operator here adds 1e-5 at most), 3e-2 in bf16 (2e-2 for the
layer; the normed rows, the router's gradient and the output are rounded once more each, 2^-8)."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import block_oracle as ob
from oracle import moe_oracle as orc
from tests.helpers import np64, scale_rel_err

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


class Block:
    def __init__(self, T=70, d=64, E=6, k=2, d_ff=48, dtype="f32", kind="layer", p=0.2, residual=True, gate="softmax", seqs=None, seq_alpha=0.02, z_beta=0.01, aux=0.0,
                 n_shared=1, bias=True, seed=0, **kw):
        import paper_2502_02581_amd as moe

        self.moe, self.p, self.kind, self.seqs = moe, p, kind, seqs
        self.k, self.E, self.gate, self.aux = k, E, gate, aux
        self.alpha, self.beta = seq_alpha, z_beta
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        g = torch.Generator().manual_seed(seed + 5)
        r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dt).to(DEV)  # noqa: E731
        self.X, self.R = r(T, d), r(T, d) if residual else None
        self.dOut = r(T, d)
        self.w = moe.MoEBlockWeights((1 + 0.2 * torch.randn(d, generator=g)).to(dt).to(DEV), r(d, std=0.1) if bias else None, r(d, E, std=2 * d ** -0.5))
        self.W = [r(E, d, d_ff, std=d ** -0.5), r(E, d, d_ff, std=d ** -0.5), r(E, d_ff, d, std=d_ff ** -0.5)]
        self.Ws = [r(n_shared, d, 24, std=d ** -0.5), r(n_shared, d, 24, std=d ** -0.5), r(n_shared, 24, d, std=24 ** -0.5)] if n_shared else [None] * 3
        self.rng = torch.tensor([99, 7], dtype=torch.int64, device=DEV)
        self.shape = moe.MoEShape(T, d, E, k, d_ff, dtype, gate)
        n_seqs = len(seqs[1]) if seqs else 1
        self.hp = moe.MoEHotPath(self.shape, n_shared, 24 if n_shared else 0, DEV, aux_alpha=aux, norm=kind, eps=EPS, dropout=p, rng=self.rng if p else None, site=4,
                                 seq_alpha=seq_alpha, z_beta=z_beta, n_seqs=n_seqs, **kw)
        self.dev_seqs = tuple(torch.tensor(s, dtype=torch.int32, device=DEV) for s in seqs) if seqs else None

    def forward(self, **kw):
        return self.hp.forward(self.w, self.X, *self.W, *self.Ws, residual=self.R, seqs=self.dev_seqs, **kw)

    def backward(self, **kw):
        return self.hp.backward(self.dOut, self.X, *self.W, *self.Ws, **kw)

    def reference(self, step=7):
        """Every result by name, from the rounded inputs."""
        b, T, d = self.hp.b, self.shape.T, self.shape.d
        x, dout = np64(self.X), np64(self.dOut)
        keep = [ob.keep(T, d, self.p, 99, step, 4 + i) if self.p else np.ones((T, d), bool) for i in (0, 1)]
        o = {}
        added = self.R is not None
        z = ob.dropout(x, keep[0], self.p, np64(self.R)) if added else x
        o["Z"] = z
        if added:
            z = np64(b["Z"])
        w, bias, Wr = np64(self.w.norm_w), np64(self.w.norm_b) if self.w.norm_b is not None else None, np64(self.w.Wr)
        xn, _, rstd, h = ob.norm_fwd(z, w, bias, self.kind, EPS)
        o["Xn"] = xn
        xr = np64(b["Xn"])
        o["logits"] = xr @ Wr
        logits = b["logits"].cpu().numpy()   # (which experts are chosen goes by the fp32 logits)
        m = [np64(t) if t is not None else None for t in (*self.W, *self.Ws)]
        dy = ob.dropout(dout, keep[1], self.p)
        if self.p:
            o["dYd"] = dy
            dy = np64(b["dYd"])
        lay = orc.layer_fwd_bwd(logits, xr, dy, *m[:3], self.k, self.gate, True, *m[3:], want_dlogits=True, aux_alpha=self.aux)
        o["Out"] = ob.dropout(np64(b["Y"]), keep[1], self.p, z)
        o["Y"] = lay["Y"]
        ranges = [(0, T)] if not self.seqs else [(a, a + n) for a, n in zip(*self.seqs)]
        counts, P, loss, ds = ob.seq_loss(logits.astype(np.float64), lay["topk_idx"], ranges, self.k, self.gate, self.alpha, self.beta)
        o.update(seq_P=P, seq_loss=loss)
        o["dlogits"] = lay["dlogits"] + ds
        dl = np64(b["dlogits"])
        if self.shape.dtype == "bf16":
            dl = np64(torch.from_numpy(dl).to(torch.bfloat16))
        o["dWr"], o["dX"] = xr.T @ dl, lay["dX"] + dl @ Wr.T
        dz, o["dnorm_w"], dbias = ob.norm_bwd(np64(b["dX"]), h, rstd, w, self.kind)
        if bias is not None:
            o["dnorm_b"] = dbias
        o["dZ"] = dz + dout
        if added and self.p:
            o["dBranch"] = ob.dropout(o["dZ"], keep[0], self.p)
        return o, counts

    def check(self, step=7):
        torch.cuda.synchronize()
        o, counts = self.reference(step)
        tol = 1e-4 if self.shape.dtype == "f32" else 3e-2
        for n, want in o.items():
            if n == "Z" and self.R is None:
                continue
            assert scale_rel_err(self.hp.b[n], want) <= tol, n
        assert np.array_equal(self.hp.b["seq_counts"].cpu().numpy(), counts)

    def outputs(self):
        names = ("Out", "dZ", "dWr", "dnorm_w", "dnorm_b", "dlogits", "seq_loss", "seq_counts", "seq_P", "dX")
        return {n: self.hp.b[n].clone() for n in names + (("dBranch",) if self.p and self.R is not None else ())}


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("p,residual", [(0.0, False), (0.0, True), (0.2, False), (0.2, True)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block(dtype, p, residual, kind):
    B = Block(dtype=dtype, p=p, residual=residual, kind=kind, bias=kind == "layer")
    assert B.forward() is B.hp.b["Out"] and B.backward() is B.hp.b["dZ"]
    B.check()


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kw", [dict(aux=0.05), dict(fused=False, aux=0.05), dict(gather=True), dict(n_shared=0), dict(overlap_shared=True), dict(T=1), dict(T=3, d=8, d_ff=8)])
def test_forms(gate, kw):
    B = Block(gate=gate, **kw)
    B.forward()
    B.backward()
    B.check()


def test_padded_batch():
    """Padding rows: part of the experts' work, not of the sequences' losses."""
    B = Block(T=96, seqs=([0, 32, 64], [20, 32, 0]), gate="sigmoid")
    B.forward()
    B.backward()
    B.check()
    assert B.hp.b["seq_counts"].sum(1).tolist() == [40, 64, 0]


def test_the_block_is_its_public_calls():
    """Bit for bit: the calls one by one, around a plain layer on the same logits and rows."""
    B = Block(T=120, dtype="bf16", aux=0.01)
    moe, b, s = B.moe, B.hp.b, B.shape
    B.forward()
    B.backward()
    plain = moe.MoEHotPath(s, 1, 24, DEV, aux_alpha=0.01)
    Z, Xn, mean, rstd = torch.empty_like(B.X), torch.empty_like(B.X), torch.empty(120, device=DEV), torch.empty(120, device=DEV)
    norm, d0, d1 = moe.MoENorm(120, s.d, "layer", EPS), moe.MoEDropout(0.2, B.rng, 4), moe.MoEDropout(0.2, B.rng, 5)
    moe.moe_norm_fwd(norm, B.X, B.w.norm_w, B.w.norm_b, Xn, mean, rstd, R=B.R, drop=d0, Z=Z)
    logits = torch.empty(120, s.E, device=DEV)
    moe.moe_router_fwd(s, Xn, B.w.Wr, logits, B.hp.ws)
    plain.forward(logits, Xn, *B.W, *B.Ws)
    out, dY = torch.empty_like(Z), torch.empty_like(Z)
    moe.moe_dropout(plain.b["Y"], d1, out, R=Z)
    assert torch.equal(out, b["Out"]) and torch.equal(plain.b["Y"], b["Y"])
    moe.moe_dropout(B.dOut, d1, dY)
    plain.backward(dY, Xn, *B.W, *B.Ws)
    f = dict(device=DEV)
    counts, P, loss, coef = torch.empty(1, s.E, dtype=torch.int32, **f), torch.empty(1, s.E, **f), torch.empty(2, **f), torch.empty(2, **f)
    moe.moe_seq_loss(s, logits, plain.b["topk_idx"], None, None, 0.02, 0.01, counts, P, loss, coef, B.hp.ws)
    moe.moe_seq_loss_bwd(s, logits, None, None, counts, coef, 1.0, True, plain.b["dlogits"])
    dWr = torch.empty_like(B.w.Wr)
    moe.moe_router_bwd(s, Xn, B.w.Wr, plain.b["dlogits"], dWr, plain.b["dX"], True, B.hp.ws)
    dR, dX, dw, db = torch.empty_like(Z), torch.empty_like(Z), torch.empty_like(B.w.norm_w), torch.empty_like(B.w.norm_b)
    moe.moe_norm_bwd(norm, plain.b["dX"], Z, B.w.norm_w, mean, rstd, dR, dw, db, B.hp.ws, dZ=B.dOut, drop=d0, dX=dX)
    for n, t in dict(dZ=dR, dBranch=dX, dnorm_w=dw, dnorm_b=db, dWr=dWr, dlogits=plain.b["dlogits"], seq_loss=loss).items():
        assert torch.equal(t, b[n]), n


def test_quant_block():
    """A block whose experts run on block-scaled operands: the calls around them are the same ones."""
    import paper_2502_02581_amd as moe

    B = Block(T=100, d=256, d_ff=136, dtype="bf16", n_shared=0, quant=True)
    W = moe.MoEQuantWeights(B.shape, B.E)
    W.update(*B.W)
    full, B.W = B.W, [W, None, None]
    B.forward()
    B.backward()
    b = B.hp.b
    plain = moe.MoEHotPath(B.shape, 0, 0, DEV, quant=True)
    plain.forward(b["logits"], b["Xn"], W)
    plain.backward(b["dYd"], b["Xn"], W)
    assert torch.equal(plain.b["Y"], b["Y"])
    assert all(torch.equal(plain.b[n][:int(b["n_active"])], b[n][:int(b["n_active"])]) for n in ("dWg_c", "dWd_c"))
    assert scale_rel_err(b["Out"], ob.dropout(np64(b["Y"]), ob.keep(100, 256, 0.2, 99, 7, 5), 0.2, np64(b["Z"]))) <= 2.0 ** -8
    assert full[0].isfinite().all()


def test_sequence_losses_of_a_plain_layer():
    """Without norm: logits as ever, the sequences' losses beside the batch's; the layer's other results keep their bits."""
    import paper_2502_02581_amd as moe

    cfg = wl.scaled(wl.CONFIGS["tiny"], T=90)
    p = {"logits": wl.make_logits(cfg), "X": wl.make_tokens(cfg, 1.0), "dY": wl.make_grad_out(cfg, 1.0)}
    p.update(wl.make_weights(cfg, "cpu", 0.1))
    g = {k: v.to(DEV) for k, v in p.items()}
    shape = moe.MoEShape(90, cfg.d, cfg.E, cfg.k, cfg.d_ff, cfg.dtype, cfg.gate, cfg.renorm)
    a, c = moe.MoEHotPath(shape, device=DEV, aux_alpha=0.001), moe.MoEHotPath(shape, device=DEV, aux_alpha=0.001, seq_alpha=0.01, n_seqs=2)
    seqs = torch.tensor([0, 50], dtype=torch.int32, device=DEV), torch.tensor([50, 30], dtype=torch.int32, device=DEV)
    W = [g[n] for n in ("Wg", "Wu", "Wd")]
    for hp, kw in ((a, {}), (c, dict(seqs=seqs))):
        hp.forward(g["logits"], g["X"], *W, **kw)
        hp.backward(g["dY"], g["X"], *W)
    for n in ("Y", "dX", "dw", "topk_idx", "aux_loss"):
        assert torch.equal(a.b[n], c.b[n]), n
    _, _, loss, ds = ob.seq_loss(np64(p["logits"]), a.b["topk_idx"].cpu().numpy(), [(0, 50), (50, 80)], cfg.k, cfg.gate, 0.01, 0.0)
    assert scale_rel_err(c.b["dlogits"], np64(a.b["dlogits"]) + ds) <= 1e-5 and scale_rel_err(c.b["seq_loss"], loss) <= 1e-4
    assert not torch.equal(a.b["dlogits"], c.b["dlogits"])


def test_streams_and_graphs():
    """Eager on another stream, and captured with the step's advance in the graph: every replay has the masks of its own step, with eager work between the replays."""
    B, E = Block(T=80, dtype="bf16"), Block(T=80, dtype="bf16")
    side = torch.cuda.Stream()

    def run(x, **kw):
        x.forward(**kw)
        x.backward(**kw)

    run(E)
    want = E.outputs()
    torch.cuda.synchronize()
    run(B, stream=side)
    side.synchronize()
    for n, t in B.outputs().items():
        assert torch.equal(t, want[n]), n
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # what a first call does once (kernels are loaded) is not captured
        run(B)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(B)
        B.rng[1:].add_(1)
    B.rng.copy_(torch.tensor([99, 7], device=DEV))
    last = None
    for i in range(4):
        for n in ("Out", "dZ", "dWr", "dnorm_w", "seq_loss", "dlogits"):
            B.hp.b[n].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = B.outputs()
        E.rng.copy_(torch.tensor([99, 7 + i], device=DEV))
        run(E)   # eager work between the replays
        for n, t in E.outputs().items():
            assert torch.equal(t, got[n]), (i, n)
        assert last is None or not torch.equal(last, got["Out"])
        last = got["Out"]


def test_two_graphs_on_one_workspace():
    """The operators captured apart, on one workspace, replayed in turn with everything cleared in between."""
    import paper_2502_02581_amd as moe

    n, d, T, E = 300, 1000, 500, 24
    g = torch.Generator().manual_seed(3)
    X, dY = torch.randn(n, d, generator=g).bfloat16().cuda(), torch.randn(n, d, generator=g).bfloat16().cuda()
    logits = torch.randn(T, E, generator=g).cuda()
    topk = torch.topk(logits, 2, 1).indices.to(torch.int32)
    norm, shape = moe.MoENorm(n, d), moe.MoEShape(T, 8, E, 2, 8, "f32")
    Y, dR, w = torch.empty_like(X), torch.empty_like(X), torch.ones(d, device=DEV).bfloat16()
    mean, rstd, dw, db = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty_like(w), torch.empty_like(w)
    counts, P, loss, coef, dl = torch.empty(1, E, dtype=torch.int32, device=DEV), torch.empty(1, E, device=DEV), torch.empty(2, device=DEV), torch.empty(2, device=DEV), torch.empty_like(logits)
    ws = torch.empty(max(moe.moe_norm_bwd_workspace_bytes(norm), moe.moe_seq_loss_workspace_bytes(shape, 1)), dtype=torch.uint8, device=DEV)

    def one():
        moe.moe_norm_fwd(norm, X, w, None, Y, mean, rstd)
        moe.moe_norm_bwd(norm, dY, X, w, mean, rstd, dR, dw, db, ws)

    def two():
        moe.moe_seq_loss(shape, logits, topk, None, None, 0.1, 0.1, counts, P, loss, coef, ws)
        moe.moe_seq_loss_bwd(shape, logits, None, None, counts, coef, 1.0, False, dl)

    outs = (Y, mean, rstd, dR, dw, db, P, loss, coef, dl)
    one()
    two()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    graphs = []
    for f in (one, two):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f()
    for i in range(4):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        for q in (graphs if i % 2 else graphs[::-1]):
            q.replay()
        torch.cuda.synchronize()
        for t, r in zip(outs, want):
            assert torch.equal(t, r)
        one()


def test_two_streams_at_once():
    """The same calls on two streams side by side, each with tensors and a workspace of its own: the bits of one after the other.  A row of 16384 values, weights' gradients from
    the blocks' sums and from the columns, sequences of many chunks, the small call's single launch and the loss that the last block writes."""
    import paper_2502_02581_amd as moe

    class Calls:
        def __init__(self, seed):
            g = torch.Generator().manual_seed(seed)
            self.jobs, self.outs = [], []
            for n, d in ((6000, 1000), (200, 1000), (40, 16384)):
                X, dY = torch.randn(n, d, generator=g).bfloat16().to(DEV), torch.randn(n, d, generator=g).bfloat16().to(DEV)
                norm, Z, Y, dR, dX = moe.MoENorm(n, d), *(torch.empty_like(X) for _ in range(4))
                drop = moe.MoEDropout(0.3, torch.tensor([seed, 5], dtype=torch.int64, device=DEV), 2)
                mean, rstd, dw, db = (torch.empty(m, device=DEV) for m in (n, n, d, d))
                w, dw, db = torch.ones(d, device=DEV).bfloat16(), dw.bfloat16(), db.bfloat16()
                self.jobs.append(("norm", norm, X, dY, w, drop, Z, Y, dR, dX, mean, rstd, dw, db, self.space(moe.moe_norm_bwd_workspace_bytes(norm))))
                self.outs += [Z, Y, dR, dX, mean, rstd, dw, db]
            for T, E, S in ((9000, 60, 3), (100, 16, 4), (5000, 8, 2500)):
                logits = torch.randn(T, E, generator=g).to(DEV)
                topk, start = torch.topk(logits, 2, 1).indices.to(torch.int32), torch.tensor([T * i // S for i in range(S + 1)], dtype=torch.int32, device=DEV)
                shape, dl, counts = moe.MoEShape(T, 8, E, 2, 8, "f32"), torch.empty_like(logits), torch.empty(S, E, dtype=torch.int32, device=DEV)
                P, loss, coef = torch.empty(S, E, device=DEV), torch.empty(2, device=DEV), torch.empty(S + 1, device=DEV)
                self.jobs.append(("seq", shape, logits, topk, start, counts, P, loss, coef, dl, self.space(moe.moe_seq_loss_workspace_bytes(shape, S))))
                self.outs += [P, loss, coef, dl]

        @staticmethod
        def space(n):
            return torch.full((n,), 255, dtype=torch.uint8, device=DEV)

        def issue(self, job):
            if job[0] == "norm":
                _, norm, X, dY, w, drop, Z, Y, dR, dX, mean, rstd, dw, db, ws = job
                moe.moe_norm_fwd(norm, X, w, None, Y, mean, rstd, R=dY, drop=drop, Z=Z)
                moe.moe_norm_bwd(norm, dY, Z, w, mean, rstd, dR, dw, db, ws, drop=drop, dX=dX)
            else:
                _, shape, logits, topk, start, counts, P, loss, coef, dl, ws = job
                moe.moe_seq_loss(shape, logits, topk, start, None, 0.1, 0.1, counts, P, loss, coef, ws)
                moe.moe_seq_loss_bwd(shape, logits, start, None, counts, coef, 1.0, False, dl)

    sides = [Calls(1), Calls(2)]
    want = []
    for c in sides:
        for job in c.jobs:
            c.issue(job)
        torch.cuda.synchronize()
        want.append([t.clone() for t in c.outs])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(6):
        for c in sides:
            for t in c.outs:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        n = len(sides[0].jobs)
        for i in range(n):   # the two streams' jobs shifted against each other
            for j, (c, s) in enumerate(zip(sides, streams)):
                with torch.cuda.stream(s):
                    c.issue(c.jobs[(i + j * turn) % n])
        torch.cuda.synchronize()
        for c, w in zip(sides, want):
            for k, (t, r) in enumerate(zip(c.outs, w)):
                assert torch.equal(t, r), (turn, k)


def test_clipping_a_blocks_gradients():
    """gradients() lists the router's and the norm's, too."""
    import paper_2502_02581_amd as moe

    B = Block(dtype="bf16", n_shared=0)
    B.forward()
    B.backward()
    grads = B.hp.gradients()
    assert len(grads) == 6
    total = sum(float((x[0][:int(x[1])] if isinstance(x, tuple) else x).double().square().sum()) for x in grads) ** 0.5
    norm, ws = torch.zeros(1, device=DEV), torch.empty(moe.moe_grad_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
    moe.moe_grad_norm(grads, norm, ws)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total


def test_refusals():
    import paper_2502_02581_amd as moe

    shape = moe.MoEShape(8, 64, 4, 2, 64)
    for kw in (dict(dropout=0.1), dict(norm="layer", dropout=0.1), dict(norm="batch")):
        with pytest.raises(moe.MoEError):
            moe.MoEHotPath(shape, device=DEV, **kw)
    B = Block(T=8, dtype="bf16", n_shared=0)
    with pytest.raises(moe.MoEError, match="no forward pass"):
        B.backward()
    with pytest.raises(moe.MoEError, match="in the place of the logits"):
        B.hp.forward(torch.zeros(8, 6, device=DEV), B.X, *B.W)
    plain = moe.MoEHotPath(B.shape, device=DEV)
    with pytest.raises(moe.MoEError, match="go with norm"):
        plain.forward(B.w, B.X, *B.W)
    with pytest.raises(moe.MoEError, match="go with norm"):
        plain.forward(torch.zeros(8, 6, device=DEV), B.X, *B.W, residual=B.R)
