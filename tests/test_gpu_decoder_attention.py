"""Decoder problems with the attention options (grouped heads, query/key norms, packed documents,
rotary variants) through inner_step, hvp and meta_grad, against float64 automatic differentiation."""
import dataclasses

import pytest
import torch

from plain_decoder import Decoder

pytestmark = pytest.mark.gpu

# Normwise.  float32 operands: the 1e-4 of the other float32 problems.  bf16 operands: every product's
# two operands are off by up to 2^-8 of themselves; a gradient passes about 30 products of two blocks
# (forward, backward, unembedding), whose errors are independent: sqrt(60) 2^-8 = 3e-2.  A
# Hessian-vector product holds each of them twice (primal and tangent), a meta-gradient two such steps.
TOL = {(0, "grad"): 1e-4, (0, "hvp"): 1e-4, (0, "meta"): 1e-4,
       (1, "grad"): 3e-2, (1, "hvp"): 6e-2, (1, "meta"): 12e-2}

BASE = Decoder(docs=((0, 7, 8, 30, 30, 60), (3, 20, 41, 55, 58, 58)), val_docs=(0, 13, 40))
CASES = {
    "all": BASE,
    "grouped": dataclasses.replace(BASE, K=1, norm=0, docs=(), val_docs=()),
    "norms": dataclasses.replace(BASE, K=4, docs=(), val_docs=()),
    "documents": dataclasses.replace(BASE, K=4, norm=0),
    "rotary": dataclasses.replace(BASE, K=4, norm=0, docs=(), val_docs=(),
                                  rope=dict(rope_dims=10, rope_interleaved=1, rope_scaling=3, rope_factor=4.0,
                                            rope_train_len=64.0, rope_slow=1.0, rope_fast=8.0, rope_mscale=1.1)),
    "wide_heads": dataclasses.replace(BASE, d=160, H=2, K=1, F=64, S=68, rows=2, val_rows=1,
                                      docs=((0, 70, 136), (0, 1, 136)), val_docs=(60, 68), L=1),
}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_00793_amd import _lib
    _lib.lib()


def _ys(c):
    ints = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")
    return ([ints(d) for d in c.docs] if c.docs else [None] * c.T), ints(c.val_docs) if c.val_docs else None


def _meta(c, data):
    from paper_2505_00793_amd import _lib as M
    theta, eta, xs, vx = data
    P = M.Problem(c.desc())
    ys, vy = _ys(c)
    d, V = torch.full((eta.numel(),), float("nan"), device="cuda"), torch.empty(1, device="cuda")
    P.mfmg_meta_grad(theta.cuda(), None, eta.cuda(), [x.cuda() for x in xs], ys, vx.cuda(), vy, d, V)
    torch.cuda.synchronize()
    return d, V


def _rel(a, b):
    return float((a.double().cpu() - b.double().cpu()).norm() / b.double().norm())


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_float64(name, prec):
    from paper_2505_00793_amd import _lib as M
    print(f"\n[decoder] {name} prec {prec}", flush=True)
    c = dataclasses.replace(CASES[name], prec=prec)
    data = theta, eta, xs, vx = c.draw(3)
    P = M.Problem(c.desc())
    assert P.mfmg_query_sizes(c.T).n_theta == theta.numel()
    ys, _ = _ys(c)
    v = torch.randn(theta.numel(), generator=torch.Generator().manual_seed(9)) * 0.1
    want = c.hvp(theta, eta, xs[0], v)
    n = theta.numel()
    g, hv, mv = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(c.rows * c.S, device="cuda")
    P.mfmg_hvp_fwd_over_rev(theta.cuda(), eta.cuda(), xs[0].cuda(), ys[0], 0, v.cuda(), g, hv, mv)
    nxt, g2, loss = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
    P.mfmg_inner_step(theta.cuda(), None, eta.cuda(), xs[0].cuda(), ys[0], 0, nxt, grad_out=g2, loss_out=loss)
    d, V = _meta(c, data)
    d64, V64 = c.meta_grad(*data)
    errs = {"grad": _rel(g, want[0]), "step": _rel(g2, want[0]), "hvp": _rel(hv, want[1]),
            "mvp": _rel(mv, want[2]), "meta": _rel(d, d64), "V": abs(float(V) / float(V64) - 1)}
    print("  " + ", ".join(f"{k} {e:.1e}" for k, e in errs.items()), flush=True)
    if c.norm:   # the gains' own gradients, which the other parameters outweigh
        off = 0
        for nm, shape in c.shapes():
            k = int(torch.tensor(shape).prod())
            if nm[:2] == "qk" and nm[2] != "v":
                assert _rel(g[off:off + k], want[0][off:off + k]) <= 2 * TOL[prec, "grad"], nm
                assert _rel(hv[off:off + k], want[1][off:off + k]) <= 2 * TOL[prec, "hvp"], nm
            off += k
    for k, kind in (("grad", "grad"), ("step", "grad"), ("hvp", "hvp"), ("mvp", "hvp"), ("meta", "meta"), ("V", "grad")):
        assert errs[k] <= TOL[prec, kind], (k, errs[k])


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
def test_rematerialisation_and_graph_replay_are_bit_identical(prec):
    """Block rematerialisation repeats the same kernels; a captured call replays to the eager result."""
    from paper_2505_00793_amd import _lib as M
    print(f"\n[decoder] remat, graph, prec {prec}", flush=True)
    c = dataclasses.replace(BASE, prec=prec, L=3)
    data = theta, eta, xs, vx = c.draw(4)
    want, V = _meta(c, data)
    got, _ = _meta(dataclasses.replace(c, remat=1), data)
    assert torch.isfinite(want).all() and torch.equal(got, want)
    P = M.Problem(c.desc())
    ws = P.workspace(P.mfmg_query_sizes(c.T).workspace_bytes)
    ys, vy = _ys(c)
    dev = (theta.cuda(), None, eta.cuda(), [x.cuda() for x in xs], ys, vx.cuda(), vy)
    out, Vo = torch.empty_like(want), torch.empty(1, device="cuda")
    P.mfmg_meta_grad(*dev, out, Vo, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.mfmg_meta_grad(*dev, out, Vo, ws=ws)
    for k in range(3):
        out.fill_(float("nan"))
        graph.replay()
        _meta(dataclasses.replace(c, remat=1), data)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(Vo, V), f"replay {k}"


def test_documents_that_are_rows_match_the_plain_decoder():
    """Documents cut at the rows are what the plain decoder does: both bf16 paths agree to within the
    bf16 bounds of either."""
    print("\n[decoder] documents at the rows", flush=True)
    c = Decoder(d=128, H=2, K=2, F=128, S=64, rows=4, val_rows=2, norm=0, prec=1)
    data = c.draw(6)
    plain, Vp = _meta(c, data)
    docs, Vd = _meta(dataclasses.replace(c, docs=((0, 64, 128, 192, 256),) * 2, val_docs=(64, 128)), data)
    assert _rel(docs, plain) <= TOL[1, "meta"]
    assert abs(float(Vd) / float(Vp) - 1) <= TOL[1, "grad"]
    one, _ = _meta(dataclasses.replace(c, docs=((0, 64, 128, 192, 256),) * 2, val_docs=(0, 0)), data)
    assert not torch.equal(one, docs)   # (two validation rows as one document are another problem)
