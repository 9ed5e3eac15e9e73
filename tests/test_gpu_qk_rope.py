"""Query/key norms and rotary positions (mfmg_qk_rope_fwd / mfmg_qk_rope_bwd), primal and dual, against
their float64 form: a result is off by at most one rounding to its type and 64 float32 steps of the
sum of its absolute terms (about forty operations lie between an input and a result, the norm's sum
of 128 squares and the angle's steps among them); a gain's gradient also by the sum over its rows."""
import math

import pytest
import torch

import packed_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_00793_amd import _lib
    _lib.lib()


FREE = dict(rope_dims=0, rope_interleaved=False, rope_base=10000.0, rope_scaling=0, rope_factor=1.0,
            rope_train_len=0.0, rope_mscale=0.0)


def _case(prec, H, K, dh, n, norm, dual, first=0, unused=0, gap=0, pos=None, seed=0, **rope):
    """One forward and backward; {name: (got, value, absolute terms)}."""
    from paper_2505_00793_amd import _lib as M
    opt = {**FREE, **rope}
    T = torch.bfloat16 if prec else torch.float32
    op = M.Attention(M.make_attn_desc(heads=H, kv_heads=K, head_dim=dh, precision=prec, qk_norm=norm,
                                      norm_eps=1e-5, **opt))
    g = torch.Generator(device="cuda").manual_seed(seed)
    N, W = first + n + unused, (H + 2 * K) * dh
    cut = max(1, n // 3)
    cu = torch.tensor([first, first + cut, first + cut, first + n], dtype=torch.int32, device="cuda")
    at = torch.zeros(N, dtype=torch.int64)
    at[first:first + cut] = torch.arange(cut)
    at[first + cut:first + n] = torch.arange(n - cut)
    if pos is not None:
        at = torch.as_tensor(pos(N), dtype=torch.int64)
    plan = M.mfmg_seq_plan(cu, N, positions=at.int().cuda() if pos is not None else None)

    def rows(s, dtype, on=True):
        if not on:
            return None
        t = torch.randn(N, W + gap, device="cuda", generator=g).mul_(s).to(dtype)[:, :W]
        t[:first] = float("nan")
        t[first + n:] = float("nan")
        return t

    def out(on=True):
        return torch.full((N, W + gap), 7.0, device="cuda", dtype=T)[:, :W] if on else None
    x, xd, dy, dyd = rows(1.5, torch.float32), rows(0.4, torch.float32, dual), rows(1, T), rows(0.4, T, dual)
    gain = 1 + 0.3 * torch.randn(2, dh, device="cuda", generator=g) if norm else None
    gaind = 0.3 * torch.randn(2, dh, device="cuda", generator=g) if norm and dual else None
    y, yd, dx, dxd = out(), out(dual), out(), out(dual)
    dgain = torch.full((2, dh), 7.0, device="cuda") if norm else None
    dgaind = torch.full((2, dh), 7.0, device="cuda") if norm and dual else None
    op.mfmg_qk_rope_fwd(plan, x, y, gain=gain, xd=xd, gaind=gaind, yd=yd)
    op.mfmg_qk_rope_bwd(plan, dy, dx, x=x if norm else None, gain=gain, dgain=dgain, dyd=dyd, dxd=dxd,
                        xd=xd if norm else None, gaind=gaind, dgaind=dgaind)
    torch.cuda.synchronize()
    got = {k: t for k, t in (("y", y), ("yd", yd), ("dx", dx), ("dxd", dxd), ("dgain", dgain),
                             ("dgaind", dgaind)) if t is not None}
    D = opt["rope_dims"] or dh
    fr = R.frequencies(D, opt["rope_base"], opt["rope_scaling"], opt["rope_factor"], opt["rope_train_len"])
    s = slice(first, first + n)

    def d(t):
        return None if t is None else (t[s] if t.shape[0] == N and t.shape[1] == W else t).double()
    val, ab = (R.Rope(H, K, dh, at[s].cuda(), D, opt["rope_interleaved"], opt["rope_mscale"] or 1.0, fr,
                      1e-5, a).run(d(x).contiguous(), d(gain), d(xd) if xd is None else d(xd).contiguous(),
                                   d(gaind), d(dy).contiguous(), d(dyd) if dyd is None else d(dyd).contiguous())
               for a in (False, True))
    for k, t in got.items():
        if k in ("dgain", "dgaind"):
            bound = (64 + n * max(H, K)) * R.E * ab[k]
            err = (t.double() - val[k]).abs()
        else:
            bound = R.unit(T) * val[k].abs() + 64 * R.E * ab[k]
            err = (t[s].double() - val[k]).abs()
            rest = torch.cat((t[:first], t[first + n:]))
            assert torch.equal(rest, torch.full_like(rest, 7.0)), f"{k}: unused rows were written"
        worst = float((err / (bound + 1e-30)).max())
        assert worst <= 1.0, f"{k}: {worst:.2f} of its bound (or not a number)"
    return got


SHAPES = [
    # heads, key heads, head size, rows, options
    (1, 1, 8, 1, {}),
    (8, 8, 64, 100, {}),
    (6, 2, 128, 67, dict(rope_dims=64)),
    (4, 1, 128, 33, dict(rope_interleaved=True, rope_base=500000.0)),
    (5, 5, 40, 70, dict(rope_dims=20)),
    (2, 1, 72, 41, dict(rope_dims=36, rope_interleaved=True)),
    (3, 1, 80, 50, dict(rope_dims=2)),
    (4, 2, 16, 130, dict(rope_dims=10, rope_interleaved=True)),
    (4, 4, 32, 64, dict(rope_scaling=1, rope_factor=4.0)),
    (4, 2, 96, 64, dict(rope_scaling=2, rope_factor=8.0, rope_dims=48)),
    (4, 2, 64, 64, dict(rope_scaling=3, rope_factor=8.0, rope_train_len=4096.0, rope_mscale=1.2)),
    (32, 8, 128, 300, {}),
    (2, 2, 64, 9000, {}),
]


@pytest.mark.parametrize("dual", [False, True], ids=["primal", "dual"])
@pytest.mark.parametrize("norm", [False, True], ids=["rope", "norm"])
@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("H,K,dh,n,opt", SHAPES, ids=lambda v: str(v).replace(" ", "") if not isinstance(v, dict) else "-".join(v))
def test_against_float64(prec, norm, dual, H, K, dh, n, opt):
    print(f"\n[rope] H {H} K {K} dh {dh} n {n} {opt} norm {norm} prec {prec} dual {dual}", flush=True)
    _case(prec, H, K, dh, n, norm, dual, first=2, unused=5, gap=16, **opt)


@pytest.mark.parametrize("inter", [False, True], ids=["half", "interleaved"])
def test_far_and_negative_positions(inter):
    """Angles of positions up to 2^31 - 1 come out as in float64 (a float32 product would be off by
    whole turns)."""
    far = [0, 1, -1, 12345678, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31, 999999937]
    print("\n[rope] far positions", flush=True)

    def pos(N):
        return [far[i % len(far)] for i in range(N)]
    # position 2^31 times a frequency's float64 rounding (2^-53 of up to one turn a step) is 2^-22
    # turns: within 64 float32 steps of the result's terms
    _case(0, 4, 2, 64, 40, False, True, pos=pos, rope_interleaved=inter)


def test_rows_of_zero_and_repeats():
    """A head of zeros has a finite norm (eps), and the gains' gradients repeat bit for bit."""
    from paper_2505_00793_amd import _lib as M
    print("\n[rope] zero rows", flush=True)
    op = M.Attention(M.make_attn_desc(heads=2, kv_heads=1, head_dim=64, qk_norm=True))
    n = 500
    x = torch.zeros(n, 256, device="cuda")
    gain = torch.ones(2, 64, device="cuda")
    y = torch.empty(n, 256, device="cuda")
    plan = M.mfmg_seq_plan(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    op.mfmg_qk_rope_fwd(plan, x, y, gain=gain)
    assert torch.equal(y, torch.zeros_like(y))
    x.normal_()
    dy = torch.randn(n, 256, device="cuda")
    outs = []
    for _ in range(3):
        dx, dgain = torch.empty_like(x), torch.empty_like(gain)
        op.mfmg_qk_rope_bwd(plan, dy, dx, x=x, gain=gain, dgain=dgain)
        outs.append((dx, dgain))
    torch.cuda.synchronize()
    assert all(torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1]) for a, b in outs)


@pytest.mark.parametrize("norm", [False, True], ids=["rope", "norm"])
def test_no_tokens_and_no_sequences(norm):
    """No rows: nothing to do, the gains' gradients are zero; rows of no sequence stay as they were."""
    from paper_2505_00793_amd import _lib as M
    print("\n[rope] nothing to do", flush=True)
    op = M.Attention(M.make_attn_desc(heads=2, kv_heads=1, head_dim=32, qk_norm=norm))
    gain = torch.ones(2, 32, device="cuda") if norm else None
    for n in (0, 6):
        plan = M.mfmg_seq_plan(torch.zeros(1, dtype=torch.int32, device="cuda"), n)
        x, y, dx = (torch.full((n, 128), 3.0, device="cuda") for _ in range(3))
        dgain = torch.full((2, 32), 5.0, device="cuda") if norm else None
        op.mfmg_qk_rope_fwd(plan, x, y, gain=gain)
        op.mfmg_qk_rope_bwd(plan, x, dx, x=x if norm else None, gain=gain, dgain=dgain)
        stats = torch.empty(2, 2, n, device="cuda")
        o = torch.full((n, 64), 3.0, device="cuda")
        op.mfmg_attn_fwd(plan, x[:, :64], x[:, 64:96], x[:, 96:], o, stats)
        op.mfmg_attn_bwd(plan, x[:, :64], x[:, 64:96], x[:, 96:], o, stats, o.clone(), dx[:, :64],
                         dx[:, 64:96], dx[:, 96:])
        torch.cuda.synchronize()
        for t in (y, dx, o):
            assert torch.equal(t, torch.full_like(t, 3.0))
        if norm:
            assert torch.equal(dgain, torch.zeros_like(dgain))


def test_block_of_operators_matches_autograd_and_differences():
    """Norms, rotation and attention run together, as a decoder block runs them, over two sequences:
    gradients against float64 autograd, their derivative along a tangent against differences of
    those gradients."""
    from paper_2505_00793_amd import _lib as M
    print("\n[rope] chained with attention", flush=True)
    H, K, dh, lens = 4, 2, 32, [70, 45]
    n, W = sum(lens), (H + 2 * K) * dh
    op = M.Attention(M.make_attn_desc(heads=H, kv_heads=K, head_dim=dh, qk_norm=True, norm_eps=1e-5, rope_dims=16))
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, xd, gain, gaind = (torch.randn(*s, device="cuda", generator=gen) for s in ((n, W), (n, W), (2, dh), (2, dh)))
    g = torch.randn(n, H * dh, device="cuda", generator=gen)
    gd = torch.randn(n, H * dh, device="cuda", generator=gen)
    cu = torch.tensor([0, 70, n], dtype=torch.int32, device="cuda")
    plan = M.mfmg_seq_plan(cu, n)
    cut = (H * dh, K * dh, K * dh)
    new = lambda w: torch.empty(n, w, device="cuda")
    y, yd, o, od, dy, dyd, dx, dxd = new(W), new(W), new(H * dh), new(H * dh), new(W), new(W), new(W), new(W)
    dgain, dgaind = torch.empty(2, dh, device="cuda"), torch.empty(2, dh, device="cuda")
    stats = torch.empty(2, H, n, device="cuda")
    op.mfmg_qk_rope_fwd(plan, x, y, gain, xd, gaind, yd)
    op.mfmg_attn_fwd(plan, *y.split(cut, 1), o, stats, *yd.split(cut, 1), od)
    op.mfmg_attn_bwd(plan, *y.split(cut, 1), o, stats, g, *dy.split(cut, 1), *yd.split(cut, 1), od, gd, *dyd.split(cut, 1))
    op.mfmg_qk_rope_bwd(plan, dy, dx, x, gain, dgain, dyd, dxd, xd, gaind, dgaind)
    torch.cuda.synchronize()

    ang = torch.cat([torch.arange(L) for L in lens]).double()[:, None] * R.frequencies(16)
    c, s = torch.cos(ang)[:, None].cuda(), torch.sin(ang)[:, None].cuda()

    def plain(x, gain):
        t = x.view(n, H + 2 * K, dh)
        t, v = t[:, :H + K], t[:, H + K:]
        w = torch.cat((gain[0].expand(H, dh), gain[1].expand(K, dh)))
        t = w * t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-5)
        a, b = t[..., :8], t[..., 8:16]
        t = torch.cat((a * c - b * s, a * s + b * c, t[..., 16:]), -1)
        q, k = t[:, :H], t[:, H:].repeat_interleave(H // K, 1)
        v = v.repeat_interleave(H // K, 1)
        out, lo = [], 0
        for L in lens:
            S = torch.matmul(q[lo:lo + L].transpose(0, 1), k[lo:lo + L].permute(1, 2, 0)) / math.sqrt(dh)
            S = S.masked_fill(torch.ones(L, L, device="cuda").triu(1).bool(), -math.inf)
            out.append(torch.matmul(S.softmax(-1), v[lo:lo + L].transpose(0, 1)).transpose(0, 1))
            lo += L
        return torch.cat(out).reshape(n, -1)

    def grads(e):
        xe, ge = (x.double() + e * xd).requires_grad_(), (gain.double() + e * gaind).requires_grad_()
        out = plain(xe, ge)
        return [out.detach(), *torch.autograd.grad(out, (xe, ge), g.double() + e * gd)]

    h = 1e-5
    base, up, dn = grads(0.0), grads(h), grads(-h)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    # chained float32 operators: a few hundred steps of 2^-24, normwise
    for got, want in zip((o, dx, dgain), base):
        assert rel(got, want) <= 300 * R.E
    # central differences in float64: h^2 and 2^-53 / h both below 1e-10 relative, so the same bound
    # times the amplification of a second derivative
    for got, a, b in zip((od, dxd, dgaind), up, dn):
        assert rel(got, (a - b) / (2 * h)) <= 1000 * R.E


@pytest.mark.parametrize("dual", [False, True], ids=["primal", "dual"])
@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("dh,dims,inter", [(64, 16, False), (64, 10, False), (64, 6, True), (8, 2, True), (128, 96, False)])
def test_infinities_pass_where_nothing_rotates(prec, dual, dh, dims, inter):
    """An infinity in a dim that does not rotate comes out as it is and reaches no other dim."""
    from paper_2505_00793_amd import _lib as M
    T = torch.bfloat16 if prec else torch.float32
    op = M.Attention(M.make_attn_desc(heads=3, kv_heads=1, head_dim=dh, precision=prec,
                                      **{**FREE, "rope_dims": dims, "rope_interleaved": inter}))
    n, W = 9, 5 * dh
    plan = M.mfmg_seq_plan(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    x = torch.ones(n, W, device="cuda")
    at = torch.zeros(n, W, dtype=torch.bool, device="cuda")
    at.view(n, 5, dh)[:, :, dims:][::2, ::2, ::3] = True
    x[at] = float("inf")
    xd = x if dual else None
    y, dx = (torch.zeros(n, W, device="cuda", dtype=T) for _ in range(2))
    yd, dxd = (torch.zeros(n, W, device="cuda", dtype=T) if dual else None for _ in range(2))
    op.mfmg_qk_rope_fwd(plan, x, y, xd=xd, yd=yd)
    g = x.to(T)
    op.mfmg_qk_rope_bwd(plan, g, dx, dyd=g if dual else None, dxd=dxd)
    for t in (y, yd, dx, dxd):
        if t is not None:
            assert torch.equal(t == float("inf"), at) and torch.isfinite(t[~at]).all()
