"""Causal attention over packed sequences with grouped heads (mfmg_attn_fwd / mfmg_attn_bwd), primal
and dual, against its float64 form within elementwise bounds (packed_ref.py): lengths from none to
several tiles, head sizes that no tile has, strided rows, unused rows and sequences that hold NaN."""
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


def _lib():
    from paper_2505_00793_amd import _lib as M
    return M


class Call:
    """Inputs, buffers and handle of one batch: `before` unused rows, the sequences, `after` more."""

    def __init__(self, prec, H, K, dh, lens, dual, before=0, after=0, seed=0, gap=0, scale=0.0):
        M = _lib()
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T = torch.bfloat16 if prec else torch.float32
        self.n = n = before + sum(lens) + after
        self.H, self.K, self.dh, self.lens, self.first, self.dual = H, K, dh, lens, before, dual
        self.scale = scale or 1 / math.sqrt(dh)
        self.op = M.Attention(M.make_attn_desc(heads=H, kv_heads=K, head_dim=dh, precision=prec, scale=scale))
        cu = torch.tensor([before] + [before + sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32)
        self.cu = cu.cuda()
        self.plan = M.mfmg_seq_plan(self.cu, n)

        def rows(w, s):
            t = torch.randn(n, w + gap, device="cuda", generator=g).mul_(s).to(self.T)[:, :w]
            t[:before] = float("nan")
            t[n - after:] = float("nan")
            return t
        W = (H + 2 * K) * dh
        cut = (H * dh, K * dh, K * dh)
        self.x = rows(W, 1.2).split(cut, 1)
        self.xd = rows(W, 0.4).split(cut, 1) if dual else (None,) * 3
        self.g, self.gd = rows(H * dh, 1.0), rows(H * dh, 0.4) if dual else None
        self.fill = 7.0

        def out(w):
            return torch.full((n, w + gap), self.fill, device="cuda", dtype=self.T)[:, :w]
        self.o, self.od = out(H * dh), out(H * dh) if dual else None
        self.dx = out(W).split(cut, 1)
        self.dxd = out(W).split(cut, 1) if dual else (None,) * 3
        self.stats = torch.full((2, H, n), float("nan"), device="cuda")
        self.ws = self.op.workspace(n).fill_(255)

    def run(self):
        self.op.mfmg_attn_fwd(self.plan, *self.x, self.o, self.stats, *self.xd, self.od)
        self.op.mfmg_attn_bwd(self.plan, *self.x, self.o, self.stats, self.g, *self.dx, *self.xd, self.od,
                              self.gd, *self.dxd, ws=self.ws)
        return self

    def outputs(self):
        d = {"o": self.o, "dq": self.dx[0], "dk": self.dx[1], "dv": self.dx[2]}
        if self.dual:
            d.update(od=self.od, dqd=self.dxd[0], dkd=self.dxd[1], dvd=self.dxd[2])
        return d

    def reference(self):
        def v(t):
            t = t.double().view(self.n, -1, self.dh) if t.is_contiguous() else t.double().reshape(self.n, -1, self.dh)
            return torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0)
        return R.attention(*map(v, self.x), self.lens, self.scale, self.T,
                           tan=tuple(map(v, self.xd)) if self.dual else None, g=v(self.g),
                           gd=v(self.gd) if self.dual else None, first=self.first)

    def check(self, skip=()):
        """Every output within its bound (sequences in `skip` excepted), unused rows untouched."""
        ref = self.reference()
        used = torch.zeros(self.n, dtype=torch.bool, device="cuda")
        lo = self.first
        for i, L in enumerate(self.lens):
            if i not in skip:
                used[lo:lo + L] = True
            lo += L
        for name, got in self.outputs().items():
            val, bound = (t.reshape(self.n, -1) for t in ref[name])
            err = (got.double() - val).abs()[used]
            worst = float((err / (bound[used] + 1e-30)).max()) if err.numel() else 0.0
            assert worst <= 1.0, f"{name}: {worst:.2f} of its bound (or not a number)"
            rest = torch.cat((got[:self.first], got[lo:]))
            assert torch.equal(rest, torch.full_like(rest, self.fill)), f"{name}: unused rows were written"


SHAPES = [
    # heads, key heads, head size, lengths
    (1, 1, 8, [1]),
    (2, 1, 16, [1, 0, 2, 31, 32, 33]),
    (4, 2, 64, [63, 64, 65, 1, 127]),
    (3, 3, 40, [128, 129, 0, 0, 17]),
    (8, 1, 128, [200, 5, 130]),
    (6, 3, 72, [257, 300]),
    (2, 2, 96, [64, 191]),
    (4, 4, 64, [700]),
    (2, 1, 128, [513]),
]


@pytest.mark.parametrize("dual", [False, True], ids=["primal", "dual"])
@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("H,K,dh,lens", SHAPES, ids=lambda v: str(v).replace(" ", ""))
def test_against_float64(prec, dual, H, K, dh, lens):
    print(f"\n[packed] H {H} K {K} dh {dh} lens {lens} prec {prec} dual {dual}", flush=True)
    c = Call(prec, H, K, dh, lens, dual, before=3, after=70, gap=16).run()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
def test_many_short_sequences(prec):
    lens = [1 + (7 * i) % 13 for i in range(90)] + [0] * 5 + [150]
    print(f"\n[packed] {len(lens)} short sequences", flush=True)
    c = Call(prec, 4, 2, 32, lens, True, after=1, scale=0.3).run()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_a_bad_sequence_stays_alone(prec, bad):
    """A sequence whose rows are not finite changes nothing of its neighbours, bit for bit."""
    lens = [70, 30, 140]
    print(f"\n[packed] a sequence of {bad}", flush=True)
    good = Call(prec, 2, 1, 64, lens, True).run()
    c = Call(prec, 2, 1, 64, lens, True)
    for t in (*c.x, *c.xd, c.g, c.gd):
        t[70:100] = bad
    c.run()
    torch.cuda.synchronize()
    for name, got in c.outputs().items():
        want = good.outputs()[name]
        assert torch.equal(got[:70], want[:70]) and torch.equal(got[100:], want[100:]), name


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
def test_large_scores(prec):
    """Scores of hundreds: one key takes all of a row, the maximum is subtracted before exp."""
    print("\n[packed] large scores", flush=True)
    c = Call(prec, 2, 2, 64, [90, 200], False, scale=8.0).run()
    torch.cuda.synchronize()
    o = c.o.float()
    assert torch.isfinite(o).all()
    q, k, v = (t.double().reshape(c.n, 2, 64) for t in c.x)
    for lo, hi in ((0, 90), (90, 290)):
        S = 8.0 * torch.einsum("qhd,khd->hqk", q[lo:hi], k[lo:hi])
        S = S.masked_fill(torch.ones(hi - lo, hi - lo, device="cuda").triu(1).bool(), -math.inf)
        top = S.topk(2, -1).values
        sure = (top[..., 0] - top[..., 1] > 30) | (top[..., 1] == -math.inf)   # e^-30 of the rest
        pick = torch.stack([v[lo:hi, h][S[h].argmax(-1)] for h in range(2)])
        got = c.o[lo:hi].double().reshape(hi - lo, 2, 64).transpose(0, 1)
        assert sure.any()
        # weights 1 to within e^-30 and the denominator's float32 steps: v itself, rounded once
        assert (got - pick).abs()[sure].max() <= 1e-5


def test_calls_repeat_bit_for_bit_and_in_graphs():
    """Two plans on one stream, replays of a captured call and a call on another stream all give the
    eager result."""
    M = _lib()
    print("\n[packed] graph and streams", flush=True)
    c = Call(1, 4, 2, 64, [100, 37, 260], True, after=5).run()
    want = {k: t.clone() for k, t in c.outputs().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[k]) for k, t in c.outputs().items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mfmg_seq_plan(c.cu, c.n, plan=c.plan)
        c.run()
    other = Call(1, 2, 2, 128, [64, 500], False, seed=3)
    for k in range(3):
        for t in c.outputs().values():
            t.fill_(c.fill)
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[n]) for n, t in c.outputs().items()), f"replay {k}"
    other.check()


def test_long_rows_pass_32_bit_offsets():
    """Rows 2^20 elements apart, so that the last ones lie past 2^31 elements."""
    print("\n[packed] wide rows", flush=True)
    M = _lib()
    n, H, dh, ld = 2200, 2, 64, 1 << 20
    op = M.Attention(M.make_attn_desc(heads=H, kv_heads=1, head_dim=dh, precision=1))
    big = torch.empty(n, ld, device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(1)
    W = (H + 2) * dh
    x = torch.randn(n, W, device="cuda", generator=g).bfloat16()
    big[:, :W] = x
    plan = M.mfmg_seq_plan(torch.tensor([0, 1000, n], dtype=torch.int32, device="cuda"), n)
    stats = torch.empty(2, H, n, device="cuda")
    cut = (H * dh, dh, dh)
    o, o2 = big[:, 1024:1024 + H * dh], torch.empty(n, H * dh, device="cuda", dtype=torch.bfloat16)
    op.mfmg_attn_fwd(plan, *big[:, :W].split(cut, 1), o, stats)
    op.mfmg_attn_fwd(plan, *x.split(cut, 1), o2, stats)
    torch.cuda.synchronize()
    assert torch.equal(o, o2)


LARGE = [
    # enough rows for the large tiles: heads * rows past 512 tiles of 128 (bf16) or 64 (fp32)
    (32, 4, 64, [700, 129, 1, 640, 63, 600]),
    (32, 8, 128, [517, 64, 300, 1300]),
    (36, 12, 96, [1000, 31, 900]),
    (64, 64, 24, [513, 256, 255, 30]),
    (44, 11, 40, [800, 777]),
]


@pytest.mark.parametrize("dual", [False, True], ids=["primal", "dual"])
@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("H,K,dh,lens", LARGE, ids=lambda v: str(v).replace(" ", ""))
def test_many_rows_against_float64(prec, dual, H, K, dh, lens):
    print(f"\n[packed] H {H} K {K} dh {dh} lens {lens} prec {prec} dual {dual}", flush=True)
    c = Call(prec, H, K, dh, lens, dual, before=1, after=9, gap=16).run()
    torch.cuda.synchronize()
    c.check()


def test_offsets_are_clamped_and_made_ascending():
    """Offsets past the rows, negative or descending: the same plan as their running maximum within the
    rows, more sequences than tokens and than one pass of the planning among them."""
    M = _lib()
    print("\n[packed] wild offsets", flush=True)
    n, H, dh = 700, 2, 32
    g = torch.Generator().manual_seed(2)
    wild = torch.randint(-200, 900, (3000,), generator=g, dtype=torch.int32)
    wild[0] = 5
    wild[1:2000] = wild[1:2000].clamp(max=300)
    wild[2990] = 2 ** 31 - 1
    wild[2995] = -2 ** 31
    tame = wild.clamp(0, n).cummax(0).values.to(torch.int32)
    op = M.Attention(M.make_attn_desc(heads=H, kv_heads=1, head_dim=dh))
    x = torch.randn(n, (H + 2) * dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    cut = (H * dh, dh, dh)
    res = []
    for cu in (wild, tame, tame.unique_consecutive()):
        plan = M.mfmg_seq_plan(cu.cuda(), n)
        o, dx = torch.full((n, H * dh), 7.0, device="cuda"), torch.full_like(x, 7.0)
        y = torch.full_like(x, 7.0)
        stats = torch.empty(2, H, n, device="cuda")
        op.mfmg_qk_rope_fwd(plan, x, y)
        op.mfmg_attn_fwd(plan, *x.split(cut, 1), o, stats)
        op.mfmg_attn_bwd(plan, *x.split(cut, 1), o, stats, x[:, :H * dh], *dx.split(cut, 1))
        torch.cuda.synchronize()
        res.append((o, dx, y))
    for got in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got, res[0]))
    first = int(tame[0])
    assert torch.equal(res[0][0][:first], torch.full((first, H * dh), 7.0, device="cuda"))


def test_many_tiles_of_one_length_class():
    """More tiles than the planning's classes of length, one long sequence among short ones: every tile
    is done once."""
    M = _lib()
    print("\n[packed] many tiles", flush=True)
    lens = [40000] + [3, 65, 1, 130] * 700
    n = sum(lens)
    op = M.Attention(M.make_attn_desc(heads=1, head_dim=8, precision=1))
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    plan = M.mfmg_seq_plan(cu, n)
    v = torch.ones(n, 8, device="cuda", dtype=torch.bfloat16)
    q, k = (torch.randn(n, 8, device="cuda").bfloat16() for _ in range(2))
    o, dv = torch.zeros_like(v), torch.zeros_like(v)
    dq, dk = torch.ones_like(v), torch.ones_like(v)
    stats = torch.empty(2, 1, n, device="cuda")
    op.mfmg_attn_fwd(plan, q, k, v, o, stats)
    assert (o.float() - 1).abs().max() <= 2 ** -6   # weights of a row sum to 1: P's rounding and o's
    op.mfmg_attn_bwd(plan, q, k, v, o, stats, v, dq, dk, dv)
    torch.cuda.synchronize()
    # the columns' weights sum to the number of rows; v is constant, so dP is, and dS vanishes
    per = dv.float()[:, 0].double().cpu()
    ends = cu.cpu().tolist()
    for a, b in zip(ends, ends[1:]):
        assert abs(float(per[a:b].sum()) / (b - a) - 1) <= 2 ** -7
    assert dq.float().abs().max() < 1 and dk.float().abs().max() < 1


@pytest.mark.parametrize("dual", [False, True], ids=["primal", "dual"])
@pytest.mark.parametrize("H,K,dh,lens", [(2, 1, 64, [900, 333]), (4, 2, 40, [515]), (3, 3, 128, [600, 20, 270]),
                                         (1, 1, 24, [256])], ids=lambda v: str(v).replace(" ", ""))
def test_few_long_float32_rows(dual, H, K, dh, lens):
    """Float32 rows few enough for tiles whose four waves share them."""
    print(f"\n[packed] H {H} K {K} dh {dh} lens {lens} dual {dual}", flush=True)
    c = Call(0, H, K, dh, lens, dual, before=0, after=2).run()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
def test_widest_rows(prec):
    """The largest leading dimension, 2^22: a block's rows span 2^30 bytes.  The same bits as from dense rows."""
    print("\n[packed] rows 2^22 elements apart", flush=True)
    M = _lib()
    n, H, dh, ld = 131, 3, 128, 1 << 22
    T = torch.bfloat16 if prec else torch.float32
    op = M.Attention(M.make_attn_desc(heads=H, kv_heads=1, head_dim=dh, precision=prec))
    plan = M.mfmg_seq_plan(torch.tensor([0, 70, 70, n], dtype=torch.int32, device="cuda"), n)
    W, Q, gen = (H + 2) * dh, H * dh, torch.Generator(device="cuda").manual_seed(2)
    wide = torch.empty(n, ld, device="cuda", dtype=T)
    part = torch.randn(n, 2 * W + 2 * Q, device="cuda", generator=gen).to(T)
    ws, out = op.workspace(n), []
    for rows in (part.clone(), wide[:, :part.shape[1]].copy_(part)):
        x, dx, o, g = rows.split((W, W, Q, Q), 1)
        cut, stats = (Q, dh, dh), torch.empty(2, H, n, device="cuda")
        op.mfmg_attn_fwd(plan, *x.split(cut, 1), o, stats)
        op.mfmg_attn_bwd(plan, *x.split(cut, 1), o, stats, g, *dx.split(cut, 1), ws=ws)
        torch.cuda.synchronize()
        out.append(torch.cat((o, dx), 1))
    assert torch.isfinite(out[0]).all() and torch.equal(*out)


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("dh", [8, 72, 128])
def test_a_key_at_minus_infinity_has_no_weight(prec, dh):
    """Scores of -inf (keys 1, 5 and 40 hold -inf where every query holds 1) leave the other keys' result."""
    print(f"\n[packed] keys at -inf, dh {dh}", flush=True)
    M = _lib()
    n, T = 70, torch.bfloat16 if prec else torch.float32
    op = M.Attention(M.make_attn_desc(heads=1, kv_heads=1, head_dim=dh, precision=prec))
    plan = M.mfmg_seq_plan(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    gen = torch.Generator(device="cuda").manual_seed(dh)
    q, k, v = (torch.randn(n, dh, device="cuda", generator=gen).to(T) for _ in range(3))
    q[:, -1] = 1
    k[[1, 5, 40], -1] = float("-inf")
    o, stats = torch.empty(n, dh, device="cuda", dtype=T), torch.empty(2, 1, n, device="cuda")
    op.mfmg_attn_fwd(plan, q, k, v, o, stats)
    torch.cuda.synchronize()
    s = (q.double() @ k.double().t()) * dh ** -0.5
    p = torch.softmax(s.masked_fill(torch.ones_like(s).triu(1).bool(), float("-inf")), 1)
    # one rounding of each weight and of the result; a score is off by dh + 8 float32 steps of its
    # absolute terms, a sum of weights by n, both in numerator and denominator
    u = R.unit(T)
    terms = (q.double().abs() @ k.double().abs().t()).nan_to_num(posinf=0.0).amax(1, keepdim=True) * dh ** -0.5
    bound = u * (p @ v.double()).abs() + (u + 2 * R.E * ((dh + 8) * terms + n)) * (p @ v.double().abs())
    assert ((o.double() - p @ v.double()).abs() <= bound).all()


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n,first", [(70, 33), (300, 64), (300, 129)])
def test_leading_keys_at_minus_infinity(prec, n, first):
    """Whole blocks of keys at -inf before a query's first finite one: the finite ones' result; queries
    that see no finite key are not a number, as softmax of a row of -inf is."""
    print(f"\n[packed] {first} of {n} keys at -inf", flush=True)
    M = _lib()
    T, dh = torch.bfloat16 if prec else torch.float32, 64
    op = M.Attention(M.make_attn_desc(heads=1, kv_heads=1, head_dim=dh, precision=prec))
    whole, part = (M.mfmg_seq_plan(torch.tensor([0, m], dtype=torch.int32, device="cuda"), m)
                   for m in (n, n - first))
    gen = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn(n, dh, device="cuda", generator=gen).to(T) for _ in range(3))
    q[:, 0] = 1
    k[:first, 0] = float("-inf")
    o, o2 = torch.empty(n, dh, device="cuda", dtype=T), torch.empty(n - first, dh, device="cuda", dtype=T)
    op.mfmg_attn_fwd(whole, q, k, v, o, torch.empty(2, 1, n, device="cuda"))
    op.mfmg_attn_fwd(part, q[first:], k[first:], v[first:], o2, torch.empty(2, 1, n - first, device="cuda"))
    torch.cuda.synchronize()
    assert torch.isnan(o[:first]).all()
    # the same weights in other blocks: two roundings of each and of the result, float32 steps of the scores
    u, m = R.unit(T), n - first
    terms = (q[first:].double().abs() @ k[first:].double().abs().t()).amax(1, keepdim=True) * dh ** -0.5
    s = (q[first:].double() @ k[first:].double().t()) * dh ** -0.5
    p = torch.softmax(s.masked_fill(torch.ones_like(s).triu(1).bool(), float("-inf")), 1)
    a = p @ v[first:].double().abs()
    bound = 2 * u * o2.double().abs() + 2 * (u + 2 * R.E * ((dh + 8) * terms + n)) * a
    assert ((o[first:].double() - o2.double()).abs() <= bound).all()


@pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
def test_equal_scores_far_below_zero(prec):
    """Scores of -2^120 on every key: the mean of the values seen."""
    print("\n[packed] scores of -2^120", flush=True)
    M = _lib()
    n, dh, T = 50, 64, torch.bfloat16 if prec else torch.float32
    op = M.Attention(M.make_attn_desc(heads=1, kv_heads=1, head_dim=dh, precision=prec, scale=1.0))
    plan = M.mfmg_seq_plan(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    q, k = (torch.zeros(n, dh, device="cuda", dtype=T) for _ in range(2))
    q[:, 3], k[:, 3] = 2.0 ** 60, -2.0 ** 60
    v = torch.randn(n, dh, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(T)
    o = torch.empty(n, dh, device="cuda", dtype=T)
    op.mfmg_attn_fwd(plan, q, k, v, o, torch.empty(2, 1, n, device="cuda"))
    torch.cuda.synchronize()
    count = torch.arange(1, n + 1, device="cuda", dtype=torch.float64)[:, None]
    want, a = v.double().cumsum(0) / count, v.double().abs().cumsum(0) / count
    # (weights of 1 are exact) one rounding of the result, n + 4 float32 steps of the sums
    assert ((o.double() - want).abs() <= R.unit(T) * want.abs() + (n + 4) * R.E * a).all()
