"""The attention operators of this library, as cases to measure.

`family` names the operator: "rope" (rotary positions on the rows of a QKV product), "norm_rope"
(RMS norms of every query and key head with the rotation, in one pass) or "attn" (causal attention
over packed sequences with grouped heads).  `pass` is "fwd", "bwd" or "both"; `dual` adds the tangents
that ride through a forward-over-reverse pass, so that a dual "bwd" returns the gradients and their
derivatives along the tangent.  The layouts are those of include/mfmg.h: rows by token, q | k | v heads
side by side, tokens of several sequences behind one another, and rows behind the last sequence that
stay as they were (here: zero).
"""
import math
import random

import torch

own = False

FP32, BF16 = 0, 1
PLAIN, LINEAR, BASE, PARTS = 0, 1, 2, 3   # how rotary frequencies are stretched for long contexts


def _rows(family, heads, kv, dh, lens, **kw):
    """A case; `lens` is "AxB" (A sequences of B tokens), or "A:total:seed" (A ragged ones)."""
    case = {"family": family, "heads": heads, "kv": kv, "dh": dh, "lens": lens, "pad": 0, "prec": BF16,
            "pass": "both", "dual": False}
    if family != "attn":
        case.update(rope_dims=dh, interleaved=False, base=10000.0, scaling=PLAIN, factor=1.0, start=0)
    case.update(kw)
    return case


def listed():
    c = []

    def add(name, case):
        c.append({"name": name, **case})

    # One row of the small decoder (8 heads of 64, 256 tokens): only latency counts.
    add("rope_256", _rows("rope", 8, 8, 64, "1x256", **{"pass": "fwd"}))
    # A long-context continuation: half of every head rotated, pairs side by side, frequencies stretched
    # by parts, positions that begin far out, documents of odd lengths with unused rows behind them.
    add("rope_far", _rows("rope", 32, 8, 128, "37:16001:5", pad=383, rope_dims=64, interleaved=True,
                          base=500000.0, scaling=PARTS, factor=8.0, start=900000))
    # A Hessian-vector product's step through the norms of a packed batch: forward and backward, dual.
    add("norm_rope_dual", _rows("norm_rope", 16, 2, 128, "21:8191:7", dual=True))
    # The same rows of a small float32 model, head sizes that no power of two divides.
    add("norm_rope_fp32", _rows("norm_rope", 10, 5, 80, "3:999:9", prec=FP32, dual=True, rope_dims=40,
                                interleaved=True))
    # A training step of a wide model, 65536 tokens: what the memory can stream.
    add("norm_rope_65536", _rows("norm_rope", 32, 8, 128, "16x4096", scaling=LINEAR, factor=2.0))
    # A few short sequences, one token among them: latency again.
    add("attn_short", _rows("attn", 8, 8, 64, "5:137:3", **{"pass": "fwd"}))
    # The decoder's inner step: 16 sequences of 256 tokens, 8 heads of 64.
    add("attn_16x256", _rows("attn", 8, 8, 64, "16x256"))
    # The decoder's Hessian-vector product at a long context.
    add("attn_dual_2x4096", _rows("attn", 8, 8, 64, "2x4096", dual=True))
    # Training on packed documents, eight query heads for each key head.
    add("attn_packed", _rows("attn", 16, 2, 128, "40:16001:11", pad=383))
    # One long prompt, forward only.
    add("attn_prompt_16384", _rows("attn", 16, 2, 128, "1x16384", **{"pass": "fwd"}))
    # A Hessian-vector product over packed documents with heads of 128.
    add("attn_dual_packed", _rows("attn", 12, 4, 128, "9:8191:13", pad=1, dual=True))
    # Float32 operands, odd lengths, a head size that no tile has.
    add("attn_fp32", _rows("attn", 6, 3, 40, "4:1531:15", prec=FP32, dual=True))
    return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    family = rng.choice(["rope", "norm_rope", "attn", "attn"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 8] if kv <= 4 else [1, 2, 4])
    dh = rng.choice([16, 32, 40, 64, 64, 72, 96, 128, 128])
    prec = rng.choice([BF16, BF16, BF16, FP32])
    dual = rng.random() < 0.5
    kw = {"prec": prec, "dual": dual, "pass": rng.choice(["fwd", "bwd", "both", "both"]),
          "pad": rng.choice([0, 0, 1, rng.randrange(2, 200)])}
    if family == "attn":
        top = 4096 if prec == FP32 else 8192
        if kw["pass"] == "bwd":
            kw["pass"] = "both"   # the backward reads what the forward saved
    else:
        top = 16384
        kw.update(rope_dims=max(4, dh // rng.choice([1, 1, 2]) // 2 * 2), interleaved=rng.random() < 0.5,
                  base=rng.choice([10000.0, 500000.0]), start=rng.choice([0, 0, _log(rng, 10, 1000000)]))
        kw["scaling"] = rng.choice([PLAIN, LINEAR, BASE, PARTS])
        kw["factor"] = 1.0 if kw["scaling"] == PLAIN else rng.choice([2.0, 4.0, 8.0])
    total = _log(rng, 16, top)
    seed = rng.randrange(1 << 20)
    n = min(total, _log(rng, 1, 64))
    while True:
        case = _rows(family, heads, kv, dh, "%d:%d:%d" % (n, total, seed), **kw)
        if work(case)["flops"] <= (3e11 if prec == BF16 else 3e10):   # less than the largest listed ones
            return case
        total //= 2


def _lens(case):
    """Lengths of the case's sequences: equal ones, or a ragged cut whose parts differ widely."""
    s = case["lens"]
    if "x" in s:
        n, length = map(int, s.split("x"))
        return [length] * n
    n, total, seed = map(int, s.split(":"))
    rng = random.Random(seed)
    w = [rng.expovariate(1.0) + 1e-3 for _ in range(n)]
    lens = [1 + int((total - n) * x / sum(w)) for x in w]
    lens[rng.randrange(n)] += total - sum(lens)
    return lens


def _width(case):
    return (case["heads"] + 2 * case["kv"]) * case["dh"]


def _mscale(case):
    return 1.0 + 0.1 * math.log(case["factor"]) if case["scaling"] == PARTS else 1.0


TRAIN_LEN, SLOW, FAST = 8192.0, 1.0, 32.0   # what PARTS frequencies were trained on


def _desc(case):
    d = dict(heads=case["heads"], kv_heads=case["kv"], head_dim=case["dh"], precision=case["prec"])
    if case["family"] != "attn":
        d.update(qk_norm=case["family"] == "norm_rope", norm_eps=1e-6, rope_dims=case["rope_dims"],
                 rope_interleaved=case["interleaved"], rope_base=case["base"], rope_scaling=case["scaling"],
                 rope_factor=case["factor"], rope_train_len=TRAIN_LEN, rope_slow=SLOW, rope_fast=FAST,
                 rope_mscale=_mscale(case))
    return d


def prepare(case, seed):
    """Inputs on the GPU, the caller's output buffers, and the plan and handle that a program keeps."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lens(case)
    used = sum(lens)
    n, H, K, dh, W = used + case["pad"], case["heads"], case["kv"], case["dh"], _width(case)
    T = torch.bfloat16 if case["prec"] == BF16 else torch.float32
    dual, fwd, bwd = case["dual"], case["pass"] != "bwd", case["pass"] != "fwd"

    def rand(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g).mul_(scale).to(dtype)

    cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
    cu[1:] = torch.tensor(lens).cumsum(0)
    st = {"case": case, "lens": lens, "n": n, "used": used, "T": T, "cu": cu.cuda()}
    if case["family"] == "attn":
        # a QKV product's rows, whose heads the operator reads in place
        qkv = rand(n, W, scale=1.2, dtype=T)
        tan = rand(n, W, scale=0.3, dtype=T) if dual else None
        cut = (H * dh, K * dh, K * dh)
        st["qkv"] = qkv.split(cut, 1)
        st["tan"] = tan.split(cut, 1) if dual else (None,) * 3
        st["do"] = rand(n, H * dh, dtype=T) if bwd else None
        st["dod"] = rand(n, H * dh, scale=0.3, dtype=T) if bwd and dual else None
        outs = [("o", H * dh, T, True), ("od", H * dh, T, dual), ("dqkv", W, T, bwd),
                ("dqkvd", W, T, bwd and dual)]
    else:
        norm = case["family"] == "norm_rope"
        at = torch.cat([torch.arange(x) for x in lens] + [torch.zeros(case["pad"], dtype=torch.int64)])
        st["pos"] = (at + case["start"]).to(torch.int32).cuda()
        st["x"] = rand(n, W, scale=1.5)
        st["gain"] = 1.0 + rand(2, dh, scale=0.2) if norm else None
        st["xd"] = rand(n, W, scale=0.3) if dual else None
        st["gaind"] = rand(2, dh, scale=0.3) if norm and dual else None
        st["dy"] = rand(n, W, dtype=T) if bwd else None
        st["dyd"] = rand(n, W, scale=0.3, dtype=T) if bwd and dual else None
        outs = [("y", W, T, fwd), ("yd", W, T, fwd and dual), ("dx", W, T, bwd), ("dxd", W, T, bwd and dual)]
        if norm and bwd:
            st["dgain"] = torch.zeros(2, dh, device="cuda")
            st["dgaind"] = torch.zeros(2, dh, device="cuda") if dual else None
    for name, w, t, want in outs:
        st[name] = torch.zeros(n, w, device="cuda", dtype=t) if want else None
    if own:
        from paper_2505_00793_amd import _lib as M
        st["op"] = M.Attention(M.make_attn_desc(**_desc(case)))
        st["plan"] = M.mfmg_seq_plan(st["cu"], n, positions=st.get("pos"))
        if case["family"] == "attn":
            st["stats"] = torch.empty(2, H, n, device="cuda")
        st["ws"] = st["op"].workspace(n) if bwd else None
    return st


def run(state):
    if own:
        return _attn_own(state) if state["case"]["family"] == "attn" else _rope_own(state)
    return _attn_plain(state) if state["case"]["family"] == "attn" else _rope_plain(state)


# ------------------------------------------------------------------ the library's calls

def _rope_own(s):
    op, case, out = s["op"], s["case"], []
    if case["pass"] != "bwd":
        op.mfmg_qk_rope_fwd(s["plan"], s["x"], s["y"], gain=s["gain"], xd=s["xd"], gaind=s["gaind"], yd=s["yd"])
        out += [s["y"], s["yd"]]
    if case["pass"] != "fwd":
        norm = case["family"] == "norm_rope"
        op.mfmg_qk_rope_bwd(s["plan"], s["dy"], s["dx"], x=s["x"] if norm else None, gain=s["gain"],
                            dgain=s.get("dgain"), dyd=s["dyd"], dxd=s["dxd"], xd=s["xd"] if norm else None,
                            gaind=s["gaind"], dgaind=s.get("dgaind"), ws=s["ws"])
        out += [s["dx"], s["dxd"], s.get("dgain"), s.get("dgaind")]
    return [t for t in out if t is not None]


def _attn_own(s):
    op, case = s["op"], s["case"]
    H, K, dh = case["heads"], case["kv"], case["dh"]
    cut = (H * dh, K * dh, K * dh)
    q, k, v = s["qkv"]
    qd, kd, vd = s["tan"]
    op.mfmg_attn_fwd(s["plan"], q, k, v, s["o"], s["stats"], qd=qd, kd=kd, vd=vd, od=s["od"])
    out = [s["o"], s["od"]]
    if case["pass"] != "fwd":
        g = s["dqkv"].split(cut, 1)
        gd = s["dqkvd"].split(cut, 1) if case["dual"] else (None,) * 3
        op.mfmg_attn_bwd(s["plan"], q, k, v, s["o"], s["stats"], s["do"], *g, qd=qd, kd=kd, vd=vd, od=s["od"],
                         dod=s["dod"], dqd=gd[0], dkd=gd[1], dvd=gd[2], ws=s["ws"])
        out += [s["dqkv"], s["dqkvd"]]
    return [t for t in out if t is not None]


# ------------------------------------------------------------------ plain form: rotation and norms

def _freqs(case, device):
    D = case["rope_dims"]
    base = case["base"]
    if case["scaling"] == BASE:
        base = base * case["factor"] ** (D / (D - 2))
    j = torch.arange(0, D, 2, dtype=torch.float64, device=device)
    f = torch.exp(-j / D * math.log(base))
    if case["scaling"] == LINEAR:
        f = f / case["factor"]
    if case["scaling"] == PARTS:
        keep = ((TRAIN_LEN * f / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0.0, 1.0)
        f = f * ((1.0 - keep) / case["factor"] + keep)
    return f


def _rope_plain(s):
    case, n, used = s["case"], s["n"], s["used"]
    H, K, dh, D, dual = case["heads"], case["kv"], case["dh"], case["rope_dims"], case["dual"]
    norm = case["family"] == "norm_rope"
    M = H + K
    angle = s["pos"][:used].double()[:, None] * _freqs(case, s["pos"].device)
    cos, sin = ((f(angle) * _mscale(case)).float()[:, None, :] for f in (torch.cos, torch.sin))

    def rot(t, back=False):
        """The rotated dims of t [tokens][heads][dh], or their rotation back."""
        a, b = (t[..., 0:D:2], t[..., 1:D:2]) if case["interleaved"] else (t[..., :D // 2], t[..., D // 2:D])
        si = -sin if back else sin
        u, v = a * cos - b * si, a * si + b * cos
        r = torch.stack((u, v), -1).flatten(-2) if case["interleaved"] else torch.cat((u, v), -1)
        return torch.cat((r, t[..., D:]), -1)

    def heads(t):
        t = t[:used].float().view(used, H + 2 * K, dh)
        return t[:, :M], t[:, M:]

    def rows(t, v, dtype):
        r = torch.zeros(n, _width(case), device=t.device, dtype=dtype)
        r[:used] = torch.cat((t, v), 1).reshape(used, -1).to(dtype)
        return r

    if norm:
        g = torch.cat((s["gain"][0].expand(H, dh), s["gain"][1].expand(K, dh)))
        x, xv = heads(s["x"])
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        xh = x * r
        if dual:
            gd = torch.cat((s["gaind"][0].expand(H, dh), s["gaind"][1].expand(K, dh)))
            xd, xdv = heads(s["xd"])
            c = (xh * xd).mean(-1, keepdim=True)
            xhd = r * (xd - c * xh)
    out = []
    if case["pass"] != "bwd":
        if not norm:
            x, xv = heads(s["x"])
        out.append(rows(rot(g * xh if norm else x), xv, s["T"]))
        if dual:
            if not norm:
                xd, xdv = heads(s["xd"])
            out.append(rows(rot(gd * xh + g * xhd if norm else xd), xdv, s["T"]))
    if case["pass"] != "fwd":
        dy, dyv = heads(s["dy"])
        dy = rot(dy, True)
        if dual:
            dyd, dydv = heads(s["dyd"])
            dyd = rot(dyd, True)
        if not norm:
            out.append(rows(dy, dyv, s["T"]))
            if dual:
                out.append(rows(dyd, dydv, s["T"]))
        else:
            def by_kind(t):
                t = t.double().sum(0)
                return torch.stack((t[:H].sum(0), t[H:].sum(0))).float()

            e = g * dy
            m = (xh * e).mean(-1, keepdim=True)
            out.append(rows(r * (e - xh * m), dyv, s["T"]))
            if dual:
                ed = gd * dy + g * dyd
                md = (xhd * e + xh * ed).mean(-1, keepdim=True)
                out.append(rows(-r * r * c * (e - xh * m) + r * (ed - xhd * m - xh * md), dydv, s["T"]))
            out.append(by_kind(dy * xh))
            if dual:
                out.append(by_kind(dyd * xh + dy * xhd))
    return out


# ------------------------------------------------------------------ plain form: attention

def _attn_plain(s):
    case, n, T = s["case"], s["n"], s["T"]
    H, K, dh, dual = case["heads"], case["kv"], case["dh"], case["dual"]
    bwd = case["pass"] != "fwd"
    G, sc = H // K, 1.0 / math.sqrt(dh)
    dev = s["cu"].device
    o = torch.zeros(n, H, dh, device=dev, dtype=T)
    od = torch.zeros_like(o) if dual else None
    g = torch.zeros(n, H + 2 * K, dh, device=dev, dtype=T) if bwd else None
    gd = torch.zeros_like(g) if bwd and dual else None
    lo = 0
    for L in s["lens"]:
        hi = lo + L
        step = max(1, min(K, (1 << 28) // (L * L * G)))   # key heads whose score matrices are held at once
        hidden = torch.ones(L, L, dtype=torch.bool, device=dev).triu(1)
        for k0 in range(0, K, step):
            k1 = min(K, k0 + step)

            def kv(t):   # [k1 - k0][1][L][dh]
                return t[lo:hi].float().view(L, K, dh)[:, k0:k1].permute(1, 0, 2).unsqueeze(1).contiguous()

            def qh(t):   # [k1 - k0][G][L][dh]
                return t[lo:hi].float().view(L, K, G, dh)[:, k0:k1].permute(1, 2, 0, 3).contiguous()

            def put(dst, t):
                dst[lo:hi, k0 * G:k1 * G] = t.permute(2, 0, 1, 3).reshape(L, -1, dh).to(T)

            def put_kv(dst, first, t):
                dst[lo:hi, first + k0:first + k1] = t.sum(1).permute(1, 0, 2).to(T)

            def nt(a, b):
                return torch.matmul(a, b.transpose(-1, -2).contiguous())

            def tn(a, b):
                return torch.matmul(a.transpose(-1, -2).contiguous(), b)

            q, k, v = qh(s["qkv"][0]), kv(s["qkv"][1]), kv(s["qkv"][2])
            S = (nt(q, k) * sc).masked_fill_(hidden, -math.inf)
            P = torch.exp(S - S.amax(-1, keepdim=True))
            P /= P.sum(-1, keepdim=True)
            O = torch.matmul(P, v)
            put(o, O)
            if dual:
                qd, kd, vd = qh(s["tan"][0]), kv(s["tan"][1]), kv(s["tan"][2])
                Sd = (nt(qd, k) + nt(q, kd)) * sc
                Pd = P * (Sd - (P * Sd).sum(-1, keepdim=True))
                put(od, torch.matmul(Pd, v) + torch.matmul(P, vd))
            if not bwd:
                continue
            do = qh(s["do"])
            dP = nt(do, v)
            A = dP - (P * dP).sum(-1, keepdim=True)
            dS = sc * P * A
            put(g, torch.matmul(dS, k))
            put_kv(g, H, tn(dS, q))
            put_kv(g, H + K, tn(P, do))
            if dual:
                dod = qh(s["dod"])
                dPd = nt(dod, v) + nt(do, vd)
                dSd = sc * (Pd * A + P * (dPd - (Pd * dP + P * dPd).sum(-1, keepdim=True)))
                put(gd, torch.matmul(dSd, k) + torch.matmul(dS, kd))
                put_kv(gd, H, tn(dSd, q) + tn(dS, qd))
                put_kv(gd, H + K, tn(Pd, do) + tn(P, dod))
        lo = hi
    return [t.view(n, -1) for t in (o, od, g, gd) if t is not None]


# ------------------------------------------------------------------ work and exact values

def work(case):
    """Every input read once, every output written once; products of visible pairs only."""
    lens = _lens(case)
    used, W, e = sum(lens), _width(case), 2 if case["prec"] == BF16 else 4
    two = 2 if case["dual"] else 1
    fwd, bwd = case["pass"] != "bwd", case["pass"] != "fwd"
    if case["family"] == "attn":
        QO = case["heads"] * case["dh"]
        pairs = sum(x * (x + 1) // 2 for x in lens)
        products = (6 if case["dual"] else 2) + ((15 if case["dual"] else 5) if bwd else 0)
        size = used * e * two * (W + QO + (QO + W if bwd else 0))
        return {"bytes": size, "flops": 2 * products * pairs * case["heads"] * case["dh"]}
    norm = case["family"] == "norm_rope"
    size, flops = 0, 0
    if fwd or norm:
        size += used * W * 4 * two if fwd else used * (W - case["kv"] * case["dh"]) * 4 * two
    if fwd:
        size += used * W * e * two
    if bwd:
        size += 2 * used * W * e * two
    flops = used * W * two * ((10 if norm else 3) * (fwd + 2 * bwd))
    return {"bytes": size, "flops": flops}


def exact(case, seed):
    """The definition in float64: automatic differentiation of one rotated and normalised head, and of
    one sequence's attention, forwards (for tangents) over backwards (for gradients)."""
    s = prepare(case, seed)
    return _attn_exact(s) if case["family"] == "attn" else _rope_exact(s)


def _through(f, x, xd, dy, dyd, case):
    """[y, yd, dx..., dxd...] as the case has them, of y = f(*x) with cotangent dy."""
    from torch.func import jvp, vjp
    fwd, bwd, dual = case["pass"] != "bwd", case["pass"] != "fwd", case["dual"]
    y = yd = gx = gxd = None
    if fwd:
        y, yd = jvp(f, x, xd) if dual else (f(*x), None)
    if bwd:
        def grads(*a):
            return vjp(f, *a[:-1])[1](a[-1])
        gx, gxd = jvp(grads, (*x, dy), (*xd, dyd)) if dual else (grads(*x, dy), None)
    return y, yd, gx, gxd


def _rope_exact(s):
    case, n, used = s["case"], s["n"], s["used"]
    H, K, dh, D, dual = case["heads"], case["kv"], case["dh"], case["rope_dims"], case["dual"]
    norm, dev = case["family"] == "norm_rope", s["cu"].device
    th = []
    for j in range(D // 2):
        f = case["base"] ** (-2.0 * j / D)
        if case["scaling"] == LINEAR:
            f /= case["factor"]
        elif case["scaling"] == BASE:
            f = (case["base"] * case["factor"] ** (D / (D - 2.0))) ** (-2.0 * j / D)
        elif case["scaling"] == PARTS:
            turns = TRAIN_LEN * f / (2.0 * math.pi)
            w = min(1.0, max(0.0, (turns - SLOW) / (FAST - SLOW)))
            f = w * f + (1.0 - w) * f / case["factor"]
        th.append(f)
    th = torch.tensor(th, dtype=torch.float64, device=dev)
    first = torch.arange(0, D, 2, device=dev) if case["interleaved"] else torch.arange(D // 2, device=dev)
    second = first + (1 if case["interleaved"] else D // 2)

    def f(x, gain, ang):
        """x [tokens][heads][dh] of one kind of head."""
        if norm:
            x = gain * x / torch.sqrt(x.square().sum(-1, keepdim=True) / dh + 1e-6)
        c, si = torch.cos(ang)[:, None] * _mscale(case), torch.sin(ang)[:, None] * _mscale(case)
        a, b = x.index_select(2, first), x.index_select(2, second)
        y = x.index_copy(2, first, a * c - b * si)
        return y.index_copy(2, second, b * c + a * si)

    W = (H + 2 * K) * dh
    res = {}
    keys = [k for k in ("y", "yd", "dx", "dxd") if s[k] is not None]
    for k in keys:
        res[k] = torch.zeros(n, W, dtype=torch.float64, device=dev)
    gains = {k: torch.zeros(2, dh, dtype=torch.float64, device=dev) for k in ("dgain", "dgaind")
             if s.get(k) is not None}
    for lo in range(0, used, 4096):
        hi = min(used, lo + 4096)
        ang = s["pos"][lo:hi].double()[:, None] * th

        def part(name, a, b):
            return s[name][lo:hi, a * dh:b * dh].double().view(hi - lo, b - a, dh) if s[name] is not None else None
        for kind, (a, b) in enumerate(((0, H), (H, H + K))):
            gain = s["gain"][kind].double() if norm else torch.ones(dh, dtype=torch.float64, device=dev)
            gaind = s["gaind"][kind].double() if norm and dual else torch.zeros_like(gain)
            y, yd, gx, gxd = _through(lambda u, w: f(u, w, ang), (part("x", a, b), gain),
                                      (part("xd", a, b), gaind), part("dy", a, b), part("dyd", a, b), case)
            for key, val in (("y", y), ("yd", yd), ("dx", gx and gx[0]), ("dxd", gxd and gxd[0])):
                if key in res:
                    res[key][lo:hi, a * dh:b * dh] = val.reshape(hi - lo, -1)
            for key, val in (("dgain", gx), ("dgaind", gxd)):
                if key in gains:
                    gains[key][kind] += val[1]
        for key, src in (("y", "x"), ("yd", "xd"), ("dx", "dy"), ("dxd", "dyd")):
            if key in res:
                res[key][lo:hi, (H + K) * dh:] = s[src][lo:hi, (H + K) * dh:].double()
    return [res[k] for k in keys] + [gains[k] for k in ("dgain", "dgaind") if k in gains]


def _attn_exact(s):
    case, n, dev = s["case"], s["n"], s["cu"].device
    H, K, dh, dual = case["heads"], case["kv"], case["dh"], case["dual"]
    G = H // K
    W = (H + 2 * K) * dh
    o, od, g, gd = (torch.zeros(n, w, dtype=torch.float64, device=dev) if s[k] is not None else None
                    for k, w in (("o", H * dh), ("od", H * dh), ("dqkv", W), ("dqkvd", W)))
    lo = 0
    for L in s["lens"]:
        hi = lo + L
        seen = torch.arange(L, device=dev)[:, None] >= torch.arange(L, device=dev)

        def f(q, k, v):   # [heads][L][dh]
            w = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(dh)
            w = torch.softmax(torch.where(seen, w, torch.full_like(w, -math.inf)), -1)
            return torch.matmul(w, v)

        step = max(1, min(H, (1 << 27) // (L * L)))
        step = step // G * G if step >= G else 1
        for h0 in range(0, H, step):
            hs = list(range(h0, min(H, h0 + step)))

            def pick(t, idx):
                return t[lo:hi].double().view(L, -1, dh)[:, idx].transpose(0, 1).contiguous() if t is not None else None

            ks = [h // G for h in hs]
            x = tuple(pick(t, i) for t, i in zip(s["qkv"], (hs, ks, ks)))
            xd = tuple(pick(t, i) for t, i in zip(s["tan"], (hs, ks, ks)))
            y, yd, gx, gxd = _through(f, x, xd, pick(s["do"], hs), pick(s["dod"], hs), case)
            for dst, val in ((o, y), (od, yd)):
                if dst is not None:
                    dst.view(n, H, dh)[lo:hi, hs] = val.transpose(0, 1)
            for dst, val in ((g, gx), (gd, gxd)):
                if dst is not None:
                    d3 = dst.view(n, H + 2 * K, dh)
                    d3[lo:hi, hs] = val[0].transpose(0, 1)
                    for i, kh in enumerate(ks):
                        d3[lo:hi, H + kh] += val[1][i]
                        d3[lo:hi, H + K + kh] += val[2][i]
        lo = hi
    return [t for t in (o, od, g, gd) if t is not None]
