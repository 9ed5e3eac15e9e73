"""Plain float64 forms of the attention operators, with elementwise bounds of what float32 sums and
one rounding to the operand type may be off by.

u is half a step of the operand type, e = 2^-24 that of float32.  A bound is a first-order one: every
rounded factor contributes its unit times the sum of the absolute products it enters; a float32 sum
of n terms contributes n e times their absolute sum.
"""
import math

import torch

E = 2.0 ** -24


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def _mm(a, b):
    return torch.matmul(a, b)


def _t(a):
    return a.transpose(-1, -2).contiguous()


def attention(q, k, v, lens, scale, dtype, tan=None, g=None, gd=None, first=0):
    """q [n][H][dh], k and v [n][K][dh] in float64 (tan: their tangents), g the cotangent of o (gd its
    tangent); sequences of `lens` tokens from token `first`.  Returns {name: (value, bound)} of o, od,
    dq, dk, dv, dqd, dkd, dvd; rows of no sequence are zero."""
    H, K, dh = q.shape[1], k.shape[1], q.shape[2]
    G, u = H // K, unit(dtype)
    dual = tan is not None
    names = ["o"] + (["od"] if dual else [])
    if g is not None:
        names += ["dq", "dk", "dv"] + (["dqd", "dkd", "dvd"] if dual else [])
    out = {x: tuple(torch.zeros_like(k if x[1:2] in ("k", "v") else q) for _ in range(2)) for x in names}
    lo = first
    for L in lens:
        sl = slice(lo, lo + L)
        lo += L
        if L == 0:
            continue
        vis = torch.tril(torch.ones(L, L, dtype=torch.bool, device=q.device))

        def put(name, h, val, bound):
            out[name][0][sl, h] += val
            out[name][1][sl, h] += bound

        for h in range(H):
            kh = h // G
            Q, Kk, V = q[sl, h], k[sl, kh], v[sl, kh]
            n = (L + 16) * E             # a float32 sum over the tokens, and what is done to its result
            gam = (dh + 4) * E
            S = scale * _mm(Q, _t(Kk))
            aS = scale * _mm(Q.abs(), _t(Kk.abs()))
            P = torch.softmax(torch.where(vis, S, torch.full_like(S, -math.inf)), -1)
            # relative error of P: the scores' own, the steps of exp2, log2 and their arguments
            eP = 2 * gam * aS.amax() + 8 * E * (1 + aS.amax()) + 8 * E + n
            kP = u + eP + n              # of P as an operand of a product over the tokens
            O = _mm(P, V)
            aO = _mm(P, V.abs())
            dO_ = kP * aO
            put("o", h, O, dO_ + u * O.abs())
            if dual:
                Qd, Kd, Vd = tan[0][sl, h], tan[1][sl, kh], tan[2][sl, kh]
                Sd = scale * (_mm(Qd, _t(Kk)) + _mm(Q, _t(Kd)))
                aSd = scale * (_mm(Qd.abs(), _t(Kk.abs())) + _mm(Q.abs(), _t(Kd.abs())))
                eSd = 2 * gam * aSd
                c = (P * Sd).sum(-1, keepdim=True)
                ac = (P * Sd.abs()).sum(-1, keepdim=True)
                ec = (P * eSd).sum(-1, keepdim=True) + (eP + n) * ac
                Pd = P * (Sd - c)
                ePd = eP * Pd.abs() + P * (eSd + ec + 4 * E * (Sd.abs() + ac))
                Od = _mm(Pd, V) + _mm(P, Vd)
                dOd_ = (kP * (_mm(P * Sd.abs(), V.abs()) + _mm(P, Vd.abs()) + c.abs() * aO)
                        + _mm(P * eSd, V.abs()) + ec * aO)
                put("od", h, Od, dOd_ + u * Od.abs())
            if g is None:
                continue
            g_ = g[sl, h]
            dP = _mm(g_, _t(V))
            edP = gam * _mm(g_.abs(), _t(V.abs()))
            # r is taken from o as stored
            r = (P * dP).sum(-1, keepdim=True)
            er = (g_.abs() * (dO_ + (u + gam) * O.abs())).sum(-1, keepdim=True)
            A = dP - r
            eA = edP + er + 4 * E * (dP.abs() + r.abs())
            dS = scale * P * A
            edS = scale * (P * eA + eP * P * A.abs()) + (u + n) * dS.abs() + 2 * E * dS.abs()
            val = _mm(dS, Kk)
            put("dq", h, val, _mm(edS, Kk.abs()) + u * val.abs())
            val = _mm(_t(dS), Q)
            put("dk", kh, val, _mm(_t(edS), Q.abs()))
            val = _mm(_t(P), g_)
            put("dv", kh, val, kP * _mm(_t(P), g_.abs()))
            if not dual:
                continue
            gd_ = gd[sl, h]
            dPd = _mm(gd_, _t(V)) + _mm(g_, _t(Vd))
            edPd = 2 * gam * (_mm(gd_.abs(), _t(V.abs())) + _mm(g_.abs(), _t(Vd.abs())))
            rd = (Pd * dP + P * dPd).sum(-1, keepdim=True)
            erd = (gd_.abs() * (dO_ + (u + 2 * gam) * O.abs())
                   + g_.abs() * (dOd_ + (u + 2 * gam) * Od.abs())).sum(-1, keepdim=True)
            B = dPd - rd
            eB = edPd + erd + 4 * E * (dPd.abs() + rd.abs())
            dSd = scale * (Pd * A + P * B)
            edSd = (scale * (ePd * A.abs() + Pd.abs() * eA + P * eB + eP * P * B.abs()
                             + 4 * E * (Pd.abs() * A.abs() + P * B.abs()))
                    + (u + n) * dSd.abs())
            val = _mm(dSd, Kk) + _mm(dS, Kd)
            put("dqd", h, val, _mm(edSd, Kk.abs()) + _mm(edS, Kd.abs()) + n * (_mm(dSd.abs(), Kk.abs()) + _mm(dS.abs(), Kd.abs())) + u * val.abs())
            val = _mm(_t(dSd), Q) + _mm(_t(dS), Qd)
            put("dkd", kh, val, _mm(_t(edSd), Q.abs()) + _mm(_t(edS), Qd.abs())
                + n * (_mm(_t(dSd.abs()), Q.abs()) + _mm(_t(dS.abs()), Qd.abs())))
            val = _mm(_t(Pd), g_) + _mm(_t(P), gd_)
            put("dvd", kh, val, _mm(_t(ePd + (u + n) * Pd.abs()), g_.abs()) + kP * _mm(_t(P), gd_.abs())
                + n * (_mm(_t(Pd.abs()), g_.abs()) + _mm(_t(P), gd_.abs())))
    for x in ("dk", "dv", "dkd", "dvd"):
        if x in out:   # their one rounding, and the float32 sum over the group
            out[x] = (out[x][0], out[x][1] * (1 + G * E) + (u + G * E) * out[x][0].abs())
    return out


def frequencies(dims, base=10000.0, scaling=0, factor=1.0, train_len=0.0, slow=1.0, fast=32.0):
    j = torch.arange(0, dims, 2, dtype=torch.float64)
    if scaling == 2:
        base = base * factor ** (dims / (dims - 2))
    f = base ** (-j / dims)
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        w = ((train_len * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * ((1 - w) / factor + w)
    return f


class Rope:
    """The rotation and norms of q | k | v rows in float64, with gradients and tangents; `absolute`
    gives the sums of the absolute terms instead, which bounds are units of."""

    def __init__(self, H, K, dh, pos, dims, interleaved, mscale, freqs, eps=None, absolute=False):
        self.H, self.K, self.dh, self.D, self.inter, self.eps = H, K, dh, dims, interleaved, eps
        ang = pos.double()[:, None] * freqs.to(pos.device)
        self.c, self.s = torch.cos(ang)[:, None] * mscale, torch.sin(ang)[:, None] * mscale
        self.ab = absolute
        if absolute:
            self.c, self.s = self.c.abs(), self.s.abs()

    def rot(self, t, back=False):
        D = self.D
        a, b = (t[..., 0:D:2], t[..., 1:D:2]) if self.inter else (t[..., :D // 2], t[..., D // 2:D])
        s = -self.s if back else self.s
        if self.ab:
            u, v = a * self.c + b * self.s, a * self.s + b * self.c
        else:
            u, v = a * self.c - b * s, a * s + b * self.c
        r = torch.stack((u, v), -1).flatten(-2) if self.inter else torch.cat((u, v), -1)
        return torch.cat((r, t[..., D:]), -1)

    def run(self, x, gain=None, xd=None, gaind=None, dy=None, dyd=None):
        """Rows [n][(H + 2K) dh]; {name: value} of y, yd, dx, dxd, dgain, dgaind."""
        H, K, dh, M = self.H, self.K, self.dh, self.H + self.K
        n = (x if x is not None else dy).shape[0]
        ab = self.ab
        A = (lambda t: None if t is None else t.abs()) if ab else (lambda t: t)
        sub = (lambda p, q: p + q) if ab else (lambda p, q: p - q)

        def heads(t):
            return None if t is None else A(t.view(n, H + 2 * K, dh))[:, :M]

        def row(t, v):
            return torch.cat((t, A(v.view(n, H + 2 * K, dh))[:, M:]), 1).reshape(n, -1)
        res = {}
        dual = xd is not None or dyd is not None
        if gain is not None:
            rep = lambda t: None if t is None else torch.cat((A(t)[0].expand(H, dh), A(t)[1].expand(K, dh)))
            g, gd = rep(gain), rep(gaind)
            X, Xd = heads(x), heads(xd)
            r = 1 / torch.sqrt((X * X).mean(-1, keepdim=True) + self.eps)
            xh = r * X
            if dual:
                c = (xh * Xd).mean(-1, keepdim=True)
                xhd = r * sub(Xd, c * xh)
        if x is not None:
            X, Xd = heads(x), heads(xd)
            res["y"] = row(self.rot(g * xh if gain is not None else X), x)
            if xd is not None:
                res["yd"] = row(self.rot(gd * xh + g * xhd if gain is not None else Xd), xd)
        if dy is None:
            return res
        v, vd = self.rot(heads(dy), True), None
        if dual:
            vd = self.rot(heads(dyd), True)
        if gain is None:
            res["dx"] = row(v, dy)
            if dual:
                res["dxd"] = row(vd, dyd)
            return res
        kinds = lambda t: torch.stack((t[:, :H].sum((0, 1)), t[:, H:].sum((0, 1))))
        e = g * v
        m = (xh * e).mean(-1, keepdim=True)
        u = sub(e, xh * m)
        res["dx"] = row(r * u, dy)
        res["dgain"] = kinds(v * xh)
        if dual:
            ed = gd * v + g * vd
            md = (xhd * e + xh * ed).mean(-1, keepdim=True)
            w = sub(sub(ed, xhd * m), xh * md)
            res["dxd"] = row((r * r * c * u if ab else -r * r * c * u) + r * w, dyd)
            res["dgaind"] = kinds(vd * xh + v * xhd)
        return res
