"""The decoder problem of include/mfmg.h with its attention options, in float64 torch: losses by the
definition, gradients and meta-gradients by automatic differentiation."""
import dataclasses
import math

import torch

import packed_ref as R


@dataclasses.dataclass
class Decoder:
    d: int = 64
    H: int = 4
    K: int = 2
    F: int = 96
    V: int = 50
    S: int = 20
    L: int = 2
    hidden: int = 8
    rows: int = 3
    val_rows: int = 2
    prec: int = 0
    lr: float = 0.2
    eps: float = 1e-5
    base: float = 10000.0
    norm: int = 1
    rope: dict = dataclasses.field(default_factory=dict)   # rope_* fields of the description
    docs: tuple = ()        # offsets of a training batch's documents (one tuple per step), or none
    val_docs: tuple = ()
    remat: int = 0
    T: int = 2
    fused: int = 1

    def desc(self):
        from paper_2505_00793_amd import _lib as M
        return M.make_desc(kind=1, widths=(1, 1), loss=1, optimizer=0, meta=3, precision=self.prec,
                           has_bias=False, rows=self.rows, val_rows=self.val_rows, sgd_lr=self.lr,
                           d_model=self.d, n_heads=self.H, d_ff=self.F, vocab=self.V, seq=self.S,
                           n_blocks=self.L, meta_hidden=self.hidden, ln_eps=self.eps,
                           rope_base=self.base, fused_attention=self.fused, block_remat=self.remat,
                           n_kv_heads=self.K, qk_norm=self.norm,
                           docs=len(self.docs[0]) - 1 if self.docs else 0,
                           val_docs=len(self.val_docs) - 1 if self.val_docs else 0, **self.rope)

    def shapes(self):
        dh, QC = self.d // self.H, (self.H + 2 * self.K) * (self.d // self.H)
        s = [("E", (self.V, self.d))]
        for b in range(self.L):
            s += [(f"g1{b}", (self.d,)), (f"b1{b}", (self.d,)), (f"qkv{b}", (self.d, QC))]
            if self.norm:
                s += [(f"qk{b}", (2, dh))]
            s += [(f"o{b}", (self.d, self.d)), (f"g2{b}", (self.d,)), (f"b2{b}", (self.d,)),
                  (f"w1{b}", (self.d, self.F)), (f"w2{b}", (self.F, self.d))]
        return s + [("gf", (self.d,)), ("bf", (self.d,)), ("U", (self.d, self.V))]

    def draw(self, seed=0):
        """theta, eta (float32 on the CPU), training and validation tokens."""
        g = torch.Generator().manual_seed(seed)
        parts = []
        for name, shape in self.shapes():
            t = torch.randn(shape, generator=g)
            if name[0] in "gb" or name[:2] == "qk" and name[2] != "v":
                t = 0.2 * t + (0.0 if name[0] == "b" else 1.0)
            elif name == "E":
                t = 0.7 * t
            else:
                t = t / math.sqrt(shape[0])
            parts.append(t.flatten())
        n_eta = self.d * self.hidden + 2 * self.hidden + 1
        eta = 0.3 * torch.randn(n_eta, generator=g)
        xs = [torch.randint(self.V, (self.rows, self.S + 1), generator=g, dtype=torch.int32)
              for _ in range(self.T)]
        vx = torch.randint(self.V, (self.val_rows, self.S + 1), generator=g, dtype=torch.int32)
        return torch.cat(parts), eta, xs, vx

    def lens(self, docs, rows):
        n = rows * self.S
        if not docs:
            return [self.S] * rows
        b = [0]
        for c in (*docs, n):
            b.append(max(b[-1], min(max(c, 0), n)))
        return [y - x for x, y in zip(b, b[1:])]

    def row_losses(self, theta, tokens, lens):
        """Cross-entropy of every loss row (b * S + s)."""
        P, off = {}, 0
        for name, shape in self.shapes():
            P[name] = theta[off:off + math.prod(shape)].view(shape)
            off += math.prod(shape)
        H, K, d = self.H, self.K, self.d
        dh = d // H
        tokens = tokens.long()
        N = tokens.shape[0] * self.S
        h = P["E"][tokens[:, :-1].reshape(-1)]
        o = dict(rope_dims=0, rope_interleaved=0, rope_scaling=0, rope_factor=1.0, rope_train_len=0.0,
                 rope_slow=1.0, rope_fast=32.0, rope_mscale=0.0)
        o.update(self.rope)
        D = o["rope_dims"] or dh
        fr = R.frequencies(D, self.base, o["rope_scaling"], o["rope_factor"], o["rope_train_len"],
                           o["rope_slow"], o["rope_fast"])
        pos = torch.cat([torch.arange(x) for x in lens])
        ang = pos.double()[:, None] * fr
        ms = o["rope_mscale"] or 1.0
        c, s = ms * torch.cos(ang)[:, None], ms * torch.sin(ang)[:, None]

        def ln(x, g, b):
            m = x.mean(-1, keepdim=True)
            return (x - m) / torch.sqrt((x - m).square().mean(-1, keepdim=True) + self.eps) * g + b

        for b in range(self.L):
            t = (ln(h, P[f"g1{b}"], P[f"b1{b}"]) @ P[f"qkv{b}"]).view(N, H + 2 * K, dh)
            qk, v = t[:, :H + K], t[:, H + K:]
            if self.norm:
                gain = torch.cat((P[f"qk{b}"][0].expand(H, dh), P[f"qk{b}"][1].expand(K, dh)))
                qk = gain * qk / torch.sqrt(qk.square().mean(-1, keepdim=True) + self.eps)
            if o["rope_interleaved"]:
                x, y = qk[..., 0:D:2], qk[..., 1:D:2]
                r = torch.stack((x * c - y * s, x * s + y * c), -1).flatten(-2)
            else:
                x, y = qk[..., :D // 2], qk[..., D // 2:D]
                r = torch.cat((x * c - y * s, x * s + y * c), -1)
            qk = torch.cat((r, qk[..., D:]), -1)
            q, k = qk[:, :H], qk[:, H:].repeat_interleave(H // K, 1)
            v = v.repeat_interleave(H // K, 1)
            out, lo = [], 0
            for n in lens:
                w = torch.einsum("qhd,khd->hqk", q[lo:lo + n], k[lo:lo + n]) / math.sqrt(dh)
                w = w.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf).softmax(-1)
                out.append(torch.einsum("hqk,khd->qhd", w, v[lo:lo + n]).reshape(n, d))
                lo += n
            h = h + torch.cat(out) @ P[f"o{b}"]
            z = ln(h, P[f"g2{b}"], P[f"b2{b}"]) @ P[f"w1{b}"]
            h = h + torch.nn.functional.gelu(z) @ P[f"w2{b}"]
        logits = ln(h, P["gf"], P["bf"]) @ P["U"]
        return torch.nn.functional.cross_entropy(logits, tokens[:, 1:].reshape(-1), reduction="none")

    def alpha(self, eta, E, tokens):
        d, m = self.d, self.hidden
        W1, b1, w2, b2 = eta[:d * m].view(d, m), eta[d * m:d * m + m], eta[d * m + m:d * m + 2 * m], eta[-1]
        e = E[tokens[:, :-1].reshape(-1).long()]
        return torch.sigmoid(torch.tanh(e @ W1 + b1) @ w2 + b2)

    def loss(self, theta, eta, E, tokens, t):
        lens = self.lens(self.docs[t] if self.docs else (), self.rows)
        return (self.alpha(eta, E, tokens) * self.row_losses(theta, tokens, lens)).mean()

    def meta_grad(self, theta, eta, xs, vx):
        """(d eta, V) in float64."""
        eta = eta.double().requires_grad_()
        th = theta.double().requires_grad_()
        E = theta[:self.V * self.d].double().view(self.V, self.d)
        for t, x in enumerate(xs):
            g, = torch.autograd.grad(self.loss(th, eta, E, x, t), th, create_graph=True)
            th = th - self.lr * g
        V = self.row_losses(th, vx, self.lens(self.val_docs, self.val_rows)).mean()
        return torch.autograd.grad(V, eta)[0], V.detach()

    def hvp(self, theta, eta, x, v, t=0):
        """(gradient, H v, <grad l_n, v> / N) in float64."""
        th = theta.double().requires_grad_()
        E = theta[:self.V * self.d].double().view(self.V, self.d)
        g, = torch.autograd.grad(self.loss(th, eta.double(), E, x, t), th, create_graph=True)
        Hv, = torch.autograd.grad(g, th, v.double())
        lens = self.lens(self.docs[t] if self.docs else (), self.rows)
        _, mv = torch.func.jvp(lambda p: self.row_losses(p, x, lens), (theta.double(),), (v.double(),))
        return g.detach(), Hv, mv / mv.numel()
