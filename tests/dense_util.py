"""Attention of N queries to M keys in 64 bits, forward and backward, with a bound for what the kernels may be off, entry by entry.

The bounds count roundings.  u: half a step of the stored type, relative (bfloat16 2^-8, float32 2^-24); e = 2^-24.  A score is a sum of
d exact (bfloat16) or rounded products in float32 and a few more operations: off by at most D_i = (d + 4) e max_j scale sum|q k|
+ 4 e max|x|, plus 2^-21 for the exponential and its argument's scaling.  So each probability, forward (against the sum of all) or from
lse, is off by a factor of at most 1 + 4 D_i =: 1 + t_i, and where it enters a product in the stored type by u more.  Sums of n terms in float32:
n e of the sum of magnitudes, at worst.
"""
from __future__ import annotations

import math

import torch

from paper_2505_14708_amd import binding as da

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": da.DA_F32, "bf16": da.DA_BF16}


def bucket(r, buckets, max_distance, bidirectional):
    """The bucket of r in integers."""
    n = buckets // 2 if bidirectional else buckets
    e, base = n // 2, n if bidirectional and r > 0 else 0
    a = abs(r) if bidirectional else max(-r, 0)
    if a < e:
        return base + a
    return base + e + sum(a ** (n - e) >= e ** (n - e - k) * max_distance ** k for k in range(1, n - e))


def bucket_map(N, M, rule):
    buckets, max_distance, bidirectional, q_pos = rule
    cut = max_distance + 1                                      # one bucket from max_distance on
    lo = -(N - 1 + q_pos)
    known = {}
    row = [known.setdefault(c, bucket(c, buckets, max_distance, bidirectional))
           for c in (max(-cut, min(cut, r)) for r in range(lo, M - q_pos))]
    r = torch.arange(M)[None, :] - torch.arange(N)[:, None] - q_pos
    return torch.tensor(row)[r - lo]


def reference(q, k, v, scale, lens=None, do=None, table=None, rule=None, u=0.0):
    """Everything in float64 (on the tensors' device) from stored tensors, with bounds: {name: (value, bound)}."""
    dev, f = q.device, torch.float64
    B, H, N, d = q.shape
    Hk, M = k.shape[1:3]
    g, e = H // Hk, 2.0 ** -24
    names = ["o", "lse"] + (["dq", "dk", "dv"] if do is not None else []) + (["dtable"] if do is not None and table is not None else [])
    shape = {"o": q.shape, "lse": (B, H, N), "dq": q.shape, "dk": k.shape, "dv": k.shape, "dtable": None if table is None else table.shape}
    out = {n: (torch.zeros(shape[n], dtype=f, device=dev), torch.zeros(shape[n], dtype=f, device=dev)) for n in names}
    which = None if table is None else bucket_map(N, M, rule).to(dev)
    for b in range(B):
        n = M if lens is None else max(0, min(M, int(lens[b])))
        for h in range(H):
            if n == 0:
                out["lse"][0][b, h] = -math.inf
                continue
            Q, K, V = q[b, h].double(), k[b, h // g, :n].double(), v[b, h // g, :n].double()
            x = scale * (Q @ K.t().contiguous())
            mag = scale * (Q.abs() @ K.abs().t().contiguous())
            if table is not None:
                t = table[:, h].double()
                x = x + torch.where(t <= -2.0 ** 100, -math.inf, t)[which[:, :n]]
            top = x.max(1, keepdim=True).values
            some = top > -math.inf
            top = torch.where(some, top, 0.0)
            p = torch.exp(x - top)
            l = p.sum(1, keepdim=True)
            p = torch.where(some, p / torch.where(some, l, 1.0), 0.0)
            seen = torch.where(p > 0, x.abs(), 0.0).max(1, keepdim=True).values
            t = 4 * ((d + 4) * e * mag.max(1, keepdim=True).values + 4 * e * seen + 2.0 ** -21) + 2 * n * e
            o = p @ V
            pv = p @ V.abs()
            ob = u * o.abs() + (u + t) * pv + 1e-30
            out["o"][0][b, h], out["o"][1][b, h] = o, ob
            out["lse"][0][b, h] = torch.where(some, top + torch.log(torch.where(some, l, 1.0)), -math.inf)[:, 0]
            out["lse"][1][b, h] = (t + 4 * e * seen)[:, 0]
            if do is None:
                continue
            G = do[b, h].double()
            dv = p.t().contiguous() @ G
            out["dv"][0][b, h // g, :n] += dv
            out["dv"][1][b, h // g, :n] += ((p * (u + t + N * e)).t().contiguous() @ G.abs())
            dp = G @ V.t().contiguous()
            dpm = G.abs() @ V.abs().t().contiguous()
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta)
            # delta comes from the stored O
            db = (G.abs() * ob).sum(1, keepdim=True) + d * e * (G.abs() * o.abs()).sum(1, keepdim=True)
            dsb = p * (db + d * e * dpm) + t * ds.abs()
            out["dq"][0][b, h] = scale * (ds @ K)
            out["dq"][1][b, h] = scale * ((dsb + (u + n * e) * ds.abs()) @ K.abs())
            out["dk"][0][b, h // g, :n] += scale * (ds.t().contiguous() @ Q)
            out["dk"][1][b, h // g, :n] += scale * ((dsb + (u + N * e) * ds.abs()).t().contiguous() @ Q.abs())
            if table is not None:
                for c in range(table.shape[0]):
                    at = which[:, :n] == c
                    out["dtable"][0][c, h] += ds[at].sum()
                    out["dtable"][1][c, h] += (dsb[at] + B * N * e * ds[at].abs()).sum()
    for name in ("dq", "dk", "dv", "dtable"):
        if name in out:
            out[name] = (out[name][0], out[name][1] * (1 + u) + u * out[name][0].abs() + 1e-30)
    return out


def check(got, ref, where=""):
    """Every entry within its bound (of float64's own errors a trace is allowed)."""
    for name, (value, bound) in ref.items():
        if name not in got:
            continue
        x = got[name].double()
        same = x == value                                        # infinities of lse
        off = torch.where(same, 0.0, (x - value).abs())
        assert not torch.isnan(x).any(), f"{where} {name}: NaN"
        over = off > bound * 1.0001 + 1e-12 * value.abs().clamp(max=1e30)
        assert not over.any(), (f"{where} {name}: {int(over.sum())} of {over.numel()} entries beyond their bound, the worst by "
                                f"{float((off / (bound + 1e-30)).max()):.2f} times, off {float(off.max()):.3g}")


def views(shapes, dtype, layout, device="cuda", fill=None):
    """{name: [B, heads, rows, d]}; shapes: [(names, B, heads, rows, d)]; "fused": token-major buffers that the names share."""
    out = {}
    for names, B, heads, rows, d in shapes:
        if layout == "fused":
            buf = torch.empty((B, rows, len(names), heads, d), dtype=DT[dtype], device=device)
            if fill is not None:
                buf.fill_(fill)
            for i, n in enumerate(names):
                out[n] = buf[:, :, i].permute(0, 2, 1, 3)
        else:
            for n in names:
                out[n] = torch.empty((B, heads, rows, d), dtype=DT[dtype], device=device)
                if fill is not None:
                    out[n].fill_(fill)
    return out


class Problem:
    """One call: inputs of a seed, outputs filled with a value that must not remain."""

    def __init__(self, dtype, B, H, Hk, N, M, d, lens=None, layout="plain", rule=None, scale=0.0, gain=1.0, seed=0, train=True):
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=gen)
        self.dtype, self.rule, self.layout, self.train = dtype, rule, layout, train
        self.scale = scale or d ** -0.5
        self.p = da.attn_problem(B, H, N, M, d, Hk=Hk, dtype=CODE[dtype], scale=scale)
        self.bias = None if rule is None else da.rel_bias(*rule)
        t = views([(("q",), B, H, N, d), (("k", "v"), B, Hk, M, d), (("do",), B, H, N, d)], dtype, layout)
        t["q"].copy_(normal(B, H, N, d) * gain)
        t["k"].copy_(normal(B, Hk, M, d))
        t["v"].copy_(normal(B, Hk, M, d))
        t["do"].copy_(normal(B, H, N, d))
        t.update(views([(("o",), B, H, N, d), (("dq",), B, H, N, d), (("dk", "dv"), B, Hk, M, d)], dtype, layout, fill=777.0))
        self.t = t
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.table = None if rule is None else (normal(rule[0], H) * 1.5).to(DT[dtype]).cuda()
        self.dtable = None if rule is None else torch.full((rule[0], H), 777.0, dtype=DT[dtype], device="cuda")
        self.lse = torch.full((B, H, N), 777.0, device="cuda")
        sizes = da.da_attn_sizes(self.p, self.bias)
        self.ws = torch.full((max(sizes.forward_ws, sizes.backward_ws, 256) // 4,), float("nan"), device="cuda")
        self.lay = da.attn_layouts(**{n: da.layout_of(x) for n, x in t.items()}) if layout == "fused" else None

    def forward(self):
        t = self.t
        if self.rule is None:
            da.da_cross_attn(self.p, t["q"], t["k"], t["v"], t["o"], self.ws, kv_len=self.lens, lse=self.lse, layouts=self.lay)
        else:
            da.da_bias_attn(self.p, self.bias, t["q"], t["k"], t["v"], self.table, t["o"], self.ws, kv_len=self.lens, lse=self.lse,
                            layouts=self.lay)

    def backward(self):
        t = self.t
        a = (t["o"], self.lse, t["do"], t["dq"], t["dk"], t["dv"])
        if self.rule is None:
            da.da_cross_attn_bwd(self.p, t["q"], t["k"], t["v"], *a, self.ws, kv_len=self.lens, layouts=self.lay)
        else:
            da.da_bias_attn_bwd(self.p, self.bias, t["q"], t["k"], t["v"], self.table, *a, self.dtable, self.ws, kv_len=self.lens,
                                layouts=self.lay)

    def results(self):
        r = {n: self.t[n] for n in ("o",) + (("dq", "dk", "dv") if self.train else ())}
        r["lse"] = self.lse
        if self.train and self.rule is not None:
            r["dtable"] = self.dtable
        return r

    def reference(self):
        t = self.t
        return reference(t["q"], t["k"], t["v"], self.scale, self.lens, t["do"] if self.train else None, self.table, self.rule,
                         u=2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24)

    def run(self):
        self.forward()
        if self.train:
            self.backward()
        return self.results()
