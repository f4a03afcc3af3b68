"""Attention to an encoder's states and attention with a learned relative position bias, as calls to time.

A text-conditioned video transformer has, next to the self attention that the rest of this library is about, a cross
attention from the video tokens to the states of a text (or image) encoder, and the text encoder itself is a stack of self
attentions whose scores carry a bias learned per head and per bucket of relative positions.  Both are here, forward and
as a training step (forward and backward).

A case names the operator ("cross" or "bias"), the direction ("forward" or "train"), B batch elements, H heads of Q that share Hk
heads of K and V, N queries, M keys, channels per head d, the type, how full the keys are ("full": no lengths are given;
"ragged": batch element b has the length that `_lengths` gives it) and how the tensors lie in memory ("plain": contiguous
[B, heads, rows, d]; "fused": the strided views of token-major projections).  For "bias" also the bucket rule of the text
encoders of the T5 kind: the number of buckets, the distance from which on there is only one, whether keys before and
behind a query have buckets of their own, and the position of query 0 among the keys.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = "f32", "bf16"


def _cross(name, direction, B, H, Hk, N, M, *, d=128, dtype=BF16, fill="full", layout="plain", gain=1.0):
    return {"name": name, "operator": "cross", "direction": direction, "B": B, "H": H, "Hk": Hk, "N": N, "M": M, "d": d,
            "dtype": dtype, "fill": fill, "layout": layout, "gain": gain}


def _bias(name, direction, B, H, N, M, *, d=64, dtype=BF16, fill="full", layout="plain", buckets=32, max_distance=128,
          bidirectional=True, q_pos=0, gain=1.0):
    return {"name": name, "operator": "bias", "direction": direction, "B": B, "H": H, "Hk": H, "N": N, "M": M, "d": d,
            "dtype": dtype, "fill": fill, "layout": layout, "gain": gain, "buckets": buckets, "max_distance": max_distance,
            "bidirectional": bidirectional, "q_pos": q_pos}


def listed():
    return [
        # the toy float32 model of the unit tests, its two frames of 16x16 tokens reading a short prompt: launches count
        _cross("cross_toy_f32", "forward", 1, 2, 2, 512, 77, d=64, dtype=F32),
        # a latent frame of 30x52 tokens, a guided and an unguided sample in one batch with prompts of their own lengths
        _cross("cross_480p_frame_ragged", "forward", 2, 24, 24, 1560, 512, fill="ragged", layout="fused"),
        # the 40-head 720p model: 21 frames read a prompt of 512 tokens
        _cross("cross_720p", "forward", 1, 40, 40, 75600, 512),
        # one new query per sequence against long encoder states whose heads are shared
        _cross("cross_one_query", "forward", 4, 32, 8, 1, 32768, fill="ragged"),
        # fine-tuning on the 480p clip
        _cross("cross_480p_train", "train", 1, 24, 24, 32760, 512),
        # a few learned queries that condense a long sequence of states (heads shared), trained
        _cross("cross_few_queries_train", "train", 2, 16, 4, 127, 20011, fill="ragged", layout="fused"),
        # a float32 check of two latent frames against image states (256 patches and a summary)
        _cross("cross_f32_train", "train", 1, 8, 8, 3120, 257, d=64, dtype=F32),
        # the text encoder's layer on two padded prompts
        _bias("bias_encoder", "forward", 2, 64, 512, 512, fill="ragged", layout="fused"),
        # one token at a time with positions that look back only
        _bias("bias_step", "forward", 8, 32, 1, 4095, bidirectional=False, q_pos=4094),
        # the text encoder trained on a batch of prompts
        _bias("bias_encoder_train", "train", 4, 64, 512, 512, fill="ragged"),
        # a long document, wide heads
        _bias("bias_long_train", "train", 1, 24, 4099, 4099, d=128),
        # a small float32 encoder, odd length
        _bias("bias_f32_train", "train", 3, 4, 197, 197, dtype=F32, fill="ragged", buckets=16, max_distance=64),
    ]


def draw(rng):
    """One more case of the same ranges: lengths over their logarithm, odd ones as likely as even ones."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    d = rng.choice([64, 128])
    dtype = F32 if rng.random() < 0.25 else BF16
    direction = rng.choice(["forward", "train"])
    fill = rng.choice(["full", "ragged"])
    layout = rng.choice(["plain", "fused"])
    gain = rng.choice([0.25, 1.0, 2.0])
    least = 2 if direction == "train" else 1       # (with one key the gradients of Q and K are zero: nothing to compare)
    if rng.random() < 0.55:
        Hk = log_int(1, 24)
        c = _cross("", direction, rng.choice([1, 1, 2, 3, 8]), Hk * rng.choice([1, 1, 2, 4]), Hk, log_int(1, 120000),
                   log_int(least, 40000), d=d, dtype=dtype, fill=fill, layout=layout, gain=gain)
    else:
        M = log_int(least, 6000)
        step = rng.random() < 0.25
        buckets = rng.choice([8, 32, 64])
        c = _bias("", direction, rng.choice([1, 2, 3, 8]), log_int(1, 64), 1 if step else M, M, d=d, dtype=dtype, fill=fill,
                  layout=layout, buckets=buckets, max_distance=rng.choice([buckets, 128, 500]), bidirectional=rng.random() < 0.7,
                  q_pos=M - 1 if step else 0, gain=gain)
    # no more than the largest listed cases: the scores of 40 heads of 75600 by 512 forward, of 24 heads of 32760 by 512 trained,
    # half a gigabyte of inputs
    most = 1.5e9 if direction == "forward" else 4.0e8
    while c["B"] * c["H"] * float(c["N"]) * c["M"] > most or \
            (c["B"] * (c["H"] * c["N"] + c["Hk"] * c["M"])) * d * 2.0 > 5.0e8:
        if c["B"] > 1:
            c["B"] //= 2
        elif c["Hk"] > 1:
            c["H"] = c["H"] // c["Hk"] * (c["Hk"] // 2)
            c["Hk"] //= 2
        elif c["operator"] == "bias":
            c["M"] = c["M"] * 3 // 4
            c["N"] = min(c["N"], c["M"])
            c["q_pos"] = c["M"] - 1 if c["q_pos"] else 0
        else:
            c["N"], c["M"] = max(1, c["N"] // 2), max(least, c["M"] * 3 // 4)
    del c["name"]
    return c


def _lengths(c):
    """Keys of each batch element (at least one): spread over the range by the golden ratio, the first one full."""
    if c["fill"] == "full":
        return [c["M"]] * c["B"]
    return [max(1, c["M"] if b == 0 else int(c["M"] * (0.1 + 0.9 * ((b * 0.6180339887) % 1.0)))) for b in range(c["B"])]


def work(c):
    lens = _lengths(c)
    size = 4 if c["dtype"] == F32 else 2
    q = c["B"] * c["H"] * c["N"] * c["d"]
    kv = 2 * c["Hk"] * sum(lens) * c["d"]
    table = c["buckets"] * c["H"] if c["operator"] == "bias" else 0
    pairs = c["H"] * float(c["N"]) * sum(lens) * c["d"]
    if c["direction"] == "forward":
        return {"bytes": size * (2 * q + kv + table), "flops": 4 * pairs}
    # Q, K, V, the gradient of O and the table are read, O and the gradients of the rest written: of a whole training step O is
    # an output of its first half and needs no second reading for the floor
    return {"bytes": size * (4 * q + 2 * kv + 2 * table), "flops": 14 * pairs}


def _dtype(c):
    return torch.float32 if c["dtype"] == F32 else torch.bfloat16


def _views(c, shape_of):
    """Tensors [B, heads, rows, d]: contiguous, or the views of buffers in which a token's heads (and, for K and V, both of them)
    lie together."""
    B, d, dt = c["B"], c["d"], _dtype(c)
    out = {}
    for names, heads, rows in shape_of:
        if c["layout"] == "fused":
            buf = torch.empty((B, rows, len(names), heads, d), dtype=dt, device="cuda")
            for i, n in enumerate(names):
                out[n] = buf[:, :, i].permute(0, 2, 1, 3)
        else:
            for n in names:
                out[n] = torch.empty((B, heads, rows, d), dtype=dt, device="cuda")
    return out


def _borders(c):
    """The distances at which a new bucket begins, beyond those that have one each: with n buckets in a direction, e = n // 2 of
    them for a distance each, the k-th of the others begins at the smallest a with (a / e)^(n - e) >= (max_distance / e)^k.
    In integers, since a distance on a border belongs to the bucket that begins there."""
    n = c["buckets"] // 2 if c["bidirectional"] else c["buckets"]
    e = n // 2
    top, a, out = n - e, e, []
    for k in range(1, top):
        while a ** top < e ** (top - k) * c["max_distance"] ** k:
            a += 1
        out.append(a)
    return n, e, out


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(c)

    def normal(shape, std):
        x = torch.empty(shape, dtype=dt, device="cuda")
        for part in x.flatten(0, 1).split(16):             # bounded temporaries
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * std)
        return x

    st = {"case": c}
    kv = [(("k", "v"), c["Hk"], c["M"])]
    t = _views(c, [(("q",), c["H"], c["N"])] + kv)
    # normalised queries and keys (bias: the T5 kind does not divide by sqrt(d), its weights do); values of unit spread
    scale = 1.0 if c["operator"] == "bias" else c["d"] ** -0.5
    t["q"].copy_(normal((c["B"], c["H"], c["N"], c["d"]), c["gain"] * c["d"] ** -0.5 / scale))
    t["k"].copy_(normal((c["B"], c["Hk"], c["M"], c["d"]), 1.0))
    t["v"].copy_(normal((c["B"], c["Hk"], c["M"], c["d"]), 1.0))
    st.update(t)
    st["scale"] = scale
    st["lens"] = None if c["fill"] == "full" else torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    if c["operator"] == "bias":
        st["table"] = (torch.randn((c["buckets"], c["H"]), generator=gen, device="cuda") * 1.5).to(dt)
        n, e, borders = _borders(c)
        st["rule"] = (n, e, torch.tensor(borders, dtype=torch.int64, device="cuda"))
    if c["direction"] == "train":
        st["do"] = _views(c, [(("do",), c["H"], c["N"])])["do"].copy_(normal((c["B"], c["H"], c["N"], c["d"]), 1.0))
    if own:
        from paper_2505_14708_amd import binding as da
        p = da.attn_problem(c["B"], c["H"], c["N"], c["M"], c["d"], Hk=c["Hk"], scale=scale,
                            dtype=da.DA_F32 if c["dtype"] == F32 else da.DA_BF16)
        st["p"] = p
        st["rel"] = None
        if c["operator"] == "bias":
            st["rel"] = da.rel_bias(c["buckets"], c["max_distance"], int(c["bidirectional"]), c["q_pos"])
            st["dtable"] = torch.empty_like(st["table"])
        st.update(_views(c, [(("o",), c["H"], c["N"])]))
        sizes = da.da_attn_sizes(p, st["rel"])
        need = sizes.forward_ws
        lay = {n: da.layout_of(st[n]) for n in "qkvo"}
        if c["direction"] == "train":
            need = max(need, sizes.backward_ws)
            g = _views(c, [(("dq",), c["H"], c["N"]), (("dk", "dv"), c["Hk"], c["M"])])
            st.update(g)
            lay.update({n: da.layout_of(st[n]) for n in ("do", "dq", "dk", "dv")})
            st["lse"] = torch.empty((c["B"], c["H"], c["N"]), dtype=torch.float32, device="cuda")
        st["layouts"] = da.attn_layouts(**lay) if c["layout"] == "fused" else None
        st["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    return st


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2505_14708_amd import binding as da
    p, lens, lay, ws = st["p"], st["lens"], st["layouts"], st["ws"]
    q, k, v, o = st["q"], st["k"], st["v"], st["o"]
    train = st["case"]["direction"] == "train"
    lse = st["lse"] if train else None
    if st["rel"] is None:
        da.da_cross_attn(p, q, k, v, o, ws, kv_len=lens, lse=lse, layouts=lay)
        if not train:
            return {"o": o}
        da.da_cross_attn_bwd(p, q, k, v, o, lse, st["do"], st["dq"], st["dk"], st["dv"], ws, kv_len=lens, layouts=lay)
        return {"o": o, "dq": st["dq"], "dk": st["dk"], "dv": st["dv"]}
    da.da_bias_attn(p, st["rel"], q, k, v, st["table"], o, ws, kv_len=lens, lse=lse, layouts=lay)
    if not train:
        return {"o": o}
    da.da_bias_attn_bwd(p, st["rel"], q, k, v, st["table"], o, lse, st["do"], st["dq"], st["dk"], st["dv"], st["dtable"], ws,
                        kv_len=lens, layouts=lay)
    return {"o": o, "dq": st["dq"], "dk": st["dk"], "dv": st["dv"], "dtable": st["dtable"]}


def _buckets(st):
    """Bucket of key j as query i sees it, by j - i + N - 1."""
    c = st["case"]
    n, e, borders = st["rule"]
    r = torch.arange(1 - c["N"], c["M"], device="cuda") - c["q_pos"]
    base = torch.zeros_like(r)
    if c["bidirectional"]:
        base = torch.where(r > 0, n, 0)
        a = r.abs()
    else:
        a = (-r).clamp_min(0)
    far = e + torch.bucketize(a, borders, right=True)
    return base + torch.where(a < e, a, far)


def _run_plain(st):
    """Scores, exponentials and products written out, a batch element and a group of heads at a time so that the scores fit."""
    c = st["case"]
    B, H, Hk, N, M, d = (c[x] for x in ("B", "H", "Hk", "N", "M", "d"))
    group, scale, train = H // Hk, st["scale"], c["direction"] == "train"
    dt = _dtype(c)
    o = torch.empty((B, H, N, d), dtype=dt, device="cuda")
    if train:
        dq = torch.empty((B, H, N, d), dtype=dt, device="cuda")
        dk, dv = (torch.empty((B, Hk, M, d), dtype=dt, device="cuda") for _ in range(2))
    cols = torch.arange(M, device="cuda")
    if c["operator"] == "bias":
        by_r = _buckets(st)
        bucket = by_r[cols[None, :] - torch.arange(N, device="cuda")[:, None] + (N - 1)]
        table = st["table"].float()
        dtable = torch.zeros((c["buckets"], H), dtype=torch.float64, device="cuda")
    step = max(1, min(Hk, int(1.0e9 // (float(group) * N * M))))
    for b in range(B):
        for h0 in range(0, Hk, step):
            hk = min(step, Hk - h0)
            heads = slice(h0 * group, (h0 + hk) * group)
            q = st["q"][b, heads].float().reshape(hk, group * N, d)
            k = st["k"][b, h0:h0 + hk].float()
            v = st["v"][b, h0:h0 + hk].float()
            s = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale)               # [hk, group*N, M]
            if c["operator"] == "bias":
                s += table[:, heads].t()[:, bucket]
            if st["lens"] is not None:
                s.masked_fill_(cols >= st["lens"][b], float("-inf"))
            s -= s.amax(2, keepdim=True)
            s.exp_()
            s /= s.sum(2, keepdim=True)
            out = torch.matmul(s, v)
            o[b, heads] = out.reshape(hk * group, N, d).to(dt)
            if not train:
                continue
            g = st["do"][b, heads].float().reshape(hk, group * N, d)
            dv[b, h0:h0 + hk] = torch.matmul(s.transpose(1, 2).contiguous(), g).to(dt)
            ds = torch.matmul(g, v.transpose(1, 2).contiguous())
            ds -= (g * out).sum(2, keepdim=True)
            ds *= s
            del s
            if c["operator"] == "bias":
                # diagonals: in rows of N + M zeros behind each other, and read again in rows of one less, each row is a place further
                x = torch.zeros((hk, N, N + M), device="cuda")
                x[:, :, :M] = ds.flip(1)
                x = x.flatten(1)[:, :N * (N + M - 1)].view(hk, N, N + M - 1).sum(1, dtype=torch.float64)
                dtable[:, heads].index_add_(0, by_r, x.t())
                del x
            dq[b, heads] = (torch.matmul(ds, k) * scale).reshape(hk * group, N, d).to(dt)
            dk[b, h0:h0 + hk] = (torch.matmul(ds.transpose(1, 2).contiguous(), q) * scale).to(dt)
            del ds
    if not train:
        return {"o": o}
    res = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if c["operator"] == "bias":
        res["dtable"] = dtable.to(dt)
    return res


def exact(c, seed):
    """From the definition in 64 bits, one head of one batch element at a time and over the keys that are there only."""
    st = prepare(c, seed)
    B, H, Hk, N, M, d = (c[x] for x in ("B", "H", "Hk", "N", "M", "d"))
    f = dict(dtype=torch.float64, device="cuda")
    train = c["direction"] == "train"
    res = {"o": torch.zeros((B, H, N, d), **f)}
    if train:
        res["dq"] = torch.zeros((B, H, N, d), **f)
        res["dk"], res["dv"] = torch.zeros((B, Hk, M, d), **f), torch.zeros((B, Hk, M, d), **f)
    which = None
    if c["operator"] == "bias":
        one_way = c["buckets"] // 2 if c["bidirectional"] else c["buckets"]
        single = one_way // 2

        def bucket_of(r):
            a = abs(r) if c["bidirectional"] else max(-r, 0)
            if a >= single:
                # floor((one_way - single) log(a / single) / log(max_distance / single)), at most the last
                t = one_way - single
                a = single + sum(a ** t * single ** k >= single ** t * c["max_distance"] ** k for k in range(1, t))
            return a + (one_way if c["bidirectional"] and r > 0 else 0)

        low = -(N - 1 + c["q_pos"])
        at = {}
        cut = max(c["max_distance"], one_way)
        rows = [at.setdefault(max(-cut, min(cut, r)), bucket_of(max(-cut, min(cut, r)))) for r in range(low, M - c["q_pos"])]
        by_r = torch.tensor(rows, device="cuda")
        r = torch.arange(M, device="cuda")[None, :] - torch.arange(N, device="cuda")[:, None] - c["q_pos"]
        which = by_r[r - low]
        if train:
            res["dtable"] = torch.zeros((c["buckets"], H), **f)
    for b, n in enumerate(_lengths(c)):
        for h in range(H):
            hk = h * Hk // H
            q, k, v = st["q"][b, h].double(), st["k"][b, hk, :n].double(), st["v"][b, hk, :n].double()
            x = st["scale"] * (q @ k.t().contiguous())
            if which is not None:
                x = x + st["table"][:, h].double()[which[:, :n]]
            p = torch.exp(x - x.max(1, keepdim=True).values)
            p = p / p.sum(1, keepdim=True)
            res["o"][b, h] = p @ v
            if train:
                g = st["do"][b, h].double()
                res["dv"][b, hk, :n] += p.t().contiguous() @ g
                y = g @ v.t().contiguous()
                y = p * (y - (p * y).sum(1, keepdim=True))
                res["dq"][b, h] = st["scale"] * (y @ k)
                res["dk"][b, hk, :n] += st["scale"] * (y.t().contiguous() @ q)
                if which is not None:
                    for t in range(c["buckets"]):
                        res["dtable"][t, h] += torch.where(which[:, :n] == t, y, 0.0).sum()
    return res
