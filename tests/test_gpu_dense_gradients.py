"""Dense attention, backward, where scores are large: the probabilities that the gradients are made of add up to 1 in every row, as the forward call's
do, whatever lse's size leaves of its last bits."""
import math

import pytest
import torch

from dense_util import Problem, bucket_map, check
from test_gpu_dense_scores import SHAPES, TYPES, weights, whole

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def unit(dtype):
    return 2.0 ** -8 if dtype == "bf16" else E


def gradients(pr, p, t, which=None):
    """Everything in 64 bits from probabilities [B,H,N,M] that the kernels' are off by a factor of at most 1 + t, with bounds (those of dense_util)."""
    (B, H, N, d), (Hk, M) = pr.t["q"].shape, pr.t["k"].shape[1:3]
    g, u = H // Hk, unit(pr.dtype)

    def wide(name):
        return pr.t[name].double().repeat_interleave(g if name in "kv" else 1, 1)

    def tr(x):
        return x.transpose(2, 3).contiguous()

    def keys(x):
        return x.unflatten(1, (Hk, g)).sum(2)
    q, k, v, G = wide("q"), wide("k"), wide("v"), wide("do")
    here = torch.ones(B, 1, M, 1, dtype=torch.float64, device="cuda")
    if pr.lens is not None:
        here = (torch.arange(M, device="cuda")[None, None, :, None] < pr.lens[:, None, None, None]).double()
    k, v = k * here, v * here
    o, pv = p @ v, p @ v.abs()
    ob = u * o.abs() + (u + t) * pv + 1e-30
    dp, dpm = G @ tr(v), G.abs() @ tr(v.abs())
    db = (G.abs() * ob).sum(3, keepdim=True) + d * E * (G.abs() * o.abs()).sum(3, keepdim=True)
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    dsb = p * (db + d * E * dpm) + t * ds.abs()
    out = {"o": (o, ob),
           "dv": (keys(tr(p) @ G), keys(tr(p * (u + t + g * N * E)) @ G.abs())),
           "dq": (pr.scale * (ds @ k), pr.scale * ((dsb + (u + M * E) * ds.abs()) @ k.abs())),
           "dk": (keys(pr.scale * (tr(ds) @ q)), keys(pr.scale * (tr(dsb + (u + g * N * E) * ds.abs()) @ q.abs())))}
    if which is not None:
        dt = [[torch.where(which == c, x, 0.0).sum((0, 2, 3)) for x in (ds, dsb + B * N * E * ds.abs())] for c in range(pr.table.shape[0])]
        out["dtable"] = tuple(torch.stack([x[i] for x in dt]) for i in (0, 1))
    for name in out:
        if name != "o":
            out[name] = (out[name][0], out[name][1] * (1 + u) + u * out[name][0].abs() + 1e-30)
    return out


def shares(pr, where):
    """The rows of dV add up to those of dO whose queries have keys, each probability rounded on its way, and dV."""
    (B, H, N, d), Hk = pr.t["q"].shape, pr.t["k"].shape[1]
    G = pr.t["do"].double() * (pr.lse > -math.inf).double()[..., None]
    want = G.unflatten(1, (Hk, H // Hk)).sum((2, 3))
    most = G.abs().unflatten(1, (Hk, H // Hk)).sum((2, 3))
    dv = pr.t["dv"].double()
    bound = most * (unit(pr.dtype) + 2.0 ** -16 + H // Hk * N * E) + unit(pr.dtype) * dv.abs().sum(2) + 1e-30
    off = (dv.sum(2) - want).abs()
    assert (off <= bound).all(), f"{where}: dV adds up to something else, at worst {float((off / bound).max()):.3g} bounds"
    for name in ("dq", "dk"):
        assert torch.isfinite(pr.t[name]).all(), (where, name)


GRADIENTS = {n: SHAPES[n] for n in ("join", "own", "pieces", "packed", "shared")}
GRADIENTS["cut"] = (1, 6, 6, 300, 2001, [1999])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("shape", list(GRADIENTS))
@pytest.mark.parametrize("scale", [1.0, 1e2, 1e4, 1e5, 1e6, 1e7, 1e9, 1e15, 1e30])
def test_probabilities_add_up(dtype, d, shape, scale):
    B, H, Hk, N, M, lens = GRADIENTS[shape]
    where = f"gradients, {shape} {dtype} d={d} scale={scale}"
    print(f"[gpu-test] {where}", flush=True)
    pr = Problem(dtype, B, H, Hk, N, M, d, lens=lens, scale=scale, seed=3)
    pr.run()
    shares(pr, where)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("shape", list(GRADIENTS))
@pytest.mark.parametrize("scale", [1e8, 1e30])
def test_the_largest_scores_have_all_the_weight(dtype, d, shape, scale):
    B, H, Hk, N, M, lens = GRADIENTS[shape]
    where = f"whole scores, gradients, {shape} {dtype} d={d} scale={scale}"
    print(f"[gpu-test] {where}", flush=True)
    pr = Problem(dtype, B, H, Hk, N, M, d, lens=lens, scale=scale, seed=1)
    whole(pr, 2)
    pr.run()
    # exponentials and their arguments 2^-21, a sum of ties, log2 of it and its exponential
    check(pr.results(), gradients(pr, weights(pr)[0], 2.0 ** -18 + 2 * M * E), where)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("low", [-3e3, -1e5, -1e7, -1e9, -1e20, -1e30])
def test_rows_that_only_large_negative_entries_reach(dtype, d, low):
    """Entries that mask in the usual way, but are numbers: in a row that has no others they make a softmax like any other.  Head 0: all
    entries, head 1: none, head 2: those of distances from 16 on, so that queries far behind the last key have only them."""
    for B, H, N, M, lens in ((2, 3, 140, 60, [60, 20]), (1, 3, 3, 3000, None), (1, 48, 700, 90, [77])):
        where = f"entries of {low} {dtype} d={d} N={N} M={M}"
        print(f"[gpu-test] {where}", flush=True)
        rule = (8, 16, 1, 0)
        pr = Problem(dtype, B, H, H, N, M, d, lens=lens, rule=rule, scale=1e-6, seed=6)
        pr.table[:, 0::3] = low
        pr.table[3, 2::3] = low                              # (8 buckets, four a direction: the last one has no end)
        pr.run()
        shares(pr, where)
        which = bucket_map(N, M, rule).cuda()
        x = pr.table.double().t()[:, which][None].expand(B, -1, -1, -1).clone()
        if lens is not None:
            x.masked_fill_(torch.arange(M, device="cuda") >= pr.lens[:, None, None, None], -math.inf)
        # scores of scale q.k below 1e-6 * 128 * 5: a factor of 1 + 2^-10 at most
        check(pr.results(), gradients(pr, torch.softmax(x, 3), 2.0 ** -10 + 2 * M * E, which), where)


@pytest.mark.parametrize("rule", [None, (8, 16, 1, 0)])
def test_captured_and_replayed_with_scores_of_either_size(rule):
    """One graph, replayed with ordinary queries and with ones whose scores are large, between eager calls: the eager call's bits."""
    pr = Problem("bf16", 2, 4, 4, 140, 1000, 64, rule=rule, lens=[1000, 90], seed=9)
    ordinary, large = pr.t["q"].clone(), pr.t["q"] * 1e7
    pr.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pr.run()
    for i, q in enumerate((large, ordinary, large, ordinary)):
        pr.t["q"].copy_(q)
        pr.run()
        shares(pr, f"replay {i} {rule}")
        want = {n: x.clone() for n, x in pr.results().items()}
        for x in pr.results().values():
            x.fill_(5.0)
        pr.ws.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for n, x in pr.results().items():
            assert torch.equal(x, want[n]), (rule, i, n)
