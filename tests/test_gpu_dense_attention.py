"""Attention to an encoder's states and attention with a relative position bias against the definitions in 64 bits, forward and backward, at
the sizes, lengths, layouts and masks where tiles, pieces and sets of rows end.  Tolerances: the bounds of dense_util."""
import math

import pytest
import torch

from dense_util import Problem, check
from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.gpu
TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]


def run(where, *a, **kw):
    print(f"[gpu-test] {where}", flush=True)
    pr = Problem(*a, **kw)
    check(pr.run(), pr.reference(), where)
    return pr


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("N,M", [(1, 1), (1, 2), (31, 33), (32, 32), (33, 31), (64, 65), (65, 64), (127, 129), (128, 1), (129, 97), (257, 77), (300, 513)])
def test_sizes_around_tiles(dtype, d, N, M):
    run(f"cross {dtype} d={d} N={N} M={M}", dtype, 2, 2, 2, N, M, d, seed=N + M)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,Hk,N", [(4, 1, 1), (6, 2, 5), (8, 2, 16), (4, 2, 33), (6, 3, 70), (4, 1, 100)])
def test_heads_that_share_keys(dtype, d, H, Hk, N):
    run(f"shared {dtype} d={d} {H}/{Hk} N={N}", dtype, 2, H, Hk, N, 150, d, lens=[150, 71], layout="fused", seed=H + N)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_lengths(dtype, d):
    """None, one, ends of tiles, more than there are, less than none; what lies behind them is not looked at."""
    lens = [0, 1, 31, 32, 63, 64, 65, 128, 200, 300, -5]
    pr = Problem(dtype, len(lens), 2, 1, 45, 200, d, lens=lens, seed=3)
    for b, n in enumerate(lens):
        for name, x in (("k", math.nan), ("v", math.inf)):
            pr.t[name][b, :, max(0, min(200, n)):] = x
    check(pr.run(), pr.reference(), f"lengths {dtype} {d}")
    assert (pr.t["o"][0] == 0).all() and (pr.lse[0] == -math.inf).all() and (pr.t["dq"][0] == 0).all()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("N,M,H,Hk", [(1, 9000, 2, 2), (3, 4099, 8, 2), (40, 6000, 2, 1), (100, 3001, 1, 1)])
def test_few_queries_many_keys(dtype, d, N, M, H, Hk):
    """The keys are cut; lengths that leave pieces empty."""
    pr = run(f"pieces {dtype} d={d} N={N} M={M}", dtype, 3, H, Hk, N, M, d, lens=[M, 200, 0], layout="fused", seed=N)
    assert da.da_attn_sizes(pr.p).forward_ws > 0


@pytest.mark.parametrize("dtype,d", TYPES)
def test_many_queries_few_keys(dtype, d):
    """The queries are cut for the gradients of K and V."""
    run(f"many queries {dtype} d={d}", dtype, 1, 2, 2, 5003, 77, d, lens=[70], seed=9)
    run(f"many queries, shared {dtype} d={d}", dtype, 2, 4, 2, 1111, 20, d, seed=9)


def test_two_sets_of_queries():
    """bf16 with enough workgroups that a wave takes 64 queries."""
    run("two sets", "bf16", 1, 24, 24, 2600, 130, 128, layout="fused", seed=1)
    run("two sets, 64 channels, shared", "bf16", 2, 32, 8, 1030, 200, 64, lens=[199, 40], seed=1)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("gain", [0.0, 30.0])
def test_flat_and_peaked(dtype, d, gain):
    run(f"gain {gain} {dtype} d={d}", dtype, 1, 2, 2, 70, 300, d, gain=gain, seed=5)


RULES = [(32, 128, 1, 0), (32, 128, 0, 0), (2, 2, 0, 0), (4, 2, 1, 0), (8, 1000, 1, 0), (256, 1024, 0, 3), (256, 300, 1, -40), (6, 17, 1, 100000),
         (7, 20, 0, -300)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("rule", RULES)
def test_bias_rules(dtype, d, rule):
    run(f"bias {dtype} d={d} {rule}", dtype, 2, 3, 3, 261, 301, d, lens=[301, 120], rule=rule, scale=0.2, layout="fused", seed=rule[0])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("N", [1, 2, 31, 64, 65, 130])
def test_bias_sizes(dtype, d, N):
    run(f"bias {dtype} d={d} N=M={N}", dtype, 2, 2, 2, N, N, d, rule=(32, 128, 1, 0), scale=0.1, seed=N)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_bias_far_and_pieces(dtype, d):
    """Squares beyond the last border on both sides; one query behind many keys; heads that share keys, each with its bias."""
    run(f"bias long {dtype} d={d}", dtype, 1, 2, 2, 700, 700, d, rule=(16, 40, 1, 0), scale=0.1, seed=2)
    run(f"bias step {dtype} d={d}", dtype, 2, 4, 4, 1, 5000, d, lens=[5000, 33], rule=(32, 128, 0, 4999), scale=0.1, seed=2)
    run(f"bias shared {dtype} d={d}", dtype, 2, 4, 2, 90, 210, d, lens=[0, 210], rule=(32, 128, 1, 7), scale=0.1, layout="fused", seed=2)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_bias_that_masks(dtype, d):
    """Minus infinity and the type's lowest value in the table: rows with some, and rows with nothing, to attend."""
    N = 140
    rule = (8, 16, 1, 0)
    for low in (-math.inf, float(torch.finfo(torch.float32 if dtype == "f32" else torch.bfloat16).min)):
        pr = Problem(dtype, 1, 2, 2, N, N, d, rule=rule, scale=0.1, lens=[100], seed=4)
        pr.table[4:, 0] = low                               # nothing ahead of the query
        pr.table[:, 1] = low                                # nothing at all
        check(pr.run(), pr.reference(), f"masking {low} {dtype} {d}")
        assert (pr.t["o"][:, 1] == 0).all() and (pr.lse[:, 1] == -math.inf).all() and (pr.t["dk"][:, 1] == 0).all()


@pytest.mark.parametrize("rule", [None, (32, 128, 1, 0)])
def test_same_bits_every_time(rule):
    pr = Problem("bf16", 2, 4, 4, 300, 1500, 128, rule=rule, lens=[1500, 900], seed=6)
    first = {n: x.clone() for n, x in pr.run().items()}
    pr.ws.fill_(3.0)
    for n, x in pr.run().items():
        assert torch.equal(x.view(torch.uint8) if x.is_contiguous() else x, first[n].view(torch.uint8) if x.is_contiguous() else first[n]), n


def test_other_stream_and_graph():
    """Forward and backward on a stream of their own, captured, and replayed with other inputs between eager calls."""
    for rule in (None, (32, 128, 1, 0)):
        pr = Problem("bf16", 2, 4, 4, 33, 2000, 64, rule=rule, lens=[2000, 700], seed=7)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            pr.run()
        s.synchronize()
        check(pr.results(), pr.reference(), "stream")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pr.run()
        for i in range(3):
            pr.t["q"].copy_(torch.randn(pr.t["q"].shape, generator=torch.Generator().manual_seed(i)))
            pr.run()
            want = {n: x.clone() for n, x in pr.results().items()}
            for x in pr.results().values():
                x.fill_(5.0)
            pr.ws.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            for n, x in pr.results().items():
                assert torch.equal(x, want[n]), (rule, i, n)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("scale", [1e-30, 1e-6, 3.0])
def test_scales(dtype, d, scale):
    """Scores that vanish beside lse, and peaked ones."""
    run(f"scale {scale} {dtype} d={d}", dtype, 1, 2, 2, 60, 200, d, scale=scale, lens=[150], seed=12)
    run(f"scale {scale} {dtype} d={d}, bias", dtype, 1, 2, 2, 60, 200, d, scale=scale, rule=(32, 128, 1, 0), seed=12)


def test_two_calls_at_once():
    """Two streams, a workspace each, at the same time: the results of one after the other."""
    for rule in (None, (32, 128, 1, 0)):
        prs = [Problem("bf16", 2, 8, 4, 90, 3000, 64, rule=rule, lens=[3000, 100], seed=s) for s in (20, 21)]
        want = [{n: x.clone() for n, x in pr.run().items()} for pr in prs]
        streams = [torch.cuda.Stream() for _ in prs]
        torch.cuda.synchronize()
        for _ in range(5):
            for pr, s in zip(prs, streams):
                with torch.cuda.stream(s):
                    pr.run()
        torch.cuda.synchronize()
        for pr, w in zip(prs, want):
            for n, x in pr.results().items():
                assert torch.equal(x, w[n]), (rule, n)


def test_rows_far_apart():
    """Offsets beyond 32 bits: rows of K and V 8 MB apart, in a buffer of 3 GB that holds nothing else."""
    M, step = 384, 4 << 20                                       # elements
    buf = torch.empty(M * step, dtype=torch.bfloat16, device="cuda")
    pr = Problem("bf16", 1, 1, 1, 40, M, 64, seed=8)
    lay = {n: da.layout_of(x) for n, x in pr.t.items()}
    for i, n in enumerate(("k", "v", "dk", "dv")):
        far = torch.as_strided(buf, (1, 1, M, 64), (M * step, 128, step, 1), 64 * i)
        far.copy_(pr.t[n])
        pr.t[n] = far
        lay[n] = da.da_layout(64, 64, step) if n in ("dk", "dv") else da.layout_of(far)
    pr.lay = da.attn_layouts(**lay)
    check(pr.run(), pr.reference(), "far rows")


def test_gradients_against_differences():
    """The backward call against central differences of the forward call (float32, a random direction for each input)."""
    pr = Problem("f32", 1, 2, 1, 20, 50, 64, rule=(8, 16, 1, 0), lens=[45], scale=0.125, seed=11)
    pr.run()
    g = {n: x.clone() for n, x in pr.results().items()}
    gen = torch.Generator().manual_seed(1)
    for name, x, grad in (("q", pr.t["q"], g["dq"]), ("k", pr.t["k"], g["dk"]), ("v", pr.t["v"], g["dv"]), ("table", pr.table, g["dtable"])):
        at, way = x.clone(), torch.randn(x.shape, generator=gen).cuda()
        h, loss = 2.0 ** -8, []
        for sign in (1, -1):
            x.copy_(at + sign * h * way)
            pr.forward()
            loss.append(float((pr.t["o"].double() * pr.t["do"].double()).sum()))
        x.copy_(at)
        slope, want = (loss[0] - loss[1]) / (2 * h), float((grad.double() * way.double()).sum())
        # rounding: 2 x 2000 entries of O off by about 2^-22, over 2h; the third derivative times h^2 / 6
        assert abs(slope - want) < 2.0 ** -10 * (float(grad.double().norm() * way.double().norm()) + 1.0), (name, slope, want)
