"""Dense attention, scores of any size: what a softmax of finite scores is does not depend on how large they are.

Inputs of -1, 0 and 1 have whole scores, which every order of summation makes exactly; times a scale of 1e8 or more a row's largest scores have all the
weight, in equal parts.  With inputs of any kind the probabilities of a row still add up to 1: O of values that are all 1."""
import math

import pytest
import torch

from dense_util import Problem

pytestmark = pytest.mark.gpu
TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
# heads of Q and K, queries, keys, lengths: waves that join, waves with columns of their own (one set, two sets), pieces of the keys joined by four
# waves a row and by one, heads that share keys with few queries and with many
SHAPES = {"join": (1, 2, 2, 60, 75, None), "own": (1, 24, 24, 1100, 75, [70]), "sets": (1, 80, 80, 1100, 75, None), "pieces": (2, 2, 2, 3, 4099, [4099, 33]),
          "many pieces": (1, 20, 20, 1100, 2001, None), "packed": (2, 8, 2, 21, 205, [205, 1]), "shared": (2, 4, 2, 300, 205, [0, 205])}


def whole(pr, seed, negative=False):
    """Q and K of -1, 0, 1; every score negative: Q of 0 and 1 with one 1 at least, K of -1."""
    gen = torch.Generator().manual_seed(seed)
    for n in ("q", "k"):
        x = torch.randint(-1, 2, pr.t[n].shape, generator=gen).float()
        if negative:
            x = -torch.ones_like(x) if n == "k" else x.abs()
            x[..., 0] = 1.0 if n == "q" else x[..., 0]
            if n == "k":
                x[..., 1:] *= torch.randint(0, 2, x[..., 1:].shape, generator=gen)
        pr.t[n].copy_(x)


def weights(pr):
    """The probabilities in 64 bits, and the whole scores: equal parts for a row's largest."""
    q, k = pr.t["q"].double(), pr.t["k"].double()
    k = k.repeat_interleave(q.shape[1] // k.shape[1], 1)
    s = torch.matmul(q, k.transpose(2, 3).contiguous())
    if pr.lens is not None:
        s.masked_fill_(torch.arange(s.shape[3], device="cuda") >= pr.lens[:, None, None, None], -math.inf)
    top = s.amax(3, keepdim=True)
    p = ((s == top) & (top > -math.inf)).double()
    return p / p.sum(3, keepdim=True).clamp_min(1.0), top[..., 0], p.sum(3)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("scale", [1e8, 1e10, 1e30])
@pytest.mark.parametrize("negative", [False, True])
def test_the_largest_scores_have_all_the_weight(dtype, d, shape, scale, negative):
    B, H, Hk, N, M, lens = SHAPES[shape]
    print(f"[gpu-test] whole scores, {shape} {dtype} d={d} scale={scale}", flush=True)
    pr = Problem(dtype, B, H, Hk, N, M, d, lens=lens, scale=scale, seed=1, train=False)
    whole(pr, 2, negative)
    pr.forward()
    p, top, ties = weights(pr)
    v = pr.t["v"].double().repeat_interleave(H // Hk, 1)
    want = torch.matmul(p, v)
    # a power of two (1, a tie) has no rounding; its scaling by the sum, the sums and the exponential's 2^-21; the stored type's rounding
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    bound = u * want.abs() + (u + 2.0 ** -20 + M * 2.0 ** -24) * torch.matmul(p, v.abs()) + 1e-30
    off = (pr.t["o"].double() - want).abs()
    assert (off <= bound).all(), f"O: {int((~(off <= bound)).sum())} of {off.numel()} beyond their bound"
    none = top == -math.inf
    assert (pr.lse[none] == -math.inf).all()
    lse = torch.where(none, 0.0, scale * top) + torch.log(ties.clamp_min(1.0))
    off = torch.where(none, 0.0, (pr.lse.double() - lse).abs())
    assert (off <= lse.abs() * 2.0 ** -22 + 2.0 ** -20).all(), "lse"


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("scale", [1.0, 1e3, 1e5, 1e6, 1e7, 1e8, 1e9, 1e10, 1e20, 1e30])
def test_probabilities_add_up(dtype, d, shape, scale):
    """Normal inputs, values of 1: O is 1, or 0 in a row without keys."""
    B, H, Hk, N, M, lens = SHAPES[shape]
    print(f"[gpu-test] probabilities, {shape} {dtype} d={d} scale={scale}", flush=True)
    pr = Problem(dtype, B, H, Hk, N, M, d, lens=lens, scale=scale, seed=3, train=False)
    pr.t["v"].fill_(1.0)
    pr.forward()
    want = torch.ones(B, device="cuda") if lens is None else (pr.lens > 0).float()
    # each probability rounded on its way into the product, the sum of all, the stored O
    bound = 2 * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + (2 * M + 8) * 2.0 ** -24
    assert ((pr.t["o"].double() - want.double()[:, None, None, None]).abs() <= bound).all()
    assert torch.isfinite(pr.lse).logical_or(want[:, None, None] == 0).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_scores_of_minus_infinity_beside_a_large_scale(dtype, d):
    """A key whose score is minus infinity weighs nothing, at any scale: K of minus infinity in one channel, where Q is 1."""
    for scale in (1.0, 1e8, 1e30):
        pr = Problem(dtype, 1, 2, 2, 60, 75, d, scale=scale, seed=4, train=False)
        whole(pr, 5)
        pr.t["q"][..., 0] = 1.0
        p0 = pr.t["k"].clone()
        pr.t["k"][:, :, 10:40, 0] = -math.inf
        print(f"[gpu-test] minus infinity {dtype} d={d} scale={scale}", flush=True)
        pr.forward()
        got = pr.t["o"].clone()
        keep = [*range(10), *range(40, 75)]
        few = Problem(dtype, 1, 2, 2, 60, len(keep), d, scale=scale, seed=4, train=False)
        few.t["q"].copy_(pr.t["q"])
        few.t["k"].copy_(p0[:, :, keep])
        few.t["v"].copy_(pr.t["v"][:, :, keep])
        few.forward()
        u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        most = pr.t["v"].double().abs().amax()
        # the same scores in other places: sums in another order, a probability's rounding against another reference
        assert ((got.double() - few.t["o"].double()).abs() <= (4 * u + 2.0 ** -18) * most).all()
