"""Dense attention in bfloat16: errors in norm, where the bounds entry by entry (dense_util) leave room for what the kernels correct.

Rounding to nearest with 8 bits is off by at most 2^-8 of a value in [1, 2), evenly: relative to values that are spread evenly over their logarithm, by
2^-8 / sqrt(3) sqrt(3/8 / ln 2) = 1.659e-3 in the mean square.  O, dK, dV and dQ have two such roundings that are independent: of each
probability (or its gradient) on its way into the second product, and of the result: 2.346e-3.  A twentieth more is for all that is float32, and for the
number of entries (ten thousand and more).  dtable has the result's alone; it is only two thousand entries with very different sizes: a quarter more.
delta from the stored O and nothing else adds about as much again where the scores are spread (4 of them here, as their standard deviation)."""
import pytest
import torch

from dense_util import Problem, bucket_map

pytestmark = pytest.mark.gpu
ROUNDING = 1.659e-3


def norms(pr, names):
    got, want = pr.run(), pr.reference()
    off = {n: float((got[n].double() - want[n][0]).norm() / want[n][0].norm()) for n in names}
    print("[gpu-test] " + " ".join(f"{n} {x:.3e}" for n, x in off.items()), flush=True)
    return off


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gain", [1.0, 4.0])
@pytest.mark.parametrize("rows,keys", [(512, 4), (512, 31), (512, 100), (64, 128), (2000, 20), (512, 512), (40, 3000)])
def test_keys_and_queries(d, gain, rows, keys):
    """dQ as far as delta is corrected before it: up to 128 keys in one piece."""
    pr = Problem("bf16", 1, 16, 16, rows, keys, d, gain=gain, seed=5)
    for n, off in norms(pr, ("o", "dk", "dv") + (("dq",) if keys <= 128 else ())).items():
        assert off < 1.05 * 2.0 ** 0.5 * ROUNDING, (n, off)


@pytest.mark.parametrize("d", [64, 128])
def test_table(d):
    pr = Problem("bf16", 1, 64, 64, 512, 512, d, rule=(32, 128, 1, 0), scale=d ** -0.5, seed=5)
    off = norms(pr, ("dtable", "dk"))
    assert off["dtable"] < 1.25 * ROUNDING and off["dk"] < 1.05 * 2.0 ** 0.5 * ROUNDING, off


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gain", [1.0, 2.0, 4.0])
@pytest.mark.parametrize("heads,rows,keys,rule", [(16, 512, 130, None), (16, 512, 512, None), (16, 512, 2000, None), (16, 40, 3000, None), (64, 300, 300, None),
                                                  (16, 512, 512, (32, 128, 1, 0))])
def test_gradient_of_queries(d, gain, heads, rows, keys, rule):
    """dQ is off by what the roundings of ds and of dQ make of the values in 64 bits here, with any number of keys, in one piece or several."""
    pr = Problem("bf16", 1, heads, heads, rows, keys, d, gain=gain, rule=rule, scale=d ** -0.5, seed=7)
    off = norms(pr, ("dq",))["dq"]
    q, k, v, do = (pr.t[n][0].double() for n in ("q", "k", "v", "do"))
    x = pr.scale * (q @ k.transpose(1, 2).contiguous())
    if rule:
        x = x + pr.table.double().t()[:, bucket_map(rows, keys, rule).cuda()]
    p, dp = torch.softmax(x, 2), do @ v.transpose(1, 2).contiguous()
    ds = p * (dp - (p * dp).sum(2, keepdim=True))
    dq = pr.scale * (ds @ k)
    least = float(((pr.scale * (ds.bfloat16().double() @ k)).bfloat16().double() - dq).norm() / dq.norm())
    assert off < 1.05 * least, (off, least)
