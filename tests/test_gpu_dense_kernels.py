"""Every dense attention kernel against the definition in 64 bits, at the problems of which test_host_dense_kernels.py says what they launch."""
import pytest

from dense_kernels import SHAPES, cases, problem
from dense_util import Problem, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,mode,dtype,d", cases())
def test_kernels(shape, mode, dtype, d):
    _, B, H, Hk, N, M, _, rule = problem(dtype, d, mode, *SHAPES[shape])
    where = f"{shape}, {mode} {dtype} d={d}"
    print(f"[gpu-test] {where}", flush=True)
    pr = Problem(dtype, B, H, Hk, N, M, d, lens=[M - 3], layout="fused", rule=rule, scale=0.1 if rule else 0.0, seed=13)
    check(pr.run(), pr.reference(), where)
