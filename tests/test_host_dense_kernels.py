"""Dense attention: which kernel runs for what (the launches are noted, nothing runs).  test_gpu_dense_kernels.py runs the same problems."""
import os

import pytest

from dense_kernels import RULE, SHAPES, TYPES, cases, problem, record, wanted
from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.skipif(not os.path.exists(da.LIB_PATH), reason="library not built")


def test_problems_reach_the_kernels_that_they_are_for(tmp_path):
    """And all of them together reach every dense kernel that the library has."""
    all_cases = cases()
    known, calls = record(tmp_path, [problem(dtype, d, mode, *SHAPES[shape]) for shape, mode, dtype, d in all_cases])
    assert len(calls) == len(all_cases)
    seen = set()
    for (shape, mode, dtype, d), call in zip(all_cases, calls):
        got = {k for k, _ in call}
        seen |= got
        for k in wanted(shape, dtype, d, mode):
            assert k in got, (shape, mode, dtype, d, k, sorted(got))
    assert seen == known, f"not run: {sorted(known - seen)}"


@pytest.mark.parametrize("rule", [None, RULE])
def test_few_columns_of_many_heads_fill_the_card(tmp_path, rule):
    """192 heads whose shorter side is at most 65: at least three waves to four SIMDs have columns of their own to work on."""
    problems = []
    for dtype, d in TYPES:
        for few in (1, 16, 32, 33, 64, 65):
            problems += [(dtype, 8, 24, 24, 16380, few, d, rule), (dtype, 8, 24, 24, few, 16380, d, rule)]
    _, calls = record(tmp_path, problems)
    for p, call in zip(problems, calls):
        few = min(p[4], p[5])
        (name, wgs), = [(k, w) for k, w in call if k[0] == ("dkv" if p[5] == few else "dq")]
        waves, join = name[3], name[4]
        busy = wgs * (waves if join > 1 else -(-few // 32))
        assert busy >= 768, (p, name, wgs)
