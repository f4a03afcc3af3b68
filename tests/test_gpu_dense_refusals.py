"""Dense attention: tensors that are not what the problem says are refused, with nothing written."""
import pytest
import torch

from dense_util import Problem
from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.gpu
CHANGES = {"host": lambda t: t.cpu(), "type": lambda t: t.double(), "rows": lambda t: t[:, :, :-1].contiguous(), "strides": lambda t: t.transpose(2, 3).contiguous().transpose(2, 3),
           "heads": lambda t: t.flatten(0, 1)}


@pytest.mark.parametrize("change", list(CHANGES))
@pytest.mark.parametrize("rule", [None, (8, 16, 1, 0)])
def test_tensors_that_are_refused(rule, change):
    pr = Problem("bf16", 2, 4, 2, 33, 70, 64, rule=rule, seed=1)
    for name in ("q", "k", "v", "do", "o", "dq", "dk", "dv"):
        good = pr.t[name]
        pr.t[name] = CHANGES[change](good)
        for call in (pr.forward, pr.backward):
            if call == pr.forward and name not in "qkvo":
                continue
            with pytest.raises(da.DaError) as e:
                call()
            assert e.value.status == -2, (name, change)
        pr.t[name] = good
    torch.cuda.synchronize()
    for name in ("o", "dq", "dk", "dv"):
        assert (pr.t[name] == 777.0).all()
    assert (pr.lse == 777.0).all()


@pytest.mark.parametrize("rule", [None, (8, 16, 1, 0)])
def test_other_tensors_that_are_refused(rule):
    pr = Problem("bf16", 2, 4, 2, 33, 70, 64, lens=[70, 3], rule=rule, seed=1)
    for name, bad in (("lens", pr.lens.long()), ("lens", pr.lens.cpu()), ("lens", pr.lens[:1]), ("lse", pr.lse.bfloat16()), ("lse", pr.lse[:, :, :5]),
                      ("lse", pr.lse.cpu()), ("ws", pr.ws.cpu()), ("ws", pr.ws[:1].expand(1 << 26)), ("table", None if rule is None else pr.table.float()),
                      ("table", None if rule is None else pr.table.t().contiguous().t()), ("dtable", None if rule is None else pr.dtable[:4])):
        if bad is None:
            continue
        good = getattr(pr, name)
        setattr(pr, name, bad)
        for call in (pr.forward, pr.backward):
            if call == pr.forward and name == "dtable":
                continue
            with pytest.raises(da.DaError) as e:
                call()
            assert e.value.status == -2, name
        setattr(pr, name, good)
    torch.cuda.synchronize()
    assert all((pr.t[n] == 777.0).all() for n in ("o", "dq", "dk", "dv"))
