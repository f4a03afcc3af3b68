"""What the binding of dense attention looks at in tensors before it hands their addresses on, without a GPU: tensors of the CPU are on device -1, which
stands for the current device here."""
import os

import pytest
import torch

from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.skipif(not os.path.exists(da.LIB_PATH), reason="library not built")
SHAPE = (2, 3, 10, 64)


def place(t, layout=None, shape=SHAPE, dtype=torch.bfloat16, device=-1):
    return da._place(t, "call", "X", shape, dtype, layout, device)


def test_what_is_accepted():
    t = torch.zeros(SHAPE, dtype=torch.bfloat16)
    assert place(t) == t.data_ptr() and place(t, da.da_layout(0, 0, 0)) == t.data_ptr() and place(t, da.layout_of(t)) == t.data_ptr()
    far = torch.zeros(2, 10, 2, 3, 64, dtype=torch.bfloat16)[:, :, 1].permute(0, 2, 1, 3)
    assert place(far, da.layout_of(far)) == far.data_ptr()
    one = torch.zeros(1, 10, 3, 64, dtype=torch.bfloat16).permute(0, 2, 1, 3)[:, :, 4:5]       # an extent of 1 has no stride
    assert place(one, da.da_layout(7, 64, 5), shape=(1, 3, 1, 64)) == one.data_ptr()
    assert place(None) is None and place(4096) == 4096


def test_single_changes_are_refused():
    t = torch.zeros(SHAPE, dtype=torch.bfloat16)
    far = torch.zeros(2, 10, 3, 64, dtype=torch.bfloat16).permute(0, 2, 1, 3)
    lay = da.layout_of(far)
    every_other = torch.zeros(2, 3, 10, 128, dtype=torch.bfloat16)[..., ::2]
    for bad, kw in ((t, dict(device=0)), (t.float(), {}), (t.half(), {}), (t, dict(shape=(2, 3, 11, 64))), (t, dict(shape=(3, 2, 10, 64))), (t[:, :2], {}),
                    (t[0], {}), (far, {}), (t.transpose(1, 2).contiguous().transpose(1, 2), {}), (t, dict(layout=lay)),
                    (far, dict(layout=da.da_layout(lay.stride_b + 8, lay.stride_h, lay.stride_n))),
                    (far, dict(layout=da.da_layout(lay.stride_b, lay.stride_h + 8, lay.stride_n))),
                    (far, dict(layout=da.da_layout(lay.stride_b, lay.stride_h, lay.stride_n + 8))),
                    (every_other, {}), (every_other, dict(layout=da.da_layout(3 * 10 * 128, 10 * 128, 128)))):
        with pytest.raises(da.DaError) as e:
            place(bad, **kw)
        assert e.value.status == -2


CALLS = {"cross": ("Q K V O ws kv_len lse", False), "cross_bwd": ("Q K V O lse dO dQ dK dV ws kv_len", False),
         "bias": ("Q K V table O ws kv_len lse", True), "bias_bwd": ("Q K V table O lse dO dQ dK dV dtable ws kv_len", True)}


def call(name, monkeypatch, device, **tensors):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
    names, bias = CALLS[name]
    p, rel = da.attn_problem(2, 3, 10, 20, 64), da.rel_bias(32, 128)
    a = {n: tensors.get(n, 0x10000) for n in names.split()}
    tail = {n: a.pop(n) for n in ("kv_len", "lse") if n in a and not (n == "lse" and name.endswith("bwd"))}
    with pytest.raises(da.DaError) as e:
        getattr(da, f"da_{name.split('_')[0]}_attn{'_bwd' if 'bwd' in name else ''}")(p, *([rel] if bias else []), *a.values(), stream=0, **tail)
    return e.value


@pytest.mark.parametrize("name", list(CALLS))
def test_a_tensor_elsewhere_among_plain_addresses(name, monkeypatch):
    """Every argument, Q or not, is looked at where it is a tensor: the host's memory is not handed to a kernel."""
    rows, keys = torch.zeros(2, 3, 10, 64, dtype=torch.bfloat16), torch.zeros(2, 3, 20, 64, dtype=torch.bfloat16)
    tensors = {"Q": rows, "K": keys, "V": keys, "O": rows, "dO": rows, "dQ": rows, "dK": keys, "dV": keys, "lse": torch.zeros(2, 3, 10),
               "kv_len": torch.zeros(2, dtype=torch.int32), "table": torch.zeros(32, 3, dtype=torch.bfloat16),
               "dtable": torch.zeros(32, 3, dtype=torch.bfloat16), "ws": torch.zeros(1 << 20, dtype=torch.uint8)}
    for n in CALLS[name][0].split():
        e = call(name, monkeypatch, 0, **{n: tensors[n]})
        assert e.status == -2 and f" {n} is " in str(e), (n, e)


@pytest.mark.parametrize("name", list(CALLS))
def test_a_workspace_that_is_smaller_than_it_looks(name, monkeypatch):
    e = call(name, monkeypatch, -1, ws=torch.zeros(1, dtype=torch.uint8).expand(1 << 30))
    assert e.status == -2 and " ws is " in str(e)
