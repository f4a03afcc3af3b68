"""Attention to an encoder's states and attention with a relative position bias: what is refused, sizes, the bucket rule compiled for the CPU,
and the launches of problems at the ends of the range, without a GPU."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

from dense_util import bucket
from launch_recorder import ROOT, STUB
from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.skipif(not os.path.exists(da.LIB_PATH), reason="library not built")
FAKE = 0x10000


def _status(fn, *a, **kw):
    with pytest.raises(da.DaError) as e:
        fn(*a, **kw)
    return e.value.status


def _calls(p, bias, layouts=None, **change):
    """Status of the forward and the backward call with addresses that nobody follows; `change` replaces single ones."""
    a = dict(Q=FAKE, K=FAKE, V=FAKE, table=FAKE, O=FAKE, ws=FAKE, kv_len=FAKE, lse=FAKE, dO=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, dtable=FAKE)
    a.update(change)
    kw = dict(kv_len=a["kv_len"], layouts=layouts, stream=0)
    if bias is None:
        return (_status(da.da_cross_attn, p, a["Q"], a["K"], a["V"], a["O"], a["ws"], lse=a["lse"], **kw),
                _status(da.da_cross_attn_bwd, p, a["Q"], a["K"], a["V"], a["O"], a["lse"], a["dO"], a["dQ"], a["dK"], a["dV"], a["ws"], **kw))
    return (_status(da.da_bias_attn, p, bias, a["Q"], a["K"], a["V"], a["table"], a["O"], a["ws"], lse=a["lse"], **kw),
            _status(da.da_bias_attn_bwd, p, bias, a["Q"], a["K"], a["V"], a["table"], a["O"], a["lse"], a["dO"], a["dQ"], a["dK"], a["dV"],
                    a["dtable"], a["ws"], **kw))


def test_structs_match_the_header():
    assert ctypes.sizeof(da.da_attn_problem) == 40 and da.da_attn_problem.scale.offset == 32
    assert ctypes.sizeof(da.da_attn_layouts) == 8 * 24 and ctypes.sizeof(da.da_rel_bias) == 16 and ctypes.sizeof(da.da_attn_dims) == 16


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -2), (dict(H=0), -2), (dict(Hk=0), -2), (dict(Hk=3), -2), (dict(Hk=8), -2), (dict(N=0), -2), (dict(M=0), -2),
    (dict(N=-1), -2), (dict(d=0), -2), (dict(dtype=2), -2), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(scale=1e-31), -2), (dict(scale=1e31), -2),
    (dict(N=(1 << 29) + 1), -2), (dict(M=(1 << 29) + 1), -2), (dict(N=1 << 29, H=8, Hk=4), -2), (dict(B=1 << 30, H=4), -2),
    (dict(d=96), -3), (dict(d=256), -3), (dict(d=32), -3)])
def test_problems_that_are_refused(change, status):
    a = dict(B=2, H=4, N=10, M=20, d=64, Hk=4)
    a.update(change)
    p = da.attn_problem(a.pop("B"), a.pop("H"), a.pop("N"), a.pop("M"), a.pop("d"), **a)
    assert _status(da.da_attn_sizes, p) == status
    assert _calls(p, None) == (status, status)
    assert _calls(p, da.rel_bias(32, 128)) == (status, status)


@pytest.mark.parametrize("rule", [(0, 128, 1, 0), (1, 128, 0, 0), (2, 128, 1, 0), (33, 128, 1, 0), (258, 1024, 1, 0), (257, 1024, 0, 0),
                                  (32, 8, 1, 0), (32, 16, 0, 0), (32, 1025, 1, 0), (32, 128, 2, 0), (32, 128, -1, 0), (32, 128, 1, (1 << 29) + 1),
                                  (32, 128, 1, -(1 << 29) - 1), (-32, 128, 1, 0)])
def test_rules_that_are_refused(rule):
    p = da.attn_problem(1, 2, 10, 10, 64)
    assert _status(da.da_attn_sizes, p, da.da_rel_bias(*rule)) == -2
    assert _calls(p, da.da_rel_bias(*rule)) == (-2, -2)


def test_pointers_that_are_refused():
    p, r = da.attn_problem(1, 2, 10, 10, 64), da.rel_bias(32, 128)
    for bias in (None, r):
        for name in ("Q", "K", "V", "O"):
            assert _calls(p, bias, **{name: None}) == (-1, -1)
            assert _calls(p, bias, **{name: FAKE + 8}) == (-5, -5)
        assert _calls(p, bias, lse=FAKE + 4) == (-5, -5) and _calls(p, bias, kv_len=FAKE + 4) == (-5, -5)
    assert _calls(p, r, table=None) == (-1, -1) and _calls(p, r, table=FAKE + 2) == (-5, -5)
    L, P, N = da.lib(), ctypes.byref(p), None
    back = [FAKE] * 3 + [N] + [FAKE] * 6 + [FAKE, 1 << 40, N]     # Q K V kv_len O lse dO dQ dK dV ws
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9, 10):
        assert L.da_cross_attn_bwd(P, N, *[N if j == i else x for j, x in enumerate(back)]) == -1, i
        if i != 10:
            assert L.da_cross_attn_bwd(P, N, *[FAKE + 8 if j == i else x for j, x in enumerate(back)]) == -5, i
    assert L.da_bias_attn(P, N, N, *[FAKE] * 4, N, FAKE, N, FAKE, 1 << 40, N) == -1           # no rule
    assert L.da_attn_sizes(P, N, N) == -1 and L.da_attn_sizes(N, N, ctypes.byref(da.da_attn_dims())) == -1


def test_workspaces_that_are_refused():
    p = da.attn_problem(1, 2, 10, 9000, 64)
    sz, L, P, V = da.da_attn_sizes(p), da.lib(), ctypes.byref(p), ctypes.c_void_p
    assert sz.forward_ws > 0 and sz.backward_ws > 0
    f = [FAKE] * 3 + [None, FAKE, None]
    assert L.da_cross_attn(P, None, *f, FAKE, sz.forward_ws - 1, None) == -4
    assert L.da_cross_attn(P, None, *f, None, sz.forward_ws, None) == -1
    assert L.da_cross_attn(P, None, *f, FAKE + 16, sz.forward_ws, None) == -5
    b = [FAKE] * 3 + [None] + [FAKE] * 6
    assert L.da_cross_attn_bwd(P, None, *b, FAKE, sz.backward_ws - 1, None) == -4


def test_layouts_that_are_refused():
    B, H, N, M, d = 2, 3, 10, 20, 64
    p = da.attn_problem(B, H, N, M, d)
    good = dict(stride_b=H * N * d, stride_h=d, stride_n=H * d)

    def calls(name, **change):
        l = da.da_layout(**dict(good, **change))
        return _calls(p, None, da.attn_layouts(**{name: l}), ws=FAKE + 16)       # gets as far as the workspace (-5) where nothing is wrong
    for name in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
        rows = M if name in ("k", "v", "dk", "dv") else N
        assert calls(name, stride_n=d - 8, stride_b=10 ** 6) == (-2, -2)
        assert calls(name, stride_h=0) == (-2, -2) and calls(name, stride_b=-64) == (-2, -2)
        assert calls(name, stride_h=d + 4, stride_b=10 ** 6) == (-5, -5)
        assert calls(name, stride_n=1 << 52) == (-2, -2)
        if name in ("o", "dq", "dk", "dv"):
            assert calls(name, stride_b=10 ** 6, stride_n=d) == (-2, -2)                # heads and rows in one place
            assert calls(name, stride_b=H * rows * d - d) == (-2, -2)
    one = da.attn_problem(1, 1, 1, 1, d)                                                # strides of extents of 1 do not matter
    l = da.attn_layouts(**{n: da.da_layout(0, 3, 1) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")})
    assert _calls(one, None, l, Q=None) == (-1, -1)


def test_tensors_that_are_refused():
    """The binding looks at tensors before it hands their addresses on (no GPU: tensors of the CPU are on no device of the library's)."""
    import torch
    p = da.attn_problem(1, 1, 4, 4, 64)
    t = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    for bad in (t.float(), t[:, :, :2], t.transpose(2, 3), t):
        with pytest.raises(da.DaError if torch.cuda.is_available() else Exception):
            da.da_cross_attn(p, bad, bad, bad, bad, None)


def test_sizes():
    """Nothing where there is nothing to join; the same with and without lengths and layouts (they are not asked for)."""
    assert da.da_attn_sizes(da.attn_problem(1, 40, 75600, 512, 128)).forward_ws == 0
    a = da.da_attn_sizes(da.attn_problem(4, 32, 1, 32768, 128, Hk=8))
    assert 0 < a.forward_ws < 1 << 28
    b = da.da_attn_sizes(da.attn_problem(1, 24, 118800, 512, 128))
    assert 2 * 24 * 118800 * 4 <= b.backward_ws < 1 << 30


def test_bucket_rule(tmp_path):
    """rel_buckets.h against integer arithmetic, at every distance."""
    src, out = tmp_path / "b.cpp", str(tmp_path / "b")
    src.write_text("""
#include <stdio.h>
#include "rel_buckets.h"
int main() {
  int n, m, w;
  while (scanf("%d %d %d", &n, &m, &w) == 3) {
    da::RelRule t;
    if (!da::make_rel_rule(n, m, w, &t)) { printf("refused\\n"); continue; }
    printf("%d", t.cut);
    for (int r = -1100; r <= 1100; ++r) printf(" %d", da::rel_bucket(t, r));
    printf("\\n");
  }
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2505_14708_amd", "csrc"), str(src), "-o", out], check=True)
    rules = [(2, 2, 0), (4, 2, 1), (3, 5, 0), (7, 20, 0), (8, 1000, 1), (16, 64, 1), (32, 128, 0), (32, 128, 1), (32, 20, 0), (64, 1024, 1), (256, 1024, 0),
             (256, 129, 0), (256, 1024, 1), (12, 96, 1), (10, 486, 0)]
    got = subprocess.run([out], input="\n".join("%d %d %d" % r for r in rules), capture_output=True, text=True, check=True).stdout.splitlines()
    for rule, line in zip(rules, got):
        x = [int(v) for v in line.split()]
        want = [bucket(r, *rule) for r in range(-1100, 1101)]
        assert x[1:] == want, rule
        cut = x[0]
        assert cut <= rule[1] and len(set(want[:1100 - cut + 1])) == 1            # one bucket from `cut` on
        if rule[2]:
            assert len(set(want[1100 + cut:])) == 1


CHILD = r"""
import ctypes, json, sys
stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
stub.launches.restype = ctypes.c_char_p
sys.path.insert(0, sys.argv[2])
from paper_2505_14708_amd import binding as da
for line in sys.stdin:
    a, rule = json.loads(line)
    p = da.attn_problem(*a[:5], Hk=a[5], dtype=a[6])
    x = [(i + 1) << 20 for i in range(10)]
    r = None if rule is None else da.rel_bias(*rule)
    if r is None:
        da.da_cross_attn(p, *x[:4], x[4], stream=0)
        da.da_cross_attn_bwd(p, *x[:10], x[4], stream=0)
    else:
        da.da_bias_attn(p, r, *x[:5], x[5], stream=0)
        da.da_bias_attn_bwd(p, r, *x[:10], x[0], x[4], stream=0)
    got = [l.split() for l in stub.launches().decode().splitlines()]
    print(json.dumps([[l[0], [int(v) for v in l[1:4]], [int(v) for v in l[4:7]], int(l[7])] for l in got]), flush=True)
"""


def test_grids_stay_within_the_launch_limits(tmp_path):
    src, out = str(tmp_path / "stub.cpp"), str(tmp_path / "libhipstub.so")
    open(src, "w").write(STUB)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", src, "-o", out], check=True)
    cases = []
    for dtype in (da.DA_F32, da.DA_BF16):
        for d in (64, 128):
            for B, H, N, M, Hk in ((1, 1, 1, 1, 1), (1, 40, 118800, 512, 40), (8, 64, 1, 100000, 8), (1 << 20, 64, 1, 1, 64), (1, 1 << 25, 1, 1, 1 << 25), (1, 1, 1 << 29, 3, 1),
                                   (1, 1, 3, 1 << 29, 1), (2, 8, 4096, 4096, 2), (30000, 1, 700, 700, 1)):
                cases += [((B, H, N, M, d, Hk, dtype), None), ((B, H, N, M, d, Hk, dtype), (256, 1024, 0, 0))]
    r = subprocess.run([sys.executable, "-c", CHILD, out, ROOT], input="\n".join(json.dumps(c) for c in cases), capture_output=True, text=True,
                       check=True, timeout=120)
    lines = r.stdout.splitlines()
    assert len(lines) == len(cases)
    for case, line in zip(cases, lines):
        launches = json.loads(line)
        assert len(launches) >= 3, case
        for name, grid, group, lds in launches:
            assert all(0 < n * g < 1 << 32 for n, g in zip(grid, group)), (name, grid, group, case)
            assert max(grid[1:]) <= 65535 and lds <= 80 * 1024, (name, grid, lds)
