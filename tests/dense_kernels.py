"""Which kernels a call of dense attention launches, from a process in which the HIP runtime's launches are only noted (launch_recorder), and the
smallest problems that reach each of them."""
from __future__ import annotations

import json
import os
import re
import subprocess
import sys

from launch_recorder import ROOT, STUB
from paper_2505_14708_amd import binding as da

NAMES = r"""
extern "C" const char* all_names() {
  static std::string out;
  out.clear();
  for (auto& n : names) out += n.second + "\n";
  return out.c_str();
}
"""
CHILD = r"""
import ctypes, json, sys
stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
stub.launches.restype = stub.all_names.restype = ctypes.c_char_p
sys.path.insert(0, sys.argv[2])
from paper_2505_14708_amd import binding as da
da.lib()
print(json.dumps(stub.all_names().decode().split()), flush=True)
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
    print(json.dumps([[l[0], int(l[1]) * int(l[2])] for l in got]), flush=True)
"""


def kernel(name):
    """("fwd", "bf16", 128, 2, 4, 1, 0) of a mangled name; None for other kernels.  Behind the channels: fwd: sets of 32 queries, waves, waves that
    join, mode (0 single heads, 1 with a bias, 2 several heads' queries as one list); dq and dkv: waves, waves that join, mode; join:
    waves to a row, mode; sum_dq: mode."""
    m = re.match(r"_ZN2da5dense\d+dense_(\w+?)_kernelI(DF16b|f)((?:Li\d+E)*)E", name)
    return m and (m[1], "bf16" if m[2] == "DF16b" else "f32", *(int(x) for x in re.findall(r"Li(\d+)E", m[3])))


def record(tmp_path, problems):
    """(all dense kernels of the library, [[(kernel, workgroups)] of a forward and a backward call]) of problems (dtype, B, H, Hk, N, M, d, rule)."""
    src, out = str(tmp_path / "stub.cpp"), str(tmp_path / "libhipstub.so")
    open(src, "w").write(STUB + NAMES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", src, "-o", out], check=True)
    code = {"f32": da.DA_F32, "bf16": da.DA_BF16}
    lines = "".join(json.dumps([[B, H, N, M, d, Hk, code[dtype]], rule]) + "\n" for dtype, B, H, Hk, N, M, d, rule in problems)
    r = subprocess.run([sys.executable, "-c", CHILD, out, ROOT], input=lines, capture_output=True, text=True, check=True, timeout=120)
    got = [json.loads(l) for l in r.stdout.splitlines()]
    known = {k for k in map(kernel, got[0]) if k}
    return known, [[(kernel(n), w) for n, w in call if kernel(n)] for call in got[1:]]


TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
RULE = (4, 20, 1, 0)
MODES = {"plain": 0, "bias": 1, "packed": 2}


def problem(dtype, d, mode, heads, rows, M):
    """Heads and rows as the kernels see them: two heads of Q to one of K and V, with half of the rows each, where they are one list."""
    if mode == "packed":
        return (dtype, 1, 2 * heads, heads, rows // 2, M, d, None)
    return (dtype, 1, heads, heads, rows, M, d, RULE if mode == "bias" else None)


# heads, rows, keys: what they stand for
SHAPES = {"two sets": (400, 130, 70), "own columns": (200, 100, 140), "joining": (2, 62, 75), "few rows, cut": (2, 4, 3000),
          "cut": (20, 110, 3000), "many rows, cut": (2, 3000, 70), "many rows, few columns": (2, 3000, 20), "heads, many rows": (100, 2100, 65),
          "heads, few columns": (192, 4200, 16), "heads, few rows": (192, 16, 4200), "many heads, few rows": (600, 40, 70)}


def wanted(shape, dtype, d, mode):
    """The kernels that a shape is for."""
    m, two = MODES[mode], dtype == "bf16"
    j = 2 if dtype == "f32" and d == 128 else 4                  # waves that join
    t = (dtype, d)
    few = (4, 1) if t == ("bf16", 128) else (j, j)
    packs = mode != "packed"                                     # (a list of several heads has fewer than 256 rows a head)
    return {"two sets": [("fwd", *t, 2 if two else 1, 4, 1, m), ("dq", *t, 4, 1, m), ("dkv", *t, 4, 1, m)],
            "own columns": [("fwd", *t, 1, 4, 1, m), ("dq", *t, 4, 1, m), ("dkv", *t, 4, 1, m)],
            "joining": [("fwd", *t, 1, j, j, m), ("dq", *t, j, j, m), ("dkv", *t, j, j, m)],
            "few rows, cut": [("fwd", *t, 1, j, j, m), ("join", *t, 4, m), ("dq", *t, j, j, m), ("sum_dq", *t, m)],
            "cut": [("fwd", *t, 1, 4, 1, m), ("join", *t, 1, m), ("dq", *t, 4, 1, m), ("sum_dq", *t, m)],
            "many rows, cut": [("sum_dkv", *t)] if packs else [],
            "many rows, few columns": [("dkv", *t, j, j, m), ("sum_dkv", *t)] if packs else [],
            "heads, many rows": [("fwd", *t, 2 if two else 1, 4, 1, m), ("dkv", *t, 4, 1, m)] if packs else [],
            "heads, few columns": [("dkv", *t, *few, m), ("sum_dkv", *t)] if packs else [],
            "heads, few rows": [("fwd", *t, 1, j, j, m), ("dq", *t, *few, m), ("sum_dq", *t, m)],
            "many heads, few rows": [("fwd", *t, 1, 4, 1, m), ("dq", *t, 4, 1, m)]}[shape]


def cases():
    """(shape, mode, dtype, d) of the shapes that mean something in that mode."""
    return [(s, m, dtype, d) for s in SHAPES for m in MODES for dtype, d in TYPES if wanted(s, dtype, d, m)]
