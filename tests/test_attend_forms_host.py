"""The form of decode attention that the library chooses for the problems of attend_forms, so that a rule
that moves does not take a form out of the GPU tests unseen."""
import ctypes
import os
import subprocess

import pytest

import attend_forms
from paper_2609_31395_amd import build

RULES = r"""
#include "actkv_internal.h"
extern "C" int waves(int D, long rows) { return actkv::attend_waves(D, rows); }
extern "C" int side(int Hkv, int D, long rows, long entries) { return actkv::attend_head_waves(Hkv, D, rows, entries); }
extern "C" int direct(int R, int Hkv, int D, long rows, long max_L, long entries, int side, int* heads) {
  return actkv::attend_direct(R, Hkv, D, rows, max_L, entries, false, side, heads);
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, lib = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(RULES)
    subprocess.run([build.hipcc(), "-O1", "-std=c++17", "-fPIC", "-shared", "-I", build.INCLUDE, "-I", build.CSRC, src,
                    "-o", lib], check=True, capture_output=True)
    r = ctypes.CDLL(lib)
    for f in (r.waves, r.side, r.direct):
        f.argtypes = None
    return r


@pytest.mark.parametrize("name", attend_forms.FORMS)
def test_the_form_is_chosen(rules, name):
    f = attend_forms.FORMS[name]
    Hq, H, D = f["heads"]
    rows, long = max(f["tokens"]) * (Hq // H), ctypes.c_long
    side = rules.side(H, D, long(rows), long(sum(f["lens"])))
    heads = ctypes.c_int()
    direct = rules.direct(len(f["lens"]), H, D, long(rows), long(max(f["lens"])), long(sum(f["lens"])), side,
                          ctypes.byref(heads))
    got = (bool(direct), heads.value if direct else side, rules.waves(D, long(rows)))
    assert got == (f["direct"], f["side"], f["waves"])
    if "pieces" in f:   # one KV head: 256 workgroups share the cost, 6 units an item beside its steps
        cost = [6 + -(-m // 32) for m in f["lens"]]
        assert 256 <= 16 * len(cost), "a wave takes a row of the join"
        assert 256 * -(-max(f["lens"]) // 32) // sum(cost) - 1 >= f["pieces"] > 64
