"""Workgroups that a fork launches, counted on the host: a library in the place of the HIP runtime's
launch configuration records the grids, and no kernel is called."""
import json
import os
import subprocess
import sys

import pytest

from paper_2609_31395_amd import build

SHIM = r"""
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim3_;
static unsigned grids[64][3];
static int n;
int __hipPushCallConfiguration(dim3_ g, dim3_ b, size_t s, void* st) {   /* 1: the kernel is not called */
  (void)b; (void)s; (void)st;
  if (n < 64) { grids[n][0] = g.x; grids[n][1] = g.y; grids[n][2] = g.z; ++n; }
  return 1;
}
int hipGetLastError(void) { return 0; }
int taken(unsigned* to) { for (int i = 0; i < n; ++i) for (int k = 0; k < 3; ++k) to[3 * i + k] = grids[i][k]; int r = n; n = 0; return r; }
"""

CALLS = r"""
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
lib.actkv_fork_pages.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int32] * 6 + [ctypes.c_int64] + [ctypes.c_void_p] * 3 + [
    ctypes.c_int64] + [ctypes.c_void_p] * 2
out = []
for call in json.loads(sys.argv[3]):
    flat = (ctypes.c_int32 * (4 * len(call["forks"])))(*[v for f in call["forks"] for v in f])
    code = lib.actkv_fork_pages(flat, 0x10000, len(call["forks"]), call["rows"], call["stride"], 4, 128, 16, 1 << 24, 0x10000,
                                0x10000, 0x10000, call["free"], 0x10000, None)
    grids = (ctypes.c_uint * 192)()
    n = shim.taken(grids)
    out.append([code, [list(grids[3 * i:3 * i + 3]) for i in range(n)]])
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("shim"))
    src, shim = os.path.join(d, "shim.c"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["gcc", "-O1", "-fPIC", "-shared", src, "-o", shim], check=True)

    def run(*calls):
        r = subprocess.run([sys.executable, "-c", CALLS, shim, build.LIB, json.dumps(calls)], check=True, capture_output=True,
                           text=True)
        return json.loads(r.stdout.splitlines()[-1])
    return run


def forks(n, shared, pages):
    return [[0, 1 + i, shared(i), pages(i)] for i in range(n)]


CASES = {
    "one": (forks(1, lambda i: 5, lambda i: 7), 100),
    "uniform": (forks(64, lambda i: 2187, lambda i: 2188), 2188),
    "all_copied": (forks(8, lambda i: 0, lambda i: 2188), 2188),
    "one_of_many_copied": (forks(256, lambda i: 0 if i == 7 else 2188, lambda i: 2188), 2188),
    "a_long_one_among_short": (forks(5000, lambda i: 0, lambda i: 40000 if i == 0 else 1), 40000),
    "most_forks": (forks(65535, lambda i: 0 if i == 65534 else 1, lambda i: 100000 if i == 65534 else 1), 100000),
}


@pytest.mark.parametrize("name", CASES)
def test_workgroups_of_a_fork_follow_its_work(launches, name):
    f, stride = CASES[name]
    fresh = sum(p - s for _, _, s, p in f)
    # (the forks go to the child in a file's worth of arguments; the largest is cut to what one holds)
    f = f if len(f) <= 5000 else f[:1] + f[-4000:]
    fresh = sum(p - s for _, _, s, p in f)
    [[code, grids]] = launches(dict(forks=f, rows=70000, stride=stride, free=fresh))
    assert code == 0 and len(grids) == 1
    wgs = grids[0][0] * grids[0][1] * grids[0][2]
    needed = len(f) * -(-stride // 1024) + fresh   # 1,024 entries of a row, or a page
    assert needed <= wgs <= needed + needed // 8 + 64
    assert all(g * 256 < 1 << 32 for g in grids[0])


def test_fresh_pages_past_the_page_ids_are_refused(launches):
    big = [[0, 1 + i, 0, 1 << 23] for i in range(257)]
    got = launches(dict(forks=big, rows=300, stride=1 << 23, free=1 << 40), dict(forks=big, rows=300, stride=1 << 23, free=5),
                   dict(forks=big[:255], rows=300, stride=1 << 23, free=1 << 40))
    assert [c for c, _ in got] == [-2, -4, 0]
    assert [len(g) for _, g in got] == [0, 0, 1]


@pytest.mark.parametrize("n", [1, 2, 64, 1000, 5000])
@pytest.mark.parametrize("most", [1, 3, 50])
def test_at_most_half_of_the_copying_workgroups_are_idle(launches, n, most):
    f = forks(n, lambda i: 60 - (i * 7919) % (most + 1), lambda i: 60)
    fresh = sum(p - s for _, _, s, p in f)
    [[code, grids]] = launches(dict(forks=f, rows=70000, stride=60, free=fresh))
    assert code == 0 and len(grids) == 1
    assert n + fresh <= grids[0][0] * grids[0][1] <= n + 2 * fresh + 64
