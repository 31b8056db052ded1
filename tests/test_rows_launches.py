"""Chains of launches of the calls on rows by index, without a GPU: what each size launches, and that a launch that fails ends its chain and is told.
(launch_shim.c stands in for the runtime's launch call; pointers are never read.)"""
import json
import os
import subprocess
import sys

import pytest

from launches import _shim

FG_ERR_LAUNCH = 5
F32, BF16 = 0, 1

CHILD = """
import ctypes, json, re, sys
lib = ctypes.CDLL(sys.argv[1])
shim = ctypes.CDLL(None)
shim.shim_name.restype = ctypes.c_char_p
i32, i64, sz, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
P = lambda: ctypes.c_void_p(1 << 20)
big = sz(1 << 50)
def call(kind, a):
    if kind == "sort":
        return lib.fg_index_sort(P(), i64(a["m"]), i64(a["n"]), P(), P(), P(), P(), big, None)
    if kind == "lookup":
        return lib.fg_lookup(P(), i32(a["type"]), i64(a["n"]), i64(a["c"]), i64(a["c"]), P(), i64(a["m"]), f32(2), P(), i64(a["c"]), None)
    if kind == "lookup_backward":
        return lib.fg_lookup_backward(P(), i32(a["type"]), i64(a["m"]), i64(a["c"]), i64(a["c"]), P(), P(), P(), i64(a["n"]), f32(1), i32(a.get("acc", 0)), P(),
                                      i32(0), i64(a["c"]), P(), big, None)
    if kind == "dispatch":
        return lib.fg_dispatch(P(), i32(a["type"]), i64(a["t"]), i64(a["c"]), i64(a["c"]), P(), i32(a["k"]), i64(a["n"]), P(), i64(a["c"]), None)
    if kind == "combine":
        return lib.fg_combine(P(), i32(a["type"]), i64(a["n"]), i64(a["c"]), i64(a["c"]), P(), P(), i64(a["t"]), i32(a["k"]), None, P(), i64(a["c"]), None)
    sort = P() if a["sorted"] else None
    return lib.fg_combine_backward(P(), i32(a["type"]), i64(a["t"]), i64(a["c"]), i64(a["c"]), P(), i64(a["n"]), i64(a["c"]), P(), P(), i32(a["k"]), sort, sort,
                                   sort, P(), i64(a["c"]), P(), P(), big, None)
out = []
for kind, a in json.loads(sys.stdin.read()):
    shim.shim_reset(0)
    status = call(kind, a)
    made = shim.shim_made()
    names = [re.search("k_[a-z_]*[a-z]", shim.shim_name(i).decode()).group() for i in range(made)]
    rows = []
    for fail in range(1, made + 1):
        shim.shim_reset(fail)
        rows.append((fail, call(kind, a), shim.shim_made()))
    out.append((status, names, rows))
print(json.dumps(out))
"""

ROWS_OF_SUMS = ["k_row_sums", "k_row_join"]
PASS = ["k_sort_count", "k_sort_scan", "k_sort_scatter"]
# (the calls, and the kernels that serve them)
CHAINS = {
    "a few entries": (("sort", dict(m=512, n=(1 << 18) - 513)), ["k_sort_few"]),
    "a few entries of more rows": (("sort", dict(m=512, n=(1 << 18) - 512)), ["k_sort_small"]),
    "some entries": (("sort", dict(m=4096, n=(1 << 14) - 4097)), ["k_sort_few"]),
    "some entries, more rows": (("sort", dict(m=1024, n=(1 << 15) - 1025)), ["k_sort_few"]),
    "some entries, still more rows": (("sort", dict(m=1024, n=(1 << 15) - 1024)), ["k_sort_small"]),
    "some entries of more rows": (("sort", dict(m=4096, n=(1 << 14) - 4096)), ["k_sort_small"]),
    "entries that one workgroup sorts": (("sort", dict(m=8192, n=100000)), ["k_sort_small"]),
    "one digit, few counts": (("sort", dict(m=4097, n=1023)), ["k_sort_count", "k_sort_scatter"]),
    "one digit, few tiles": (("sort", dict(m=262144, n=8)), ["k_sort_count", "k_sort_scatter"]),
    "one digit, more tiles": (("sort", dict(m=262145, n=8)), PASS),
    "one digit": (("sort", dict(m=8193 * 4, n=1023)), PASS),
    "two digits, few counts": (("sort", dict(m=65536, n=131072)), ["k_sort_count"] + ["k_sort_scatter"] * 2 + ["k_sort_bounds"]),
    "four digits, few counts": (("sort", dict(m=20000, n=1 << 30)), ["k_sort_count"] + ["k_sort_scatter"] * 4 + ["k_sort_bounds"]),
    "two digits": (("sort", dict(m=65537, n=131072)), PASS * 2 + ["k_sort_bounds"]),
    "two digits, many entries": (("sort", dict(m=1 << 21, n=(1 << 20) - 1)), PASS * 2 + ["k_sort_bounds"]),
    "three digits": (("sort", dict(m=500000, n=1 << 20)), PASS * 3 + ["k_sort_bounds"]),
    "four digits": (("sort", dict(m=500000, n=1 << 30)), PASS * 4 + ["k_sort_bounds"]),
    "lookup": (("lookup", dict(type=BF16, n=1000, c=1024, m=500)), ["k_lookup"]),
    "lookup, narrow rows": (("lookup", dict(type=BF16, n=1000, c=7, m=500)), ["k_lookup"]),
    "lookup, past the caches": (("lookup", dict(type=BF16, n=1000, c=2048, m=1 << 17)), ["k_lookup"]),
    "gradient, few entries": (("lookup_backward", dict(type=BF16, m=1024, c=512, n=5000)), ["k_row_sums_few"]),
    "gradient, few entries of few rows": (("lookup_backward", dict(type=BF16, m=1024, c=512, n=100)), ROWS_OF_SUMS),
    "gradient, few entries of many rows": (("lookup_backward", dict(type=BF16, m=31, c=512, n=500000)), ["k_row_sums"]),
    "gradient, some": (("lookup_backward", dict(type=BF16, m=10000, c=512, n=5000)), ROWS_OF_SUMS),
    "gradient, many": (("lookup_backward", dict(type=F32, m=1 << 20, c=20, n=5000, acc=1)), ["k_row_sums", "k_row_parts", "k_row_join"]),
    "dispatch": (("dispatch", dict(type=F32, t=5000, c=1000, k=4, n=20000)), ["k_dispatch"]),
    "combine": (("combine", dict(type=F32, t=5000, c=1000, k=4, n=20000)), ["k_combine"]),
    "combine of no rows": (("combine", dict(type=F32, t=5000, c=1000, k=4, n=0)), ["k_lookup"]),
    "combine's gradients, rows named once": (("combine_backward", dict(type=BF16, t=5000, c=1000, k=4, n=20000, sorted=0)), ["k_combine_grad"]),
    "combine's gradients, shared rows": (("combine_backward", dict(type=F32, t=900, c=64, k=13, n=900, sorted=1)), ["k_row_sums", "k_row_join"]),
    "combine's gradients, shared rows of many entries": (("combine_backward", dict(type=F32, t=500000, c=64, k=40, n=900, sorted=1)),
                                                         ["k_row_sums", "k_row_parts", "k_row_join"]),
    "combine's gradients, wide shared rows": (("combine_backward", dict(type=F32, t=9000, c=260, k=40, n=9000, sorted=1)),
                                              ["k_row_sums", "k_row_parts", "k_row_join", "k_combine_grad"]),
    "combine's gradients, few wide shared rows": (("combine_backward", dict(type=F32, t=100, c=258, k=4, n=90, sorted=1)), ["k_row_sums_few", "k_combine_grad"]),
}


@pytest.fixture(scope="module")
def answers():
    from paper_2511_10442_amd import binding
    binding.lib()
    r = subprocess.run([sys.executable, "-c", CHILD, binding.LIB_PATH], input=json.dumps([c for c, _ in CHAINS.values()]), capture_output=True, text=True,
                       env=dict(os.environ, LD_PRELOAD=_shim()), timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr
    return dict(zip(CHAINS, json.loads(r.stdout.splitlines()[-1])))


@pytest.mark.parametrize("name", list(CHAINS))
def test_chain(answers, name):
    status, names, rows = answers[name]
    assert status == 0 and names == CHAINS[name][1]
    for fail, status, made in rows:
        assert status == FG_ERR_LAUNCH and made == fail, "launch %d of %d failed: status %d, %d launches" % (fail, len(names), status, made)
