"""Entry points where host memory runs out: a status, no exception through the C interface (which ends the process).
Each in a process of its own whose address space may hardly grow."""

from __future__ import annotations

import subprocess
import sys

import pytest

pytest.importorskip("torch")

CHILD = """
import ctypes as C, resource, sys
import numpy as np
from paper_2608_25523_amd import binding as B
L = B.LIB
many = 2 ** 31 - 1
zero, one = np.zeros(2, np.int32), np.zeros(1, np.int32)
ptr = lambda x: x.ctypes.data_as(C.POINTER(C.c_int32))
at = lambda i: C.c_void_p(1 << 40 | i << 20)
free = B.Allocator(64 << 20)
ids = free.alloc(3)
size = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (size + (48 << 20),) * 2)
out = C.c_void_p()

def plan():
    pool = B.pfx_pool(many, 16, 1, 64, None, None)
    pt, b = B.pfx_prefix_table(0, ptr(zero), ptr(zero), ptr(zero)), B.pfx_batch(0, *[ptr(zero)] * 5)
    return L.pfx_plan_create(C.byref(pool), C.byref(pt), C.byref(b), 1, 3, None, C.byref(out))

def pool(n):
    return B.pfx_pool(n, 16, 1, 64, at(1), at(2))

def pool8(n):
    return B.pfx_pool8(n, 16, 1, 64, at(1), at(2), at(3))

def copy(call, d, s):
    return call(C.byref(d), C.byref(s), ptr(one), ptr(one), 1, at(4), 4096, None)

calls = dict(
    plan=plan,
    allocator=lambda: L.pfx_alloc_create(many, C.byref(out)),
    free=lambda: L.pfx_free_pages(free.h, ids.ctypes.data_as(C.c_void_p), 3),
    page_copy=lambda: copy(L.pfx_page_copy, pool(many), pool(1)),
    page_copy8=lambda: copy(L.pfx_page_copy8, pool8(many), pool8(1)),
    page_dequantize=lambda: copy(L.pfx_page_dequantize, pool(many), pool8(1)),
)
for name in sys.argv[1:]:
    rc = calls[name]()
    print(name, rc, B.pfx_last_error(), flush=True)
    assert rc == B.PFX_ENOMEM and "host allocation failed" in B.pfx_last_error()
    assert not out.value
assert free.num_free() == (64 << 20) - 3
"""


@pytest.mark.parametrize("name", ["plan", "allocator", "free", "page_copy", "page_copy8", "page_dequantize"])
def test_a_status_where_memory_runs_out(name):
    r = subprocess.run([sys.executable, "-c", CHILD, name],
                       capture_output=True, text=True, timeout=120, cwd=__file__.rsplit("/tests/", 1)[0])
    assert r.returncode == 0, (r.returncode, r.stdout[-500:], r.stderr[-1500:])


def test_page_copy_refuses_negative_page_counts():
    import ctypes as C

    import numpy as np

    from paper_2608_25523_amd import binding as B
    ids = np.zeros(1, np.int32).ctypes.data_as(C.c_void_p)
    at = [C.c_void_p(1 << 40 | i << 20) for i in range(3)]
    for d, s in ((-1, 1), (1, -1)):
        pools = [B.pfx_pool(n, 16, 1, 64, at[0], at[1]) for n in (d, s)]
        rc = B.LIB.pfx_page_copy(C.byref(pools[0]), C.byref(pools[1]), ids, ids, 1, at[2], 4096, None)
        assert rc == B.PFX_ERANGE, B.pfx_last_error()
