"""A pool's rotary table that could not be set up whole is not there: later calls try again, none takes a part of it for
the table. Without a GPU: the runtime's allocations and copies are stood in for, and end where the test says."""
import os
import subprocess
import sys

from paper_2510_18546_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNTIME = r"""
#include <stddef.h>
int mallocs = 0, copies = 0, held = 0;                 /* how many more of them work; blocks that are held */
int hipMalloc(void **p, size_t n)
{
    (void)n;
    *p = NULL;
    if (mallocs-- <= 0)
        return 2;
    ++held;
    *p = (void *)0x100000;
    return 0;
}
int hipFree(void *p) { held -= p != NULL; return 0; }
int hipMemcpy(void *to, const void *from, size_t n, int kind)
{
    (void)to, (void)from, (void)n, (void)kind;
    return copies-- > 0 ? 0 : 1;
}
"""

CALLS = """
import ctypes, sys
runtime = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
from paper_2510_18546_amd import binding as B
lib = B.load()
count = lambda name: ctypes.c_int.in_dll(runtime, name)
P = 0x10000
for mallocs, copies in ((1, 0), (2, 0), (2, 1)):
    pool = B.kv_pool_create(None, None, [30, 5], 4, 1e4, 4096, dtype=B.EN_BF16, shape=(2, 2, 40, 64), k_ptr=0x1000, v_ptr=0x2000)
    plan = B.segment_select(pool, [0, 1], [0, 1, 2], 20)
    attend = lambda: B.STATUS[lib.segmented_tree_attention(pool.handle, plan.handle, 4, P, P, P, P, P, P, P, P, P, 1 << 40, None)]
    gather = lambda: B.STATUS[lib.gather_rope(pool.handle, plan.handle, P, P, P, P, None)]
    for call in (attend, gather):
        count("mallocs").value, count("copies").value = mallocs, copies
        print(call(), lib.en_last_error().decode(), count("held").value, sep="|")
        count("mallocs").value = 0                     # from here on nothing is to be had, for the plan's block neither
        print(call(), lib.en_last_error().decode(), count("held").value, sep="|")
    pool.close()
"""


def test_a_table_that_was_not_set_up_whole_is_not_there(tmp_path):
    B.load()
    (tmp_path / "runtime.c").write_text(RUNTIME)
    so = str(tmp_path / "runtime.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", so, str(tmp_path / "runtime.c")], check=True)
    got = subprocess.run([sys.executable, "-c", CALLS, so], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert got.returncode == 0, got.stderr
    lines = [line.split("|") for line in got.stdout.splitlines()]
    assert len(lines) == 12
    for status, text, held in lines:
        assert status == "EN_ERR_DEVICE" and "rotary table" in text and held == "0", (status, text, held)
