"""Page copies of more than one launch (CPU only): the lists that the launches read, one behind the other, are the call's copies, and no
list is overwritten before the launch that reads it has run.  A launch takes up to 32768 copies, up to 256 in its arguments; four pinned
lists go round."""
import os
import subprocess
import sys

import pytest

from test_host_beams_builds import _plain_build
from test_host_sanitizers import ROOT

CHILD = """
import ctypes as C, sys
import numpy as np
from paper_2510_25412_amd import binding
op, n = sys.argv[1], int(sys.argv[2])
lib = binding.load()
near = C.create_string_buffer(4 << 20)
at = (C.addressof(near) + 255) // 256 * 256
cfg = binding.make_config(8, 2, 128, 16, "bf16", 2 * n + 8, device=0, pool=1 << 40, workspace=at, workspace_bytes=2 << 20, decode_waves=1)
ctx = binding.Context(cfg)
f = ctx.kv_open(None)
if op == "withdraw":
    ctx.plan_append([f], [16 * n - 3])
    assert ctx.kv_pages(f) == list(range(n))
    go = lambda: ctx.pool_withdraw(0, n, None)
    want = [[i, n + i, 16 if i < n - 1 else 13] for i in range(n)]
elif op == "fork":
    ctx.plan_append([f], [7])
    go = lambda: ctx.kv_fork_batch([f] * n, True, None)
    want = [[0, 1 + i, 7] for i in range(n)]
else:                                        # n files take over another, whose last page they copy
    ctx.plan_append([f], [21])
    g = [f] + [ctx.kv_open(None) for _ in range(n)]
    go = lambda: ctx.kv_reorder(g, [-1] + [0] * n, True, None)
    want = [[1, 2 + i, 5] for i in range(n)]
lib.listed_forget()
go()
copies = ctx.last_copies()
assert np.array_equal(copies, want)
read, sizes, by_args = [], [], []
lib.listed_launches.restype = C.c_int64
for i in range(lib.listed_launches()):
    k = lib.listed_copies(C.c_int64(i))
    words = np.empty((k, 3), np.int32)
    lib.listed_words(C.c_int64(i), words.ctypes.data_as(C.c_void_p))
    read.append(words)
    sizes.append(k)
    by_args.append(lib.listed_by_args(C.c_int64(i)))
read = np.concatenate(read)
assert np.array_equal(read[:, 2] & ~256, copies[:, 2]) and np.array_equal(read[:, :2], copies[:, :2])
assert sizes == [min(32768, n - off) for off in range(0, n, 32768)], sizes
assert by_args == [int(k <= 256) for k in sizes], (by_args, sizes)
if op == "withdraw":
    assert ctx.kv_pages(f) == list(range(n, 2 * n)) and ctx.pool_withdrawn() == n
out = (C.c_int64 * 5)()
lib.queued_finish(out)
print("RESULT", out[0])
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return _plain_build(tmp_path_factory.mktemp("listed"), "listed_copies.cpp")


@pytest.mark.parametrize("op,n", [("withdraw", n) for n in (256, 257, 32767, 32768, 32769, 32768 + 256, 32768 + 257, 2 * 32768 + 1000, 5 * 32768 + 7)]
                         + [("fork", 32768 + 100), ("fork", 2 * 32768 + 1000), ("reorder", 32768 + 300)])
def test_copies_of_several_launches(lib, op, n):
    p = subprocess.run([sys.executable, "-c", CHILD, op, str(n)], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=lib), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-4000:]
    assert p.stdout.split("RESULT")[1].split() == ["0"]
