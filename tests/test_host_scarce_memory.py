"""Rotated appends, bounds and sparse preds when the host's memory runs out at any of their allocations (CPU only): an error, and nothing has changed."""
import os
import shutil
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, CSRC, ROCM

CHILD = """
import ctypes as C, sys
from paper_2510_25412_amd import binding
lib = binding.load()
near = C.create_string_buffer(32 << 20)
at = (C.addressof(near) + 255) // 256 * 256
lib.memory_left.argtypes = [C.c_int64]
rows, layers = 1 << 45, int(sys.argv[2])
rope, sp = binding.make_rope(), binding.make_sparse(3, 1, 1, rope=binding.make_rope())
call = {"append": lambda ctx, f: lib.sym_kv_append_rope(ctx.h, 2, f, one, rope, None, rows, rows, None),
        "bounds": lambda ctx, f: lib.sym_kv_bounds(ctx.h, 2, f, None),
        "sparse": lambda ctx, f: lib.sym_pred_sparse(ctx.h, 2, f, one, sp, rows, rows, rows, rows, None, None),
        "begin": lambda ctx, f: lib.sym_pred_begin_sparse(ctx.h, 2, f, one, sp, None)}[sys.argv[1]]
one = (C.c_int32 * 2)(1, 2)
state = lambda ctx, f: [(ctx.kv_len(h), ctx.kv_pages(h), ctx.kv_bounded(h)) for h in f] + [ctx.free_pages()]
failed = 0
for n in range(200):
    cfg = binding.make_config(8, 2, 128, 16, "bf16", 400, device=0, pool=1 << 40, workspace=at, workspace_bytes=16 << 20, decode_waves=1, n_layers=layers)
    ctx = binding.Context(cfg)
    assert lib.sym_bounds_attach(ctx.h, 1 << 44, binding.bounds_bytes(cfg)) == 0
    # an append before it has the file system's own lists at their size; the call's rows go to pages that are there
    f = [ctx.kv_open(None), ctx.kv_open(None)]
    ctx.plan_append(f, [300, 700])
    handles = (C.c_int32 * 2)(*f)
    before = state(ctx, f)
    lib.memory_left(n)
    code = call(ctx, handles)
    lib.memory_left(-1)
    after = state(ctx, f)
    if code == 0:
        ctx.lib.sym_pred_end(ctx.h)
        ctx.close()
        break
    failed += 1
    assert code == binding.SYM_ENOSPC and after == before, (n, code, before, after)
    for _ in range(2):                       # and the same call goes through with memory
        assert call(ctx, handles) == 0, ctx.lib.sym_strerror(ctx.h)
        ctx.lib.sym_pred_end(ctx.h)
    ctx.close()
else:
    raise AssertionError("never went through")
print("RESULT", failed)
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(tmp_path_factory.mktemp("scarce") / "libsymphony_kv_scarce.so")
    srcs = [os.path.join(CSRC, f) for f in ("kvfs.cpp", "desc.cpp", "sched.cpp", "capi.cpp")] + [os.path.join(ROOT, "tests", "sanitize", "scarce_memory.cpp")]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", *srcs, "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    return out


@pytest.mark.parametrize("call,layers", [("append", 1), ("append", 3), ("bounds", 1), ("sparse", 1), ("begin", 1), ("begin", 3)])
def test_every_allocation_may_fail(lib, call, layers):
    p = subprocess.run([sys.executable, "-c", CHILD, call, str(layers)], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=lib), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=120)
    assert p.returncode == 0, p.stdout[-3000:]
    assert int(p.stdout.split("RESULT")[1]) >= (1 if call != "bounds" else 0)
