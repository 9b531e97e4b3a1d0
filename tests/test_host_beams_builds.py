"""The host half of the beams' calls (CPU only) under sanitizers, with a device that is always behind: no list of copies may be overwritten
before the launch that reads it has run, and with memory that runs out: an error, and nothing has changed."""
import os
import shutil
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, CSRC, ROCM, _build, _runtime


@pytest.mark.skipif(_runtime("libasan.so") is None, reason="g++ with libasan is not installed")
def test_host_half_under_address_and_undefined_behavior_sanitizers(tmp_path):
    lib = _build(str(tmp_path), "asan", ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined"])
    runtime = _runtime("libasan.so")
    env = dict(os.environ, SYMPHONY_KV_LIB=lib, LD_PRELOAD=runtime + (":" + os.environ["LD_PRELOAD"] if os.environ.get("LD_PRELOAD") else ""),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    p = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_host_beams.py"), "-x", "-q", "-s", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert p.returncode == 0 and "runtime error" not in p.stdout and "Sanitizer" not in p.stdout and " passed" in p.stdout, p.stdout[-4000:]


CHILD = """
import ctypes as C, random, sys
import numpy as np
from paper_2510_25412_amd import binding
seed, blind = int(sys.argv[1]), sys.argv[2] == "blind"
lib = binding.load()
near = C.create_string_buffer(96 << 20)
at = (C.addressof(near) + 255) // 256 * 256
lib.queued_be_blind(blind)
r, layers = random.Random(seed), 1 + 2 * (seed % 2)
cfg = binding.make_config(8, 2, 128, 16, "bf16", 9000, device=0, pool=at, workspace=at, workspace_bytes=64 << 20, decode_waves=256, n_layers=layers)
ctx, files, out = binding.Context(cfg), [], 0
files = [ctx.kv_open(None) for _ in range(4)]
for f in files:
    ctx.kv_append(f, 1000 + f, at, at, None)
for step in range(300):
    op = r.choice(["fork", "fork", "reorder", "reorder", "reorder", "withdraw", "withdraw", "pred", "select"])
    if op == "fork":
        files += [int(h) for h in ctx.kv_fork_batch([r.choice(files) for _ in range(r.choice([3, 300, 700]))], True, None)]
        if len(files) > 1500:
            ctx.kv_remove_batch(files[4:1200])
            files = files[:4] + files[1200:]
    elif op == "reorder":
        some = r.sample(files, min(len(files), r.choice([4, 300, 900])))
        ctx.kv_reorder(some, [r.randrange(len(some)) for _ in some], True, None)
    elif op == "withdraw":
        first = r.choice([0, 4500])
        if ctx.free_pages() > 5000:
            ctx.pool_withdraw(first, 4500, None)
            ctx.pool_return(first, 4500)
    elif op == "pred" and layers == 1:
        live = r.sample(files, 4)
        ctx.pred_batch(live, [1] * 4, at, at, at, at, None)
    elif op == "select":
        beams = np.array([2, 3], np.int32)
        plan = (binding.SymBeamState * 1)(binding.SymBeamState(at, at, 1, 0, 100, 100))
        assert lib.sym_beam_states(ctx.h, 2, beams.ctypes.data_as(C.POINTER(C.c_int32)), 5, at + (1 << 20), 1, plan, None) == 0
out = (C.c_int64 * 5)()
lib.queued_finish(out)
print("RESULT", *out)
"""


def _plain_build(folder, device):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(folder / "libsymphony_kv_host.so")
    srcs = [os.path.join(CSRC, f) for f in ("kvfs.cpp", "desc.cpp", "sched.cpp", "capi.cpp")] + [os.path.join(ROOT, "tests", "sanitize", device)]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", *srcs, "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    return out


@pytest.fixture(scope="module")
def queued_lib(tmp_path_factory):
    return _plain_build(tmp_path_factory.mktemp("queued"), "queued_beams.cpp")


@pytest.fixture(scope="module")
def scarce_lib(tmp_path_factory):
    return _plain_build(tmp_path_factory.mktemp("scarce"), "scarce_beams.cpp")


def _run(lib, seed, mode):
    p = subprocess.run([sys.executable, "-c", CHILD, str(seed), mode], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=lib), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-4000:]
    line = [x for x in p.stdout.splitlines() if x.startswith("RESULT")][-1]
    return dict(zip(("overwritten", "launches", "records", "waits", "most_unrecorded"), map(int, line.split()[1:])))


@pytest.mark.parametrize("seed", range(4))
def test_no_list_of_copies_is_overwritten_before_it_is_read(queued_lib, seed):
    r = _run(queued_lib, seed, "true")
    assert r["launches"] > 150 and r["waits"] > 20            # the ring of four came round again and again
    assert r["overwritten"] == 0


def test_a_wait_that_does_not_wait_is_noticed(queued_lib):
    assert _run(queued_lib, 0, "blind")["overwritten"] > 0


SCARCE = """
import ctypes as C, sys
from paper_2510_25412_amd import binding
lib = binding.load()
near = C.create_string_buffer(32 << 20)
at = (C.addressof(near) + 255) // 256 * 256
lib.memory_left.argtypes = [C.c_int64]
op, n_files = sys.argv[1], int(sys.argv[2])
def call(ctx, some, out):
    n = len(some)
    h = (C.c_int32 * n)(*some)
    if op == "fork": return lib.sym_kv_fork_batch(ctx.h, n, h, 1, out, None)
    if op == "reorder": return lib.sym_kv_reorder(ctx.h, n, h, (C.c_int32 * n)(*[(i + 1) % n for i in range(n)]), 1, None)
    if op == "remove": return lib.sym_kv_remove_batch(ctx.h, n, h)
    return lib.sym_pool_withdraw(ctx.h, 0, 300, None)
failed = 0
for n in range(5000):
    cfg = binding.make_config(8, 2, 128, 16, "bf16", 3000, device=0, pool=1 << 40, workspace=at, workspace_bytes=16 << 20, decode_waves=1)
    ctx = binding.Context(cfg)
    files = [ctx.kv_open(None) for _ in range(3)]
    ctx.plan_append(files, [300, 5, 700])
    files += [ctx.kv_fork(files[i % 3]) for i in range(n_files)]
    every = range(3 * len(files) + 4)
    def one(h):
        try:
            return ctx.kv_len(h), ctx.kv_pages(h)
        except binding.SymError:
            return None
    state = lambda: [one(h) for h in every] + [ctx.free_pages(), ctx.pool_withdrawn()]
    before, out = state(), (C.c_int32 * len(files))()
    lib.memory_left(n)
    code = call(ctx, files, out)
    lib.memory_left(-1)
    if code == 0:
        ctx.close()
        break
    failed += 1
    assert code == binding.SYM_ENOSPC and state() == before, (n, code)
    assert call(ctx, files, out) == 0, ctx.lib.sym_strerror(ctx.h)       # and the same call goes through with memory
    if op == "fork":                         # with the handles that it would have given at first
        assert sorted(out) == list(range(max(files) + 1, max(files) + 1 + len(files))), list(out)
        files += list(out)
    if op != "remove":
        ctx.kv_remove_batch(files)
    assert ctx.free_pages() + ctx.pool_withdrawn() == 3000
    ctx.close()
else:
    raise AssertionError("never went through")
print("RESULT", failed)
"""


@pytest.mark.parametrize("op,files", [("fork", 4), ("fork", 70), ("fork", 300), ("reorder", 4), ("reorder", 300), ("remove", 4), ("remove", 130), ("withdraw", 4), ("withdraw", 300)])
def test_every_allocation_may_fail(scarce_lib, op, files):
    p = subprocess.run([sys.executable, "-c", SCARCE, op, str(files)], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=scarce_lib), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-3000:]
    assert int(p.stdout.split("RESULT")[1]) >= 1
