"""The host half of the beams' calls (CPU only) under sanitizers, and with a device that is always behind: no list of copies may be
overwritten before the launch that reads it has run."""
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


@pytest.fixture(scope="module")
def queued_lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(tmp_path_factory.mktemp("queued") / "libsymphony_kv_queued.so")
    srcs = [os.path.join(CSRC, f) for f in ("kvfs.cpp", "desc.cpp", "sched.cpp", "capi.cpp")] + [os.path.join(ROOT, "tests", "sanitize", "queued_beams.cpp")]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", *srcs, "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    return out


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
