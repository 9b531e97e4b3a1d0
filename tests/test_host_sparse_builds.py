"""The host half of rotated appends, page bounds and sparse preds (CPU only) under sanitizers, and with a device that is always behind: no
staging buffer may be overwritten before the launch that reads it has run."""
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
    p = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_host_sparse.py"), "-x", "-q", "-s", "-p", "no:cacheprovider",
                        "-k", "not rope_rows"], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert p.returncode == 0 and "runtime error" not in p.stdout and "Sanitizer" not in p.stdout and " passed" in p.stdout, p.stdout[-4000:]


CHILD = """
import ctypes as C, random, sys
from paper_2510_25412_amd import binding
seed, blind = int(sys.argv[1]), sys.argv[2] == "blind"
lib = binding.load()
near = C.create_string_buffer(96 << 20)
at = (C.addressof(near) + 255) // 256 * 256
lib.queued_be_blind(blind)
r, layers = random.Random(seed), 1 + 2 * (seed % 2)
cfg = binding.make_config(8, 2, 128, 16, "bf16", 6000, device=0, pool=at, workspace=at, workspace_bytes=64 << 20, decode_waves=256, n_layers=layers)
ctx, files = binding.Context(cfg), []
assert lib.sym_bounds_attach(ctx.h, at, binding.bounds_bytes(cfg)) == 0
rope = binding.make_rope()
for step in range(300):
    op = r.choice(["append", "append", "sparse", "sparse", "sparse", "bounds", "fork", "dense", "rows", "cut"])
    live = r.sample(files, min(len(files), r.randint(1, 12)))
    new = [r.choice([1, 1, 2, 40]) for _ in live]
    if op == "append" or not files:
        if len(files) < 30:
            files.append(ctx.kv_open(None))
        some = r.sample(files, r.randint(1, len(files)))
        ctx.kv_append_rope(some, [r.choice([1, 17, 90, 2100 if ctx.free_pages() > 3000 else 3]) for _ in some], r.choice([rope, None]), at, at, None, None)
    elif op == "sparse":
        sp = binding.make_sparse(r.choice([2, 9, 100]), 0, 1, rope=r.choice([rope, None]), dense_layers=layers > 1 and r.random() < 0.5)
        if layers == 1:
            ctx.pred_sparse(live, new, sp, at, at, at, at, None, None)
        else:
            ctx.pred_begin_sparse(live, new, sp, None)
            for layer in range(layers):
                (ctx.pred_layer if sp.dense_layers and layer == 1 else ctx.pred_layer_sparse)(layer, at, at, at, at, stream=None)
    elif op == "bounds":
        ctx.kv_bounds(live, None)
    elif op == "dense" and layers == 1:
        ctx.pred_batch(live, new, at, at, at, at, None)
    elif op == "rows":
        lib.sym_rope_rows(ctx.h, rope, 5, at, at + (1 << 20), at + (1 << 20), None, None, None)
    elif op == "fork":
        files.append(ctx.kv_fork(live[0]))
    elif op == "cut":
        ctx.kv_truncate([live[0]], [r.randint(0, ctx.kv_len(live[0]))])
    while ctx.free_pages() < 1500 or len(files) > 34:
        ctx.kv_remove(files.pop(0))
    for f in files:
        assert 0 <= ctx.kv_bounded(f) <= ctx.kv_len(f) // 16
out = (C.c_int64 * 5)()
lib.queued_finish(out)
print("RESULT", *out)
"""


@pytest.fixture(scope="module")
def queued_lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(tmp_path_factory.mktemp("queued") / "libsymphony_kv_queued.so")
    srcs = [os.path.join(CSRC, f) for f in ("kvfs.cpp", "desc.cpp", "sched.cpp", "capi.cpp")] + [os.path.join(ROOT, "tests", "sanitize", "queued_longcontext.cpp")]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", *srcs, "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    return out


def _run(lib, *args):
    p = subprocess.run([sys.executable, "-c", CHILD, *map(str, args)], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=lib), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-4000:]
    return list(map(int, [x for x in p.stdout.splitlines() if x.startswith("RESULT")][-1].split()[1:]))


@pytest.mark.parametrize("seed", range(4))
def test_no_staging_buffer_is_overwritten_before_it_is_read(queued_lib, seed):
    overwritten, launches, _, waits, _ = _run(queued_lib, seed, "waits")
    assert launches > 400 and waits > 50 and overwritten == 0


def test_a_wait_that_does_not_wait_is_noticed(queued_lib):
    assert _run(queued_lib, 0, "blind")[0] > 0
