"""The scratch of sparse preds (CPU only): a device that computes nothing looks at what its launches are given.  A batch is taken as long as its lists, its
turned query rows and one token in the fewest parts fit the workspace; what a batch does not use takes no room."""
import os
import shutil
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, CSRC, ROCM

PRELUDE = """
import ctypes as C, random, sys
from paper_2510_25412_amd import binding
lib = binding.load()
near = C.create_string_buffer(200 << 20)
at = (C.addressof(near) + 255) // 256 * 256
lib.scratch_of.argtypes = [C.c_size_t] + [C.c_int64] * 3
kept = []
def context(hq, hkv, dtype, n_pages, bytes, layers=1):
    cfg = binding.make_config(hq, hkv, 128 if dtype == "bf16" else 64, 16, dtype, n_pages, device=0, pool=1 << 40, workspace=at, workspace_bytes=bytes, decode_waves=1, n_layers=layers)
    ctx = binding.Context(cfg)
    kept.append(ctx)
    assert lib.sym_bounds_attach(ctx.h, 1 << 44, binding.bounds_bytes(cfg)) == 0
    lib.scratch_of(at, bytes, hq // hkv, 128 if dtype == "bf16" else 64)
    return ctx
def seen():
    out = (C.c_int64 * 4)()
    lib.scratch_seen(out)
    return list(out)          # sections that lie wrong, attention launches, fewest and most parts of a row's list
rows = 1 << 45
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(tmp_path_factory.mktemp("scratch") / "libsymphony_kv_scratch.so")
    srcs = [os.path.join(CSRC, f) for f in ("kvfs.cpp", "desc.cpp", "sched.cpp", "capi.cpp")] + [os.path.join(ROOT, "tests", "sanitize", "scratch_longcontext.cpp")]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", *srcs, "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]

    def child(code):
        p = subprocess.run([sys.executable, "-c", PRELUDE + code], cwd=ROOT, env=dict(os.environ, SYMPHONY_KV_LIB=out), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert p.returncode == 0, p.stdout[-4000:]
    return child


def test_a_batch_that_fits_with_fewer_parts_is_taken(run):
    # one token, 2 kv heads of 2 query heads, 300 of 700 pages: 5.6 KB of scores, lists of 3 KB, and 2 * 2 * 130 * 4 bytes for each of up to 37 parts
    run("""
want = {}
for kb in (256, 64, 48, 40):
    ctx = context(4, 2, "bf16", 720, kb << 10)
    f = ctx.kv_open(None)
    ctx.plan_append([f], [11195])
    ctx.pred_sparse([f], [1], binding.make_sparse(300, 1, 1), rows, rows, rows, rows, None, None)
    want[kb] = seen()
    assert want[kb][0] == 0 and want[kb][1] == 1 and ctx.kv_len(f) == 11196
assert want[256][2:] == [37, 37] and 20 <= want[64][2] < 37 and 10 <= want[48][2] < want[64][2] and 5 <= want[40][2] < want[48][2]
ctx = context(4, 2, "bf16", 9000, 40 << 10)      # 8700 pages: 70 KB of scores
f = ctx.kv_open(None)
ctx.plan_append([f], [139195])
try:
    ctx.pred_sparse([f], [1], binding.make_sparse(300, 1, 1), rows, rows, rows, rows, None, None)
    raise AssertionError("taken without room for the scores")
except binding.SymError as e:
    assert e.code == binding.SYM_ENOSPC and ctx.kv_len(f) == 139195 and seen()[1] == 0
""")


def test_lists_longer_than_a_workgroup_holds_keep_their_parts(run):
    run("""
for kb, taken in ((4096, True), (64, True), (46, False)):      # 5000 pages read whole: three parts at least, 6.5 KB each, and lists of 20 KB
    ctx = context(8, 1, "f32", 5100, kb << 10)
    f = ctx.kv_open(None)
    ctx.plan_append([f], [79990])
    try:
        ctx.pred_sparse([f], [1], binding.make_sparse(6000, 1, 1), rows, rows, rows, rows, None, None)
        assert taken and seen()[0] == 0 and seen()[2] >= 3, (kb, seen())
    except binding.SymError as e:
        assert not taken and e.code == binding.SYM_ENOSPC, (kb, e)
""")


def test_scores_that_stay_in_a_workgroup_take_no_room(run):
    # 40 tokens of 8 heads, 2000 pages: 64 KB of scores a token, which the attention keeps for itself; 80 KB of turned rows, lists of 10 KB
    run("""
ctx = context(8, 8, "bf16", 2100, 128 << 10)
f = ctx.kv_open(None)
ctx.plan_append([f], [32000])
ctx.pred_sparse([f], [40], binding.make_sparse(16, 1, 1, rope=binding.make_rope()), rows, rows, rows, rows, None, None)
assert seen()[:2] == [0, 1], seen()
""")


@pytest.mark.parametrize("seed", range(3))
def test_sections_of_any_batch_lie_in_the_workspace(run, seed):
    run(f"""
r = random.Random({seed})
done = refused = 0
for _ in range(250):
    dtype, hkv = r.choice(["bf16", "f32"]), r.choice([1, 2, 8])
    layers = r.choice([1, 1, 2])
    try:
        ctx = context(hkv * r.choice([1, 2, 8]), hkv, dtype, 9000, int(2 ** r.uniform(16, 24)), layers)
    except binding.SymError as e:                      # not even the smallest dense batch
        assert e.code == binding.SYM_ENOSPC
        continue
    files = [ctx.kv_open(None) for _ in range(r.choice([1, 1, 3, 40]))]
    lens = [int(2 ** r.uniform(0, 17 if len(files) == 1 else 12)) for _ in files]
    ctx.plan_append(files, lens)
    new = [r.choice([1, 1, 1, int(2 ** r.uniform(0, 7))]) for _ in files]
    sp = binding.make_sparse(int(2 ** r.uniform(1, 13)), 0, 1, rope=r.choice([None, binding.make_rope()]), dense_layers=layers > 1 and r.random() < 0.5)
    before = [ctx.kv_len(f) for f in files]
    try:
        if layers == 1:
            ctx.pred_sparse(files, new, sp, rows, rows, rows, rows, None, None)
        else:
            for _ in range(2):
                ctx.pred_begin_sparse(files, new, sp, None)
                for layer in range(layers):
                    ctx.pred_layer_sparse(layer, rows, rows, rows, rows, None, None)
        done += 1
    except binding.SymError as e:
        assert e.code == binding.SYM_ENOSPC, e
        assert [ctx.kv_len(f) for f in files] in (before, [n + m for n, m in zip(before, new)])
        refused += 1
    assert seen()[0] == 0
    ctx.close()
    kept.clear()
assert done > 100 and refused > 5, (done, refused)
""")
