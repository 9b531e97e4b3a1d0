"""The choice among a row's scores, round by round on the host (CPU only): scores that are not finite, the ends of the range of whole numbers,
places past the end of the scores."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import longcontext as lc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ is not installed")
    out = str(tmp_path_factory.mktemp("choice") / "choice_rounds.so")
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{os.path.join(ROOT, 'paper_2510_25412_amd', 'csrc')}",
           os.path.join(ROOT, "tests", "sanitize", "choice_rounds.cpp"), "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    lib = C.CDLL(out)
    lib.choice_pick.restype, lib.choice_pick.argtypes = C.c_int64, [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_void_p]
    lib.choice_range.argtypes = [C.c_uint32, C.c_uint32]
    return lib


def order_of(x):
    """Scores as whole numbers of the same order, NaN above all (as the kernel writes them)."""
    x = np.asarray(x, np.float32) + np.float32(0)
    b = x.view(np.uint32)
    return np.where(np.isnan(x), np.uint32(0xffffffff), np.where(b >> 31, ~b, b | np.uint32(0x80000000))).astype(np.uint32)


def picked(lib, scores, want, fill):
    keys = np.ascontiguousarray(order_of(scores))
    out = np.full(len(keys) + fill, -1, np.int32)
    n = lib.choice_pick(keys.ctypes.data, len(keys), fill, want, out.ctypes.data)
    assert n >= 0, n
    return out[:n].tolist()


def wanted(scores, want):
    return [p - 1 for p in lc.choose(np.concatenate([[0], scores, [0]]).astype(np.float32), len(scores) + 2, want + 2, 1, 1)[1:-1]]


@pytest.mark.parametrize("special", [float("inf"), float("nan"), -float("inf"), 3.4e38, -3.4e38, 2.0e38])
@pytest.mark.parametrize("pages,some,want", [(100, 20, 7), (240, 50, 30), (100, 99, 1), (64, 64, 63), (37, 2, 1), (2, 1, 1), (500, 3, 3), (500, 3, 4), (500, 4, 3)])
def test_more_pages_of_an_extreme_score_than_are_wanted(lib, special, pages, some, want):
    r = np.random.default_rng(pages)
    scores = (10 * r.standard_normal(pages)).astype(np.float32)
    scores[r.permutation(pages)[:some]] = special
    for fill in (0, 1, 300):
        assert picked(lib, scores, want, fill) == wanted(scores, want)


@pytest.mark.parametrize("seed", range(8))
def test_mixtures(lib, seed):
    r = np.random.default_rng(seed)
    for _ in range(250):
        pages = int(r.integers(2, 400))
        scores = (r.choice([1e-3, 1.0, 1e30]) * r.standard_normal(pages)).astype(np.float32)
        for special in (float("inf"), float("nan"), -float("inf"), 3.4e38, -3.4e38, 0.0, -0.0):
            if r.random() < 0.4:
                scores[r.random(pages) < r.choice([0.02, 0.3, 0.9])] = special
        want = int(r.integers(1, pages))
        assert picked(lib, scores, want, int(r.integers(0, 300))) == wanted(scores, want)


def test_every_step_of_a_range_lies_inside_it(lib):
    # ends near every power of two, and near both ends of the whole numbers
    ends = sorted({min(max((1 << b) + d, 1), 0xffffffff) for b in range(33) for d in (-257, -256, -255, -2, -1, 0, 1, 2, 255, 256, 257)} |
                  {0xffffffff - (1 << b) for b in range(32)} | {0xff800000, 0xff7fffff, 0x007fffff, 0x00800000})
    for i, lo in enumerate(ends):
        for hi in ends[i:]:
            assert lib.choice_range(lo, hi) == 0, (hex(lo), hex(hi))
