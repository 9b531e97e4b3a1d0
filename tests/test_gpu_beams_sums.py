"""Normalisers of the choice on the GPU: rows whose sums are whole numbers have to be exact to the last bit of the score, long rows of any
logits within the errors of their sums' steps; and page copies of more than one launch.

Rows of any logits.  A term is exp2(t), t = (x - c) log2 e <= 0: x - c, the constant and the product are off by half a step each, at most 3 * 2^-24 of t,
so the term by 3 ln 2 |t| 2^-24 < 2.1 |t| 2^-24 of itself; when c rises, what was added is scaled by another such power, and all the t of a term add
up to the one that it has at the end.  Weighted by the terms, |t| is at most log2 N for N terms: with weights w = 2^t / S it is the entropy of w less log2 S,
and S >= 1.  Beside that: the power itself, 1 step (2 * 2^-24), a lane's sum of n terms n * 2^-24, and for each of its n / 4 batches (8 of fp32) at most one scaling,
a power and a product, 3 * 2^-24; so for n = a lane's groups of 16 bytes under 2.1 log2 N + 2 + 2 n steps of 2^-24, and one scaling more, 3, where lanes are joined.
The rest is done in 64 bits; the score is rounded to 32 at the end, 2^-24 of it."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import beams as oracle
from paper_2510_25412_amd import binding
from test_gpu_beams import TYPES, U, Files, choose, ctx, make  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [1, 7, 8, 9, 513, 4099, 32768, 40961, 131071, 131072, 1000003])
def test_every_logit_is_counted_once(ctx, dtype, vocab):  # noqa: F811
    # equal logits: each term is 1, each sum a whole number, the score's only errors the logarithm's in 64 bits and its rounding to 32
    print(f"[case] equal logits counted, vocab={vocab} {dtype}", flush=True)
    beams, best = [3, 2], 5
    r = np.random.default_rng(vocab)
    for value in (0.0, -1.25, 96.0):
        x = torch.full((5, vocab), value, dtype=TYPES[dtype], device="cuda")
        s = torch.tensor([-1.0, -3.5, -2.0, 0.0, -100.0], device="cuda")
        masks = [None, r.random((5, vocab)) < 0.5, r.random((5, vocab)) < 3 / vocab]
        for allowed in masks:
            got = choose(ctx, x, s, beams, best, allowed)
            count = np.full(5, vocab) if allowed is None else allowed.sum(1)
            for g, b, row in [(g, b, 3 * g + b) for g in range(2) for b in range(beams[g])]:
                of = got[1][g] == b
                with np.errstate(divide="ignore"):
                    want = float(s[row]) - np.log(float(count[row]))
                assert (np.abs(got[0][g][of].astype(np.float64) - want) <= 1.0001 * U * abs(want)).all(), (value, row, got[0][g][of], want)
            want = oracle.select(x.double().cpu().numpy(), s.double().cpu().numpy(), beams, best, allowed)
            assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])


@pytest.mark.parametrize("dtype,vocab,groups", [("bf16", 131072, 1), ("bf16", 131071, 40), ("f16", 100003, 3), ("f32", 131072, 2), ("f32", 65537, 16)])
@pytest.mark.parametrize("spread", [0.5, 4.0])
def test_sums_of_long_rows(ctx, dtype, vocab, groups, spread):  # noqa: F811
    print(f"[case] sums of {groups} x 4 rows of {vocab} {dtype} spread={spread}", flush=True)
    x, s = make(4 * groups, vocab, dtype, vocab + groups, spread)
    got = choose(ctx, x, s, [4] * groups, 8)
    want = oracle.select(x.double().cpu().numpy(), s.double().cpu().numpy(), [4] * groups, 8)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    # a part has 40960 logits of 16 bits at most, 10240 of fp32 (80 and 40 groups to a lane), and never more than the row
    n = min(math.ceil(vocab / 64 / (4 if dtype == "f32" else 8)), 40 if dtype == "f32" else 80)
    off = np.abs(got[0].astype(np.float64) - want[0])
    assert (off <= U * np.abs(want[0]) + (2.1 * math.log2(vocab) + 2 + 2 * n + 3) * U).all(), off.max()


def test_copies_of_two_launches():
    # 33100 pages out of the pool's lower half: a launch of 32768 copies and one of the rest; and as many forks' last pages
    f = Files(1, 1, pages=70000)
    h = f.open(16 * 33100 - 5)
    before = f.sess.pool.clone()
    f.ctx.pool_withdraw(0, 33100, f.sess.stream)
    torch.cuda.synchronize()
    copies = f.ctx.last_copies()
    assert len(copies) == 33100 and f.ctx.kv_pages(h) == copies[:, 1].tolist() and copies[-1, 2] == 11
    pool, was = f.sess.pool.view(70000, 4, 16, 128), before.view(70000, 4, 16, 128)
    at = torch.from_numpy(copies[:, :2].astype(np.int64)).cuda()
    assert torch.equal(pool[at[:-1, 1]], was[at[:-1, 0]])
    s, d, n = copies[-1].tolist()
    assert torch.equal(pool[d, :, :n], was[s, :, :n]) and torch.equal(pool[d, :, n:], was[d, :, n:])
    rest = torch.ones(70000, dtype=torch.bool, device="cuda")
    rest[at[:, 1]] = False
    assert torch.equal(pool[rest], was[rest])
    f.check([h])
    f.ctx.kv_remove(h)
    f.ctx.pool_return(0, 33100)
    parent = f.open(7)
    before = f.sess.pool.clone()
    new = f.ctx.kv_fork_batch([parent] * 33000, True, f.sess.stream)
    torch.cuda.synchronize()
    copies = f.ctx.last_copies()
    assert len(copies) == 33000 and len(set(copies[:, 1].tolist())) == 33000 and set(copies[:, 2].tolist()) == {7}
    at = torch.from_numpy(copies[:, 1].astype(np.int64)).cuda()
    pool, was = f.sess.pool.view(70000, 4, 16, 128), before.view(70000, 4, 16, 128)
    assert torch.equal(pool[at, :, :7], was[copies[0, 0], :, :7].expand(33000, 4, 7, 128)) and torch.equal(pool[at, :, 7:], was[at, :, 7:])
    f.ctx.kv_remove_batch(new)
    f.sess.close()
