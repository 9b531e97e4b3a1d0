"""Beams on the GPU: choices against the definition in 64 bits, state rows, files that are forked, reordered and moved, and all of
them together in a search.

Tolerance of a score: its rounding to 32 bits, 2^-24 of it, and the normaliser's error.  Every exponent is (x - c) log2 e <= 0 with c the
largest so far: two roundings of 2^-24 of the exponent's size t, 1 ulp of the exponential and as much for every step of c, weighted by 2^-t; t 2^-t <=
0.54, so together under 4 * 2^-24 of the sum, and the sum of n values in 32 bits adds at most n * 2^-24, n = a lane's octets of a part plus 3."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import beams as oracle
from paper_2510_25412_amd import binding, driver, synth

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    sess = driver.HipSession(synth.Shape(8, 8, 128, 16, "bf16"), 4, None, "cuda:0", max_lips=1, max_tokens=64, max_entries=64)
    yield sess.ctx
    sess.close()


def stream():
    return torch.cuda.current_stream().cuda_stream


def words_of(allowed):
    """Truth values [rows, vocab] as int32 words; bits behind the vocabulary are set: nobody may look at them."""
    a = np.concatenate([allowed, np.ones((len(allowed), -allowed.shape[1] % 32), bool)], 1)
    return torch.from_numpy(np.packbits(a, axis=1, bitorder="little").view(np.int32).copy()).cuda()


def choose(ctx, logits, scores, beams, best, allowed=None, words=None, guard=True):
    """The library's choice; every output stands between guards that have to stay."""
    n = len(beams) * best
    out = [torch.full((n + 16,), v, dtype=t, device="cuda") for v, t in ((7.5, torch.float32), (77, torch.int32), (77, torch.int32))]
    size = binding.beam_scratch_bytes(beams, logits.shape[1], best)
    scratch = torch.full((size + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    if allowed is not None and words is None:
        words = words_of(allowed)
    ctx.beam_select(beams, best, logits, scores, *[o[8:8 + n] for o in out], scratch[:size], words, stream())
    torch.cuda.synchronize()
    for o, v in zip(out, (7.5, 77, 77)):
        assert (o[:8] == v).all() and (o[8 + n:] == v).all()
    assert (scratch[size:] == 0xAB).all()
    return [o[8:8 + n].view(len(beams), best).cpu().numpy() for o in out]


def compare(got, logits, scores, beams, best, allowed=None):
    want = oracle.select(logits.double().cpu().numpy(), scores.double().cpu().numpy(), beams, best, allowed)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    none = want[1] < 0
    assert (got[0][none] == -np.inf).all()
    n = math.ceil(logits.shape[1] / 512) + 3
    off = np.abs(got[0].astype(np.float64)[~none] - want[0][~none])
    assert (off <= U * np.abs(want[0][~none]) + (4 + n) * U).all(), off.max(initial=0)


def make(rows, vocab, dtype, seed, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn((rows, vocab), generator=g)).to(TYPES[dtype]).cuda(), (-20 * torch.rand((rows,), generator=g)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 15, 16, 31, 33, 255, 511, 512, 513, 2047, 2048, 2049, 4100, 16391])
def test_choices_at_every_ragged_end(ctx, dtype, vocab):
    print(f"[case] select vocab={vocab} {dtype}", flush=True)
    beams = [1, 4, 3]
    x, s = make(8, vocab, dtype, vocab)
    for best in (1, 5, 8, 33):
        compare(choose(ctx, x, s, beams, best), x, s, beams, best)
        allowed = np.random.default_rng(vocab + best).random((8, vocab)) < 0.4
        compare(choose(ctx, x, s, beams, best, allowed), x, s, beams, best, allowed)


@pytest.mark.parametrize("beams,vocab,best,dtype", [([64], 3001, 128, "f32"), ([1] * 600, 1000, 2, "bf16"), ([16] * 5, 20011, 32, "f16"), ([8, 1, 64, 2], 9001, 64, "f32"),
                                                    ([4], 131072, 8, "bf16"), ([2] * 3000, 700, 4, "f32"), ([5], 65537, 100, "f32"), ([64] * 70, 1500, 17, "f32")])
def test_choices_of_every_shape(ctx, beams, vocab, best, dtype):
    print(f"[case] select {len(beams)} groups vocab={vocab} best={best} {dtype}", flush=True)
    x, s = make(sum(beams), vocab, dtype, best)
    compare(choose(ctx, x, s, beams, best), x, s, beams, best)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [5, 300, 5000, 40000])
def test_equal_logits(ctx, dtype, vocab):
    # every logit the same, few values, one row like another: the lowest beam and token
    print(f"[case] equal logits vocab={vocab} {dtype}", flush=True)
    beams, rows = [3, 2], 5
    flat = torch.full((rows, vocab), 1.25, dtype=TYPES[dtype], device="cuda")
    same = torch.full((rows,), -3.0, device="cuda")
    steps = torch.randint(0, 3, (rows, vocab), generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]).cuda()
    alike = make(1, vocab, dtype, 3)[0].expand(rows, vocab).contiguous()
    zeros = torch.where(torch.rand((rows, vocab), generator=torch.Generator().manual_seed(2)) < 0.5, 0.0, -0.0).to(TYPES[dtype]).cuda()
    for x in (flat, steps, alike, zeros):
        for best in (1, 8, 70, 128):
            got = choose(ctx, x, same, beams, best)
            if x is steps and len({tuple(r) for r in x.float().softmax(-1).double().cpu().numpy()}) > 1:
                # rows' normalisers differ; the order of equal scores within a row is what is looked at
                compare(got, x, same, beams, best)
            else:
                compare(got, x, same, beams, best)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("best", [8, 100, 128])
def test_many_equals_in_few_places(ctx, dtype, best):
    # rows 0..6 of a group have their largest logits in the first 512 of 40960, where a sixteenth of the threads look; then 640 places of one
    # row that a sixth of them have looked at, among equal smaller ones
    print(f"[case] equals in few places best={best} {dtype}", flush=True)
    x = torch.full((64, 40960), -1.0, dtype=TYPES[dtype], device="cuda")
    x[:7, :512] = 3
    s = torch.full((64,), -2.0, device="cuda")
    compare(choose(ctx, x, s, [64], best), x, s, [64], best)
    y = torch.full((1, 131072), -1.0, dtype=TYPES[dtype], device="cuda")
    part = y.view(64, 4, 64, 8)
    part[0::8, 0, :, 0] = 3
    part[1::8, 0, :16, 0] = 3
    compare(choose(ctx, y, s[:1], [1], best), y, s[:1], [1], best)


def test_equal_rows_at_unlike_addresses(ctx):
    # rows of an odd number of logits begin at every alignment: their scores have to be equal to the bit
    row = make(1, 4099, "bf16", 5)[0]
    x = row.expand(16, 4099).contiguous()
    s = torch.full((16,), -2.0, device="cuda")
    got = choose(ctx, x, s, [16], 32)
    compare(got, x, s, [16], 32)
    assert len(set(got[0][0, :16])) == 1 and got[1][0, :16].tolist() == list(range(16))


@pytest.mark.parametrize("order", ["up", "down", "saw", "peaks"])
def test_sorted_rows(ctx, order):
    # the value that leaves about as many as wanted is a guess: rows where all of the largest lie with one lane, or behind one another
    vocab = 30011
    v = torch.arange(vocab, dtype=torch.float32)
    x = {"up": v / 1000, "down": (vocab - v) / 1000, "saw": (v % 512) + v / vocab, "peaks": torch.where((v % 2048) < 8, 20 + v / vocab, -v / vocab)}[order].expand(4, vocab).contiguous().cuda()
    s = torch.tensor([-1.0, -2.5, -2.0, -0.5], device="cuda")
    for best in (1, 4, 16, 64, 128):
        compare(choose(ctx, x, s, [4], best), x, s, [4], best)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_values_that_are_not_finite(ctx, dtype):
    print(f"[case] not finite {dtype}", flush=True)
    vocab, rows, beams = 3000, 12, [12]
    x, s = make(rows, vocab, dtype, 9)
    low = torch.finfo(TYPES[dtype]).min
    x[0, 100], x[1, 5], x[2] = float("nan"), float("inf"), -math.inf
    x[3, ::2], x[4, 1:], x[5] = low, low, low
    x[6, :], x[6, 17] = -math.inf, 2.0
    s[7], s[8], s[9], s[10] = -math.inf, math.inf, float("nan"), -1e30
    compare(choose(ctx, x, s, beams, 20), x, s, beams, 20)
    # the same in places that are not allowed changes nothing
    allowed = np.random.default_rng(0).random((rows, vocab)) < 0.5
    allowed[4] = False
    clean, _ = make(rows, vocab, dtype, 10)
    dirty = clean.clone()
    bad = torch.from_numpy(~allowed).cuda()
    for k, v in enumerate((float("nan"), float("inf"), -math.inf, low, torch.finfo(TYPES[dtype]).max)):
        dirty[k::5] = torch.where(bad[k::5], torch.tensor(v, dtype=TYPES[dtype], device="cuda"), dirty[k::5])
    a, b = choose(ctx, clean, s, beams, 20, allowed), choose(ctx, dirty, s, beams, 20, allowed)
    compare(a, clean, s, beams, 20, allowed)
    assert all(np.array_equal(p, q) for p, q in zip(a, b))


def test_masks_that_leave_little_or_nothing(ctx):
    vocab, rows = 50021, 8
    x, s = make(rows, vocab, "f16", 12)
    allowed = np.zeros((rows, vocab), bool)
    for i, n in enumerate([0, 1, 2, 7, 20, 600, vocab - 1, vocab]):
        allowed[i, np.random.default_rng(i).permutation(vocab)[:n]] = True
    for beams in ([8], [1] * 8, [5, 3]):
        for best in (1, 8, 16, 100):
            compare(choose(ctx, x, s, beams, best, allowed), x, s, beams, best, allowed)
    first, last = np.zeros((2, rows, vocab), bool)
    first[:, 0] = last[:, -1] = True
    for a in (first, last):
        compare(choose(ctx, x, s, [8], 10, a), x, s, [8], 10, a)


def test_rows_that_lie_apart(ctx):
    x, s = make(6, 1203, "bf16", 20)
    far = torch.full((6, 1500), float("nan"), dtype=torch.bfloat16, device="cuda")
    far[:, 3:1206] = x
    allowed = np.random.default_rng(3).random((6, 1203)) < 0.5
    wide = torch.zeros((6, 60), dtype=torch.int32, device="cuda")
    wide[:, 5:43] = words_of(allowed)
    compare(choose(ctx, far[:, 3:1206], s, [2, 4], 9), x, s, [2, 4], 9)
    compare(choose(ctx, far[:, 3:1206], s, [2, 4], 9, allowed, wide[:, 5:43]), x, s, [2, 4], 9, allowed)
    shared = words_of(allowed[:1]).expand(6, 38)              # one mask for all rows has to be written out
    with pytest.raises(ValueError):
        choose(ctx, x, s, [2, 4], 9, allowed, shared)


def test_many_requests_of_unlike_widths(ctx):
    # more than travel with a launch
    beams = np.random.default_rng(6).integers(1, 6, 700).tolist()
    x, s = make(sum(beams), 300, "bf16", 60)
    s[torch.rand(len(s), generator=torch.Generator().manual_seed(1)).cuda() < 0.4] = -math.inf      # some requests have no beam left
    compare(choose(ctx, x, s, beams, 6), x, s, beams, 6)


def test_the_largest_vocabulary(ctx):
    for dtype in ("bf16", "f32"):
        print(f"[case] largest vocabulary {dtype}", flush=True)
        x, s = make(2, 1 << 24, dtype, 61)
        x[1, -1], x[0, 0] = 30.0, 29.0
        compare(choose(ctx, x, s, [2], 5), x, s, [2], 5)


@pytest.mark.parametrize("rows,vocab,dtype,beams,best", [(1060, 131071, "bf16", 4, 8), (528, 131072, "f32", 4, 8), (2050, 65536, "f16", 5, 40)])
def test_logits_beyond_the_last_level_cache(ctx, rows, vocab, dtype, beams, best):
    print(f"[case] {rows} rows of {vocab} {dtype}", flush=True)
    x, s = torch.empty((rows, vocab), dtype=TYPES[dtype], device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3)).mul_(2.5), -20 * torch.rand(rows, device="cuda")
    groups = rows // beams
    got = choose(ctx, x, s, [beams] * groups, best)
    for g in [0, 1, groups // 2, groups - 1]:
        at = slice(g * beams, (g + 1) * beams)
        compare([o[g:g + 1] for o in got], x[at], s[at], [beams], best)


def test_two_calls_at_once(ctx):
    # on two streams, with scratch of their own
    jobs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for k in range(2):
        x, s = make(64, 30011 + k, "bf16", 70 + k)
        jobs.append((x, s, [torch.empty((16, 8), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)],
                     torch.empty(binding.beam_scratch_bytes([4] * 16, 30011 + k, 8), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, s, out, scratch), st in zip(jobs, streams):
            ctx.beam_select([4] * 16, 8, x, s, *out, scratch, None, st.cuda_stream)
    torch.cuda.synchronize()
    for x, s, out, _ in jobs:
        compare([o.cpu().numpy() for o in out], x, s, [4] * 16, 8)


def test_far_rows(ctx):
    # row offsets beyond 2^32 bytes, and beyond 2^31 elements
    stride, rows = 1 << 29, 6
    big = torch.empty((rows - 1) * stride + 1000, dtype=torch.float32, device="cuda")
    view = torch.as_strided(big, (rows, 1000), (stride, 1))
    x, s = make(rows, 1000, "f32", 30)
    view.copy_(x)
    compare(choose(ctx, view, s, [6], 12), x, s, [6], 12)


def test_scores_far_from_zero(ctx):
    # logits around 1e5: the normaliser is as exact as the logits are
    x, s = make(4, 6000, "f32", 31, spread=3.0)
    x += 1e5
    got = choose(ctx, x, s, [4], 8)
    compare(got, x, s, [4], 8)


def test_binding_refuses(ctx):
    x, s = make(4, 100, "bf16", 1)
    out = [torch.empty((1, 8), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    scratch = torch.empty(binding.beam_scratch_bytes([4], 100, 8), dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.SymError):                     # as many rows as beams
        ctx.beam_select([3], 8, x, s, *out, scratch, None, stream())
    for bad in [dict(logits=x[:1].expand(4, 100)), dict(logits=x.t().contiguous().t()), dict(logits=x.double()), dict(scores=s[:3]), dict(scores=s.double()), dict(scores=s.int()), dict(best=9),
                dict(allowed=torch.zeros((4, 3), dtype=torch.int32, device="cuda")), dict(allowed=torch.zeros((3, 4), dtype=torch.int32, device="cuda")),
                dict(allowed=torch.zeros((4, 4), device="cuda"))]:
        a = dict(dict(beams=[4], best=8, logits=x, scores=s, allowed=None), **bad)
        with pytest.raises((ValueError, TypeError)):
            ctx.beam_select(a["beams"], a["best"], a["logits"], a["scores"], *out, scratch, a["allowed"], stream())


# ---- state rows ---------------------------------------------------------------------------------

def moved(x, parents, beams, dim):
    """x with row r replaced by its parent's, where that is one."""
    at, row = [], 0
    for b in beams:
        at += [row + (p if 0 <= p < b else r) for r, p in enumerate(parents[row:row + b])]
        row += b
    return x.index_select(dim, torch.tensor(at, device=x.device))


@pytest.mark.parametrize("beams", [[4], [1, 2, 3], [8, 5], [16, 9], [32, 17, 1], [64, 33]])
@pytest.mark.parametrize("inplace", [True, False])
def test_state_rows(ctx, beams, inplace):
    print(f"[case] states {beams} inplace={inplace}", flush=True)
    rows, r = sum(beams), np.random.default_rng(len(beams) + 2 * inplace)
    parents = np.concatenate([r.integers(-2, b + 2, b) for b in beams])
    parents[-1] = 2 ** 31 - 1
    dev = torch.from_numpy(parents.astype(np.int32)).cuda()
    g = torch.Generator().manual_seed(rows)
    shapes = [((rows, 517), 0), ((3, rows, 40), 1), ((2, 2, rows, 5, 7), 2), ((rows,), 0), ((rows, 4096), 0), ((rows, 0), 0), ((1, rows, 1), 1), ((5, rows, 33000), 1), ((rows, 3), 0)]
    types = [torch.int32, torch.bfloat16, torch.int8, torch.int64, torch.float32, torch.int8, torch.int8, torch.int16, torch.uint8]
    xs = [torch.randint(-100, 100, s, generator=g).to(t).cuda() for (s, _), t in zip(shapes, types)]
    want = [moved(x, parents, beams, d) if x.numel() else x.clone() for x, (_, d) in zip(xs, shapes)]
    out = xs if inplace else [torch.full_like(x, 55) for x in xs]
    before = [x.clone() for x in xs]
    ctx.beam_states(beams, dev, binding.make_states([(o, x, d) for o, x, (_, d) in zip(out, xs, shapes)]), stream())
    torch.cuda.synchronize()
    for i, (o, w) in enumerate(zip(out, want)):
        assert torch.equal(o, w), i
    if not inplace:
        assert all(torch.equal(x, b) for x, b in zip(xs, before))


def test_state_rows_of_odd_places(ctx):
    # rows that begin anywhere, with others' bytes between them
    beams, parents = [3, 2], [2, 0, 0, 1, 0]
    dev = torch.tensor(parents, dtype=torch.int32, device="cuda")
    for width in (1, 15, 16, 17, 31, 4095, 4111):
        for gap in (0, 1, 9):
            buf = torch.randint(0, 255, (2, 5, width + gap), dtype=torch.uint8, generator=torch.Generator().manual_seed(width)).cuda()
            flat = torch.full((buf.numel() + 40,), 9, dtype=torch.uint8, device="cuda")
            view = flat[3:3 + buf.numel()].view(buf.shape)
            view.copy_(buf)
            want = buf.clone()
            want[:, :, :width] = moved(buf[:, :, :width].contiguous(), parents, beams, 1)
            ctx.beam_states(beams, dev, binding.make_states([(view[:, :, :width], view[:, :, :width], 1)]), stream())
            torch.cuda.synchronize()
            assert torch.equal(view, want) and (flat[:3] == 9).all() and (flat[3 + buf.numel():] == 9).all(), (width, gap)


def test_many_groups_and_long_rows(ctx):
    r = np.random.default_rng(5)
    beams = r.integers(1, 5, 1300)
    rows = int(beams.sum())
    parents = np.concatenate([r.integers(0, b, b) for b in beams])
    x = torch.randint(-1000, 1000, (2, rows, 130), dtype=torch.int32, device="cuda")
    want = moved(x, parents, beams, 1)
    ctx.beam_states(beams, torch.from_numpy(parents.astype(np.int32)).cuda(), binding.make_states([(x, x, 1)]), stream())
    assert torch.equal(x, want)
    x = torch.randint(-128, 127, (3, 3 << 24), dtype=torch.int8, device="cuda")            # a row of two stretches of columns
    y = x.clone()
    ctx.beam_states([3], torch.tensor([1, 2, 0], dtype=torch.int32, device="cuda"), binding.make_states([(y, y, 0)]), stream())
    assert torch.equal(y, x[[1, 2, 0]])
    x = torch.randint(-128, 127, (1300, 900001), dtype=torch.int8, device="cuda")          # many groups of rows that are cut, and of an odd length
    p = torch.from_numpy(np.tile([1, 0], 650).astype(np.int32)).cuda()
    y = x.clone()
    ctx.beam_states([2] * 650, p, binding.make_states([(y, y, 0)]), stream())
    assert torch.equal(y.view(650, 2, -1)[:, 0], x.view(650, 2, -1)[:, 1]) and torch.equal(y.view(650, 2, -1)[:, 1], x.view(650, 2, -1)[:, 0])
    del x, y
    x = torch.randint(-1000, 1000, (700, 8, 70000), dtype=torch.int16, device="cuda")      # an outer dimension that is cut
    y = torch.empty_like(x)
    ctx.beam_states([2] * 4, p[:8], binding.make_states([(y, x, 1)] * 1 + [(x[:, :, :0], x[:, :, :0], 1)]), stream())
    assert torch.equal(y[:, 0::2], x[:, 1::2]) and torch.equal(y[:, 1::2], x[:, 0::2])
    del x, y
    far = torch.empty((5, 3, 1 << 30), dtype=torch.int8, device="cuda")                    # an array beyond 2^32 bytes, strides too
    view = far[:, :, :1000]
    view.copy_(torch.randint(-128, 127, (5, 3, 1000), dtype=torch.int8, device="cuda"))
    want = view[:, [2, 2, 1]].clone()
    ctx.beam_states([3], torch.tensor([2, 2, 1], dtype=torch.int32, device="cuda"), binding.make_states([(view, view, 1)]), stream())
    assert torch.equal(view, want)


def test_plans_of_states_are_checked(ctx):
    x = torch.zeros((4, 8, 6), device="cuda")
    for bad in [[(x, x[:, :4], 1)], [(x, x.half(), 1)], [(x.transpose(1, 2), x.transpose(1, 2), 0)], [(x, x, 1), (x[:, :4].contiguous(), x[:, :4].contiguous(), 1)]]:
        with pytest.raises(ValueError):
            binding.make_states(bad)
    plan = binding.make_states([(x, x, 1)])
    for beams, parents, error in [([7], torch.zeros(7, dtype=torch.int32, device="cuda"), ValueError), ([8], torch.zeros(7, dtype=torch.int32, device="cuda"), ValueError),
                                  ([7], torch.zeros(8, dtype=torch.int32, device="cuda"), binding.SymError)]:
        with pytest.raises(error):
            ctx.beam_states(beams, parents, plan, stream())
    with pytest.raises(TypeError):
        ctx.beam_states([8], torch.zeros(8, device="cuda"), plan, stream())


# ---- files ----------------------------------------------------------------------------------------

class Files:
    """A session over a poisoned pool, with every file's rows on the host."""

    def __init__(self, Hkv=2, layers=1, dtype="bf16", pages=400, order=None, Hq=None):
        D = 128 if dtype == "bf16" else 64
        self.t, self.layers, self.Hkv, self.D = TYPES[dtype], layers, Hkv, D
        self.sess = driver.HipSession(synth.Shape(Hq or Hkv, Hkv, D, 16, dtype), pages, order, "cuda:0", max_lips=300, max_tokens=4096, max_entries=1 << 14, poison=True, n_layers=layers)
        self.ctx, self.rows, self.g = self.sess.ctx, {}, torch.Generator().manual_seed(Hkv + 10 * layers)

    def append(self, h, n):
        k, v = (torch.randn((self.layers, n, self.Hkv, self.D), generator=self.g).to(self.t).cuda() for _ in range(2))
        if n:
            self.ctx.kv_append(h, n, k, v, self.sess.stream)
            torch.cuda.synchronize()
        old = self.rows.get(h)
        self.rows[h] = (k, v) if old is None else tuple(torch.cat(p, 1) for p in zip(old, (k, v)))

    def open(self, n):
        h = self.ctx.kv_open(None)
        self.append(h, n)
        return h

    def check(self, files):
        for h in files:
            for layer in range(self.layers):
                want = [x[layer] for x in self.rows[h]]
                assert self.ctx.kv_len(h) == len(want[0])
                if not len(want[0]):
                    continue
                got = [torch.empty_like(x) for x in want]
                self.ctx.kv_read(h, 0, len(want[0]), *got, self.sess.stream, layer=layer)
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want)), (h, layer)

    def untouched(self, copies, before):
        """The pool is what it was but for the copies' filled slots."""
        pool = self.sess.pool.view(self.layers, -1, 4 * self.Hkv, 16, 128)
        want = before.view(pool.shape).clone()
        for s, d, n in copies.tolist():
            want[:, d, :, :n] = before.view(pool.shape)[:, s, :, :n]
        assert torch.equal(pool, want)


@pytest.mark.parametrize("Hkv,layers,dtype", [(1, 1, "bf16"), (2, 3, "f32"), (3, 1, "bf16"), (8, 2, "bf16"), (5, 1, "f32"), (12, 1, "bf16")])
def test_forked_and_reordered_files(Hkv, layers, dtype):
    print(f"[case] files Hkv={Hkv} layers={layers} {dtype}", flush=True)
    f = Files(Hkv, layers, dtype)
    parents = [f.open(n) for n in (1, 15, 16, 17, 40, 0)]
    take = [0, 1, 1, 2, 3, 3, 3, 4, 5]
    before = f.sess.pool.clone()
    new = f.ctx.kv_fork_batch([parents[i] for i in take], True, f.sess.stream)
    for h, i in zip(new, take):
        f.rows[int(h)] = f.rows[parents[i]]
    f.untouched(f.ctx.last_copies(), before)
    assert sorted(f.ctx.last_copies()[:, 2].tolist()) == [1, 1, 1, 1, 8, 15, 15]
    f.check(parents + new.tolist())
    for h, n in zip(new, (1, 2, 17, 1, 1, 30, 1, 8, 5)):              # they grow apart
        f.append(int(h), n)
    kv = [int(h) for h in new]
    r = np.random.default_rng(Hkv)
    for _ in range(4):
        src = r.integers(-1, len(kv), len(kv))
        before = f.sess.pool.clone()
        f.ctx.kv_reorder(kv, src, True, f.sess.stream)
        old = {h: f.rows[h] for h in kv}
        f.rows.update({h: old[kv[s]] if s >= 0 else old[h] for h, s in zip(kv, src)})
        f.untouched(f.ctx.last_copies(), before)
        f.check(parents + kv)
        for h in kv:
            f.append(h, int(r.integers(1, 20)))
        f.check(parents + kv)
    assert f.ctx.get_stats()["cow_copies"] >= 7
    f.ctx.kv_remove_batch(kv + parents)
    assert f.ctx.free_pages() == 400
    f.sess.close()


def test_more_copies_than_travel_with_a_launch():
    # 32, 256 and more: the list in the arguments, in more of them, in pinned memory
    f = Files(1, 2, pages=1500)
    parent = f.open(7)
    for n in (32, 33, 256, 257, 600):
        before = f.sess.pool.clone()
        launches = f.ctx.get_stats()["kernel_launches"]
        new = f.ctx.kv_fork_batch([parent] * n, True, f.sess.stream)
        assert f.ctx.get_stats()["kernel_launches"] == launches + 1
        f.untouched(f.ctx.last_copies(), before)
        f.rows.update({int(h): f.rows[parent] for h in new})
        f.check(new[[0, n // 2, n - 1]].tolist())
        f.ctx.kv_remove_batch(new)
    f.sess.close()


@pytest.mark.parametrize("Hkv,layers,dtype,scatter", [(1, 1, "f32", False), (2, 3, "bf16", True), (8, 1, "bf16", True), (3, 2, "f32", False)])
def test_withdrawn_pages(Hkv, layers, dtype, scatter):
    print(f"[case] withdraw Hkv={Hkv} layers={layers} {dtype}", flush=True)
    pages = 160
    order = np.random.default_rng(1).permutation(pages).astype(np.int32) if scatter else None
    f = Files(Hkv, layers, dtype, pages, order)
    files = [f.open(n) for n in (300, 17, 1, 500, 64)]
    child = f.ctx.kv_fork(files[0])
    f.rows[child] = f.rows[files[0]]
    short = f.ctx.kv_fork(files[3])                           # sees fewer tokens of a page than another
    f.ctx.kv_truncate([short], [490])
    f.rows[short] = tuple(x[:, :490] for x in f.rows[files[3]])
    bounds = torch.full((layers, pages, Hkv, 2, f.D), 9.0, dtype=f.t, device="cuda")
    f.ctx.bounds_attach(bounds)
    f.ctx.kv_bounds(files, f.sess.stream)
    live = files + [child, short]

    def bounds_hold():
        for h in files:
            for i, p in enumerate(f.ctx.kv_pages(h)[:f.ctx.kv_bounded(h)]):
                k = f.rows[h][0][:, 16 * i:16 * i + 16]
                assert torch.equal(bounds[:, p, :, 0], k.amin(1)) and torch.equal(bounds[:, p, :, 1], k.amax(1))

    f.check(live)
    for first, n in [(0, 40), (100, 60), (40, 1), (41, 0)]:
        before = f.sess.pool.clone()
        f.ctx.pool_withdraw(first, n, f.sess.stream)
        f.untouched(f.ctx.last_copies(), before)
        assert not any(first <= p < first + n for h in live for p in f.ctx.kv_pages(h))
        f.sess.pool.view(layers, pages, -1)[:, first:first + n] = 0xFF      # the caller's now
        f.check(live)
        bounds_hold()
        assert [f.ctx.kv_bounded(h) for h in files] == [f.ctx.kv_len(h) // 16 for h in files]
        for h in files:
            if f.ctx.free_pages() > 8:
                f.append(h, 5)
        f.check(live)
        f.ctx.pool_return(first, n)
        f.ctx.kv_bounds(files, f.sess.stream)
    f.sess.close()


def test_a_large_pool_moves_and_waiting_files_with_it():
    f = Files(2, 1, pages=2400)
    files = [f.open(n) for n in (9000, 5000, 3300)]
    f.ctx.kv_offload([files[1]], f.sess.stream)
    shared = f.ctx.kv_fork(files[2])
    f.rows[shared] = f.rows[files[2]]
    f.ctx.kv_offload([files[2]], f.sess.stream)               # its pages stay: another file has them
    f.ctx.pool_withdraw(0, 1200, f.sess.stream)
    assert len(f.ctx.last_copies()) > binding_args()
    f.check([files[0], shared])
    f.ctx.pool_return(0, 1200)
    f.ctx.kv_restore(files[1:], f.sess.stream)
    f.check(files + [shared])
    f.sess.close()


def binding_args():
    return 256              # copies that travel with a launch


def test_refused_while_a_batch_is_open_and_in_a_capture():
    f = Files(8, 2, Hq=8)
    h = f.open(20)
    other = f.open(20)
    f.ctx.pred_begin([h], [1], f.sess.stream)
    for fn, args in [(f.ctx.kv_reorder, ([h, other], [1, 1], True)), (f.ctx.kv_fork_batch, ([h], False)), (f.ctx.kv_remove_batch, ([h],)), (f.ctx.pool_withdraw, (0, 1)), (f.ctx.pool_return, (0, 1))]:
        with pytest.raises(binding.SymError) as e:
            fn(*args)
        assert e.value.code == binding.SYM_EBUSY
    x, s = make(4, 100, "bf16", 1)                            # choices and state rows go on
    compare(choose(f.ctx, x, s, [4], 8), x, s, [4], 8)
    f.ctx.pred_end()
    before = f.ctx.kv_pages(h), f.ctx.kv_pages(other), f.ctx.free_pages()
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=st):
        for fn, args in [(f.ctx.kv_reorder, ([h, other], [1, 1], True, st.cuda_stream)), (f.ctx.kv_fork_batch, ([h], True, st.cuda_stream)), (f.ctx.pool_withdraw, (0, 1, st.cuda_stream))]:
            with pytest.raises(binding.SymError) as e:
                fn(*args)
            assert e.value.code == binding.SYM_EINVAL
        x.add_(0)
    assert (f.ctx.kv_pages(h), f.ctx.kv_pages(other), f.ctx.free_pages()) == before
    f.sess.close()


# ---- together -------------------------------------------------------------------------------------

def test_recorded_choices_and_states(ctx):
    # two graphs with scratch of their own, replayed in turn on new inputs, with eager work between
    runs, keep = [], []
    for k, (beams, vocab, best) in enumerate([([4, 3], 5001, 8), ([2] * 5, 40000, 3)]):
        x, s = make(sum(beams), vocab, "bf16", 40 + k)
        out = [torch.empty((len(beams), best), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
        scratch = torch.empty(binding.beam_scratch_bytes(beams, vocab, best), dtype=torch.uint8, device="cuda")
        rows = sum(beams)
        state, parents = torch.zeros((3, rows, 100), device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
        plan = binding.make_states([(state, state, 1)])
        ctx.beam_select(beams, best, x, s, *out, scratch, None, stream())
        torch.cuda.synchronize()
        g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=st):
            ctx.beam_select(beams, best, x, s, *out, scratch, None, st.cuda_stream)
            ctx.beam_states(beams, parents, plan, st.cuda_stream)
        runs.append((g, beams, vocab, best, x, s, out, state, parents))
        keep.append(scratch)                                  # a graph writes there again
    for turn in range(4):
        wants = []
        for k, (g, beams, vocab, best, x, s, out, state, parents) in enumerate(runs):
            nx, ns = make(sum(beams), vocab, "bf16", 100 * turn + k)
            p = np.concatenate([np.random.default_rng(turn).integers(0, b, b) for b in beams])
            x.copy_(nx), s.copy_(ns), state.normal_(), parents.copy_(torch.from_numpy(p.astype(np.int32)))
            wants.append(moved(state, p, beams, 1))
        for run in runs:
            run[0].replay()
        torch.cuda.synchronize()
        for (g, beams, vocab, best, x, s, out, state, parents), want in zip(runs, wants):
            compare([o.cpu().numpy() for o in out], x, s, beams, best)
            assert torch.equal(state, want)
            (x.float() @ torch.ones((vocab, 2), device="cuda")).sum().item()


def test_another_stream(ctx):
    x, s = make(8, 70001, "f32", 3)
    out = [torch.empty((2, 6), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    scratch = torch.empty(binding.beam_scratch_bytes([4, 4], 70001, 6), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx.beam_select([4, 4], 6, x, s, *out, scratch, None, st.cuda_stream)
    st.synchronize()
    compare([o.cpu().numpy() for o in out], x, s, [4, 4], 6)


@pytest.mark.parametrize("layers", [1, 2])
def test_a_search(layers):
    """Requests of 4, 1 and 3 beams: fork, pred, choose, move states and files, pages withdrawn on the way.  A beam's file has to hold the rows of
    its own tokens, its outputs those of dense attention over them, and its score the sum of the steps' log-probabilities."""
    print(f"[case] search layers={layers}", flush=True)
    Hkv, D, vocab, steps = 2, 64, 300, 9
    beams = [4, 1, 3]
    rows, first = sum(beams), np.repeat(np.concatenate([[0], np.cumsum(beams)[:-1]]), beams)
    f = Files(Hkv, layers, "f32", pages=300, Hq=4)
    g = torch.Generator().manual_seed(7)
    ek, ev = (torch.randn((layers, vocab, Hkv, D), generator=g).cuda() for _ in range(2))
    eq = torch.randn((layers, vocab, 4, D), generator=g).cuda()
    head = (torch.randn((4 * D, vocab), generator=g) * 0.7).cuda()
    prompts = [torch.randint(0, vocab, (n,), generator=g).tolist() for n in (21, 16, 40)]
    tops = []
    for p in prompts:
        h = f.ctx.kv_open(None)
        at = torch.tensor(p, device="cuda")
        f.ctx.kv_append(h, len(p), ek[:, at].contiguous(), ev[:, at].contiguous(), f.sess.stream)
        tops.append(h)
    kv = f.ctx.kv_fork_batch(np.repeat(tops, beams), True, f.sess.stream)
    f.ctx.kv_remove_batch(tops)
    history = torch.zeros((rows, steps + 1), dtype=torch.int32, device="cuda")
    scores = torch.full((rows,), -math.inf, device="cuda")
    scores[sorted(set(first.tolist()))] = 0.0                # at first a request's beams are all the same
    last = torch.tensor([p[-1] for p, b in zip(prompts, beams) for _ in range(b)], device="cuda")
    told = [list(p) for p, b in zip(prompts, beams) for _ in range(b)]
    logp, best = [0.0] * rows, max(beams)
    plan = binding.make_states([(history, history, 0)])
    out = [torch.empty((len(beams), best), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    scratch = torch.empty(binding.beam_scratch_bytes(beams, vocab, best), dtype=torch.uint8, device="cuda")
    attn = torch.empty((layers, rows, 4, D), device="cuda")
    for step in range(steps):
        q, k, v = (e[:, last].contiguous() for e in (eq, ek, ev))
        cows = f.ctx.get_stats()["cow_copies"]
        if layers == 1:
            f.ctx.pred_batch(kv, [1] * rows, q[0], k[0], v[0], attn[0], f.sess.stream)
        else:
            f.ctx.pred_begin(kv, [1] * rows, f.sess.stream)
            for layer in range(layers):
                f.ctx.pred_layer(layer, q[layer], k[layer], v[layer], attn[layer], f.sess.stream)
        assert f.ctx.get_stats()["cow_copies"] == cows       # what a pred would copy is copied already
        for i in range(rows):
            told[i].append(int(last[i]))
        logits = attn.sum(0).flatten(1) @ head
        f.ctx.beam_select(beams, best, logits, scores, *out, scratch, None, f.sess.stream)
        got = [o.cpu().numpy() for o in out]
        compare(got, logits, scores, beams, best)
        source, took = [], []
        for i, b in enumerate(beams):
            source += got[1][i, :b].tolist()
            took += got[2][i, :b].tolist()
        lp = torch.log_softmax(logits.double(), -1).cpu().numpy()
        told, logp = [list(told[o + s]) for o, s in zip(first, source)], [logp[o + s] + lp[o + s, t] for o, s, t in zip(first, source, took)]
        parents = torch.tensor(source, dtype=torch.int32, device="cuda")
        f.ctx.beam_states(beams, parents, plan, f.sess.stream)
        history[:, step] = torch.tensor(took, dtype=torch.int32, device="cuda")
        f.ctx.kv_reorder(kv, np.array(source) + first, True, f.sess.stream)
        scores = torch.cat([out[0][i, :b] for i, b in enumerate(beams)])
        last = torch.tensor(took, device="cuda")
        if step == 4:
            f.ctx.pool_withdraw(0, 40, f.sess.stream)
            f.sess.pool.view(layers, 300, -1)[:, :40] = 0xFF
    torch.cuda.synchronize()
    assert np.allclose(scores.cpu().numpy(), logp, rtol=0, atol=steps * 40 * U * max(1, max(map(abs, logp))))
    for i, h in enumerate(kv):
        at = torch.tensor(told[i], device="cuda")
        f.rows[int(h)] = (ek[:, at], ev[:, at])
        n = len(prompts[np.searchsorted(np.cumsum(beams), i, side="right")])
        assert history[i, :steps].tolist() == told[i][n + 1:] + [int(last[i])]
    f.check([int(h) for h in kv])
    f.ctx.kv_remove_batch(kv)
    assert f.ctx.free_pages() == 260
    f.sess.close()


@pytest.mark.parametrize("pareto_index", [0.5, 2.0])
def test_rag_answers_with_beams(pareto_index):
    """The RAG driver with three beams to an answer, replayed operation by operation on the state model: every batch's outputs, the
    page tables at the end; its scores fall from beam to beam."""
    from oracle.driver import OracleSession
    from paper_2510_25412_amd import rag
    shape = synth.Shape(32, 8, 128, 16, synth.BF16)
    cfg = rag.RagConfig(n_docs=6, doc_tokens=75, answer_tokens=4, retain=2, pareto_index=pareto_index, rate_per_s=20000.0, n_requests=16, prefill_chunk=64,
                        max_batch=6, max_wait_us=200.0, seed=17, beams=3, vocab=1001)
    sess = driver.HipSession(shape, 600, max_lips=18, max_tokens=6 * 64 + 64, max_entries=18 * 10 + 64, poison=True)
    print(f"[case] rag with beams, pareto={pareto_index}", flush=True)
    d = rag.RagDriver(sess, cfg, trace=True)
    res = d.run()
    assert res["requests"] == 16 and res["cached_topics"] <= 2
    osess = OracleSession(shape, 600)
    osess.model = oracle.BeamFiles(600, 16)
    outputs = iter(d.outputs)
    for op in d.trace:
        h = osess.h
        if op[0] == "pred":
            T = sum(op[2])
            ref = osess.pred(dict(files=op[1], n_tokens=op[2], q=d.q_host[:T], k_new=d.k_host[:T], v_new=d.v_host[:T]), dtype=np.float64)
            got = next(outputs)
            assert (np.abs(got - ref) <= 2e-3 * np.maximum(1.0, np.abs(ref))).all()      # the bar of every bf16 pred
        elif op[0] == "fork_batch":
            new, copies = osess.model.kv_fork_batch([h[f] for f in op[2]], True)
            h.update(zip(op[1], new))
            for c in copies:
                osess.pool.copy_slots(*c)
        elif op[0] == "reorder":
            for c in osess.model.kv_reorder([h[f] for f in op[1]], op[2], True):
                osess.pool.copy_slots(*c)
        elif op[0] == "remove_batch":
            osess.model.kv_remove_batch([h.pop(f) for f in op[1]])
        else:
            osess.setup([op])
    assert set(d.h) == set(osess.h) and sess.ctx.free_pages() == osess.model.free_pages()
    for fid in d.h:
        assert sess.ctx.kv_pages(d.h[fid]) == osess.model.kv_pages(osess.h[fid])
    osess.model.audit()
    # every request ends with the best of its beams first, and a token for every step
    scores, tokens = d.scores.cpu().numpy(), d.tokens.cpu().numpy()
    assert np.isfinite(scores).all() and (np.diff(scores, axis=1) <= 0).all()
    assert (tokens >= 0).all() and (tokens < 1001).all()
    d.close()
    assert sess.ctx.free_pages() == 600
    sess.close()
