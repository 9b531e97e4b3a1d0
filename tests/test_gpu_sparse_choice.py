"""The pages that sparse preds choose on the GPU where scores are extreme, equal or very many, against a choice by torch on the files' own bounds (sums
in 64 bits, rounded to 32; whole numbers, so equal)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2510_25412_amd import binding, driver, synth

pytestmark = pytest.mark.gpu

P = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DIM = {"bf16": 128, "f32": 64}
INF, NAN = float("inf"), float("nan")


def ranked(score):
    """Indices of fp32 scores [.., pages] from the highest, ties to the lower index, NaN above all."""
    bits = (score + np.float32(0)).view(np.uint32).astype(np.int64)
    order = np.where(bits >> 31 == 1, 0xffffffff - bits, bits + (1 << 31))
    return np.argsort(np.where(np.isnan(score), -1, (1 << 32) - order), axis=-1, kind="stable")


class Files:
    """Files of `pages` pages each (the last one without its last token) over a pool of random rows, whose bounds are attached."""

    def __init__(self, dtype, hq, hkv, pages, seed):
        self.dtype, self.hq, self.hkv, self.D, self.pages = dtype, hq, hkv, DIM[dtype], pages
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        total = sum(pages) + 2
        self.sess = driver.HipSession(synth.Shape(hq, hkv, self.D, P, dtype), total, None, max_lips=len(pages), max_tokens=4096, max_entries=total + 64)
        ctx = self.ctx = self.sess.ctx
        self.bounds = torch.zeros((total, hkv, 2, self.D), dtype=TYPES[dtype], device="cuda")
        ctx.bounds_attach(self.bounds)
        self.kv = [ctx.kv_open(None) for _ in pages]
        ctx.plan_append(self.kv, [P * n - 1 for n in pages])
        self.pool = self.sess.pool.view(TYPES[dtype]).view(-1, hkv, 2, 2, P, self.D // 2)
        self.pool.copy_(torch.randn(self.pool.shape, generator=self.g, device="cuda", dtype=TYPES[dtype]))

    def ids(self, i):
        return torch.tensor(self.ctx.kv_pages(self.kv[i]), device="cuda")

    def plant(self, i, some, values):
        """One key element of `some` pages of file i in every head: the values in turn."""
        r = np.random.default_rng(i + some)
        at = self.ids(i)[torch.from_numpy(r.permutation(np.arange(1, self.pages[i] - 2))[:some]).cuda()]
        for head in range(self.hkv):
            half, slot, d = int(r.integers(2)), int(r.integers(P)), int(r.integers(self.D // 2))
            self.pool[at, head, 0, half, slot, d] = torch.tensor([values[j % len(values)] for j in range(len(at))], device="cuda").to(TYPES[self.dtype])

    def check(self, budget, first, last):
        """One token to each file, its choice compared; returns the outputs."""
        n = len(self.kv)
        q = torch.randn((n, self.hq, self.D), generator=self.g, device="cuda", dtype=TYPES[self.dtype])
        k = torch.randn((n, self.hkv, self.D), generator=self.g, device="cuda", dtype=TYPES[self.dtype])
        out = torch.full((n, self.hq, self.D), NAN, device="cuda")
        pick = torch.full((n, self.hkv, budget), -7, dtype=torch.int32, device="cuda")
        self.ctx.pred_sparse(self.kv, [1] * n, binding.make_sparse(budget, first, last), q, k, k, out, pick, self.sess.stream)
        torch.cuda.synchronize()
        got = pick.cpu()
        grouped = q.double().view(n, self.hkv, self.hq // self.hkv, self.D)
        up, down = grouped.clamp(min=0).sum(2), grouped.clamp(max=0).sum(2)
        for i, pages in enumerate(self.pages):
            if pages <= budget:
                want = torch.arange(budget).where(torch.arange(budget) < pages, torch.tensor(-1))
                assert (got[i] == want).all(), i
                continue
            b = self.bounds[self.ids(i)[first:pages - last]].double()
            score = ((b[:, :, 1] * up[i]).sum(-1) + (b[:, :, 0] * down[i]).sum(-1)).float().cpu().numpy().T          # [Hkv, pages]
            rank = ranked(score)
            middle = np.sort(rank[:, :budget - first - last], axis=1) + first
            want = np.concatenate([np.tile(np.arange(first), (self.hkv, 1)), middle, np.tile(np.arange(pages - last, pages), (self.hkv, 1))], 1)
            assert np.array_equal(got[i].numpy(), want), (i, pages)
        self.ctx.kv_truncate(self.kv, [P * x - 1 for x in self.pages])
        return out

    def close(self):
        self.sess.close()


# the number of scores decides how many a thread holds and where they are computed: one wavefront's worth, a thread's, scored by the workgroups
# that attend, held four to thirty-two to a thread, read again in every round
@pytest.mark.parametrize("pages", [40, 240, 600, 2300, 5000, 9000, 17000])
@pytest.mark.parametrize("dtype,values", [("bf16", [INF]), ("bf16", [NAN]), ("bf16", [INF, NAN, -INF]), ("f32", [3.4e38, -3.4e38]), ("f32", [INF, 2e38, NAN])])
def test_more_extreme_scores_than_are_wanted(pages, dtype, values):
    print(f"[case] extreme scores {dtype} {values} {pages}", flush=True)
    files = Files(dtype, 2, 1, [pages], pages)
    some = pages // 3
    files.plant(0, some, values)
    for budget in (4, 9, min(some // 2 + 3, 1500), min(some + 5, 3000)):
        files.check(budget, 1, 2)
    files.close()


@pytest.mark.parametrize("values", [[INF], [NAN, INF]])
def test_many_rows_with_extreme_scores(values):
    # more rows and heads than compute units: the attention scores for itself
    files = Files("bf16", 16, 8, [30 + 17 * i for i in range(40)], 3)
    for i in range(0, 40, 2):
        files.plant(i, files.pages[i] // 2, values)
    for budget in (6, 40):
        files.check(budget, 1, 1)
    files.close()


@pytest.mark.parametrize("dtype,hq", [("bf16", 16), ("f32", 8)])
def test_many_rows_of_very_different_lengths(dtype, hq):
    # four wavefronts to a workgroup, one file each of the numbers of scores that a thread of them holds: 1, 4, 8, 16, 32, and read again
    pages = [200, 900, 1500, 3000, 4500, 8500] + list(range(1, 61, 2))
    files = Files(dtype, hq, 8, pages, 11)
    for budget, first, last in ((9, 1, 2), (333, 0, 1), (2500, 3, 4)):
        files.check(budget, first, last)
    for i in range(6):
        files.plant(i, 120, [INF, NAN])
    files.ctx.bounds_attach(files.bounds)                        # (the bounds of the planted pages are computed again)
    files.check(60, 1, 1)
    files.close()
