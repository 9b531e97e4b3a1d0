"""Host half of rotary positions, page bounds and sparse preds (CPU only): refusals that change nothing, and how many leading pages
of a file have bounds, against a model that knows what every page held when its bounds were computed."""
import random

import numpy as np
import pytest

from paper_2510_25412_amd import binding

EINVAL, EBADF, ENOSPC, EBUSY = binding.SYM_EINVAL, binding.SYM_EBADF, binding.SYM_ENOSPC, binding.SYM_EBUSY
BUF = 1 << 20           # an address that a host-only context never follows


def host_ctx(n_pages=64, dtype="bf16", n_layers=1):
    D = 128 if dtype == "bf16" else 64
    cfg = binding.make_config(32, 8, D, 16, dtype, n_pages, device=-1, n_layers=n_layers)
    ctx = binding.Context(cfg)
    ctx.lib.sym_bounds_attach(ctx.h, BUF, binding.bounds_bytes(cfg))
    return ctx


def refused(code, fn, *args, **kw):
    with pytest.raises(binding.SymError) as e:
        fn(*args, **kw)
    assert e.value.code == code, e.value


def state(ctx, files):
    return [(ctx.kv_len(f), ctx.kv_pages(f), ctx.kv_bounded(f)) for f in files], ctx.free_pages()


def test_size_of_the_bounds():
    for dtype, D in (("bf16", 128), ("f32", 64)):
        assert binding.bounds_bytes(binding.make_config(32, 8, D, 16, dtype, 100, n_layers=3)) == 3 * 100 * 8 * 2 * 256
    assert binding.bounds_bytes(binding.make_config(32, 8, 128, 16, "f32", 100)) == 0


def test_attach_is_checked_and_forgets_what_was_there():
    ctx = host_ctx(8)
    f = ctx.kv_open(None)
    ctx.plan_append([f], [40])
    ctx.kv_bounds([f])
    assert ctx.kv_bounded(f) == 2
    size = binding.bounds_bytes(ctx.cfg)
    assert ctx.lib.sym_bounds_attach(ctx.h, BUF + 16, size) == EINVAL
    assert ctx.lib.sym_bounds_attach(ctx.h, BUF, size - 1) == ENOSPC
    assert ctx.kv_bounded(f) == 2
    assert ctx.lib.sym_bounds_attach(ctx.h, BUF, size) == 0 and ctx.kv_bounded(f) == 0
    ctx.bounds_attach(None)
    refused(EINVAL, ctx.kv_bounds, [f])
    refused(EINVAL, ctx.pred_begin_sparse, [f], [1], binding.make_sparse(4))
    refused(EBADF, ctx.kv_bounded, 99)


@pytest.mark.parametrize("kw", [dict(layout=2), dict(layout=-1), dict(dims=3), dict(dims=130), dict(dims=-2), dict(base=0.0), dict(base=-1.0), dict(base=float("nan")),
                                dict(base=float("inf")), dict(factor=-1.0), dict(factor=float("nan")), dict(magnitude=float("inf")), dict(original_len=-1),
                                dict(original_len=8, low_turns=4.0, high_turns=4.0), dict(original_len=8, low_turns=float("nan")), dict(factor=1e-300)])
def test_ropes_that_make_no_sense(kw):
    ctx = host_ctx()
    f = ctx.kv_open(None)
    before = state(ctx, [f])
    rope = binding.make_rope(**kw)
    refused(EINVAL, ctx.kv_append_rope, [f], [3], rope, BUF, BUF)
    refused(EINVAL, ctx.pred_begin_sparse, [f], [3], binding.make_sparse(4, rope=rope))
    assert ctx.lib.sym_rope_rows(ctx.h, rope, 4, BUF, 2 * BUF, 2 * BUF, None, None, None) == EINVAL
    assert b"host-only" not in ctx.lib.sym_strerror(ctx.h)
    assert state(ctx, [f]) == before


def test_rope_rows_arguments():
    ctx = host_ctx()
    rope, n = binding.make_rope(), 16
    call = lambda pos, q, qo, k, ko, r=rope, n=n: (ctx.lib.sym_rope_rows(ctx.h, r, n, pos, q, qo, k, ko, None), ctx.lib.sym_strerror(ctx.h).decode())  # noqa: E731
    q, k, far = 1 << 24, 1 << 26, 1 << 28
    nq, nk = n * 32 * 256, n * 8 * 256
    for bad in [(None, q, q, None, None), (BUF, q, None, None, None), (BUF, None, q, None, None), (BUF, q, q, k, None), (BUF, q + 8, q + 8, None, None),
                (BUF + 2, q, q, None, None), (BUF, q, q + 16, None, None), (BUF, q, q + nq - 16, None, None), (BUF, q, far, q + nq, far + 16),
                (BUF, q, far, k, q + nq - 16), (BUF, q, k + nk - 16, k, k), (BUF, q, far, k, far + nq - 16), (q + 64, q, q, None, None), (k, q, q, k, k)]:
        code, what = call(*bad)
        assert code == EINVAL and "host-only" not in what, (bad, what)
    for good in [(BUF, q, q, k, k), (BUF, q, far, None, None), (BUF, None, None, k, far), (BUF, q, far, k, far + nq)]:
        code, what = call(*good)
        assert code == EINVAL and "host-only" in what, (good, what)
    assert call(BUF, q, q, None, None, None)[0] == EINVAL and call(BUF, q, q, None, None, rope, -1)[0] == EINVAL
    torch = pytest.importorskip("torch")
    with pytest.raises(TypeError):
        ctx.rope_rows(rope, torch.zeros(2, dtype=torch.int64), None, None, None, None)
    with pytest.raises(ValueError):
        ctx.rope_rows(rope, torch.zeros(2, dtype=torch.int32), torch.zeros((3, 32, 128), dtype=torch.bfloat16), torch.zeros((3, 32, 128), dtype=torch.bfloat16), None, None)


def test_append_and_sparse_pred_arguments():
    ctx = host_ctx(8)
    f, g = ctx.kv_open(None), ctx.kv_open(None)
    ctx.plan_append([f, g], [20, 30])
    before = state(ctx, [f, g])
    rope, sp = binding.make_rope(), binding.make_sparse
    for files, n, code in [([f, 77], [1, 1], EBADF), ([f], [0], EINVAL), ([f, g], [1, -4], EINVAL), ([f], [1 << 30], ENOSPC)]:
        refused(code, ctx.kv_append_rope, files, n, rope, BUF, BUF)
        refused(code, ctx.pred_begin_sparse, files, n, sp(4))
        refused(code, ctx.pred_sparse, files, n, sp(4), BUF, BUF, BUF, BUF)
    for bad in (sp(0), sp(4, -1, 1), sp(4, 1, 0), sp(4, 2, 3), sp(2**31 - 1, 2**31 - 1, 2), sp(4, positions=BUF), sp(4, rope=rope, positions=BUF + 1)):
        refused(EINVAL, ctx.pred_begin_sparse, [f], [1], bad)
        assert b"host-only" not in ctx.lib.sym_strerror(ctx.h)
    refused(EINVAL, ctx.kv_append_rope, [f], [1], rope, BUF + 8, BUF)
    refused(EINVAL, ctx.kv_append_rope, [f], [1], None, BUF, BUF, BUF)                # positions without a rope
    refused(EINVAL, ctx.pred_sparse, [f], [1], sp(4), BUF + 4, BUF, BUF, BUF)
    refused(EINVAL, ctx.pred_layer_sparse, 0, BUF, BUF, BUF, BUF)                      # no batch is open
    with pytest.raises(ValueError):
        ctx.kv_append_rope([f, g], [1], rope, BUF, BUF)
    with pytest.raises(ValueError):
        ctx.pred_begin_sparse([f], [1, 1], sp(4))
    for call in (lambda: ctx.kv_append_rope([f], [1], rope, BUF, BUF), lambda: ctx.pred_begin_sparse([f], [1], sp(4))):
        refused(EINVAL, call)
        assert b"host-only" in ctx.lib.sym_strerror(ctx.h)
    ctx.kv_append_rope([], [], None, BUF, BUF)                                         # nothing to do
    assert state(ctx, [f, g]) == before
    many = host_ctx(8, n_layers=2)
    h = many.kv_open(None)
    refused(EINVAL, many.pred_sparse, [h], [1], sp(4), BUF, BUF, BUF, BUF)


def test_files_on_the_host_are_refused():
    ctx = host_ctx(16)
    f = ctx.kv_open(None)
    ctx.plan_append([f], [33])
    ctx.kv_offload([f])
    refused(EBUSY, ctx.kv_bounds, [f])


@pytest.mark.parametrize("seed", range(6))
def test_leading_pages_with_bounds_against_a_model(seed):
    """The model keeps, per pool page, the 16 token ids that its bounds were computed from; a file's bounded pages must be
    full pages whose bounds are of exactly the tokens the file has there."""
    r, ctx = random.Random(seed), host_ctx(200)
    files, fresh, of_page = {}, iter(range(1 << 40)), {}       # handle -> token ids
    for step in range(500):
        op = r.choice(["open", "append", "append", "append", "fork", "truncate", "bounds", "bounds", "extract", "merge", "away", "back", "remove"])
        live = [h for h in files if not ctx.kv_waiting(h)]
        h = r.choice(live) if live else None
        try:
            if op == "open" or h is None:
                files[ctx.kv_open(None)] = []
            elif op == "append":
                n = r.choice([1, 1, 5, 16, 40])
                ctx.plan_append([h], [n])
                files[h] = files[h] + [next(fresh) for _ in range(n)]
            elif op == "fork":
                files[ctx.kv_fork(h)] = list(files[h])
            elif op == "truncate":
                n = r.randint(0, len(files[h]))
                ctx.kv_truncate([h], [n])
                files[h] = files[h][:n]
            elif op == "bounds":
                some = r.sample(live, min(len(live), 2))
                ctx.kv_bounds(some)
                for x in some:
                    pages = ctx.kv_pages(x)
                    for p in range(len(files[x]) // 16):
                        of_page[pages[p]] = files[x][16 * p:16 * p + 16]
                    assert ctx.kv_bounded(x) == len(files[x]) // 16
            elif op == "extract":
                idx = sorted(r.sample(range(len(files[h])), len(files[h]) // 2)) if r.random() < 0.5 else list(range(len(files[h])))
                files[ctx.kv_extract(h, idx)] = [files[h][i] for i in idx]
            elif op == "merge":
                some = r.sample(live, min(len(live), 2))
                files[ctx.kv_merge(some)] = sum((files[x] for x in some), [])
            elif op == "away":
                ctx.kv_offload([h])
            elif op == "back":
                gone = [x for x in files if ctx.kv_waiting(x)]
                if gone:
                    ctx.kv_restore([r.choice(gone)])
            elif op == "remove" or len(files) > 12:
                ctx.kv_remove(h)
                del files[h]
        except binding.SymError as e:
            assert e.code == ENOSPC
            for x in list(files)[::2]:
                ctx.kv_remove(x)
                del files[x]
        for x, ids in files.items():
            pages, n = ctx.kv_pages(x), ctx.kv_bounded(x)
            assert 0 <= n <= len(ids) // 16
            for p in range(n):
                assert pages[p] >= 0 and of_page[pages[p]] == ids[16 * p:16 * p + 16], (step, op, x, p)
