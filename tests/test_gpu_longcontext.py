"""Rotary positions, rotated appends, bounds of pages and sparse preds on the GPU, against oracle/longcontext.py in 64 bits.

Tolerances.  A turned element is computed in 64 bits and rounded by way of 32 to the storage type: half a step of the value, eps / 2,
and what the angle is off: positions below 2^31 times at most 1/2 pi turns in 64 bits, 2^31 * 2^-53 turns and as much for the factor, 3e-6 of
the pair's size (far positions; 1e-9 below 2^20).  Bounds and the choice of pages are exact.  An output of attention: scores are sums of D
products in fp32, off by at most D * 2^-24 * sum |q k| * scale = e; a weight is then off by e + 2^-22 (exponential) + 2^-17
(what the weights are cut to with 8 heads per kv head), relative, and the output by twice that of the largest |v|."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import longcontext as lc
from paper_2510_25412_amd import binding, driver, synth

pytestmark = pytest.mark.gpu

P = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DIM = {"bf16": 128, "f32": 64}


def session(dtype, hq, hkv, n_pages, layers=1, order=None, poison=True, bounds=True, **kw):
    sess = driver.HipSession(synth.Shape(hq, hkv, DIM[dtype], P, dtype), n_pages, order, max_lips=64, max_tokens=4096, max_entries=1 << 15, poison=poison, n_layers=layers, **kw)
    if bounds:
        sess.bounds = torch.full((layers, n_pages, hkv, 2, DIM[dtype]), float("nan"), dtype=TYPES[dtype], device="cuda")
        sess.ctx.bounds_attach(sess.bounds)
    return sess


def rows(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(TYPES[dtype]).cuda()


def f64(t):
    return t.double().cpu().numpy()


def read(sess, h, layer=0):
    n = sess.ctx.kv_len(h)
    s = sess.shape
    k, v = (torch.empty((n, s.n_kv_heads, s.head_dim), dtype=TYPES[s.dtype], device="cuda") for _ in range(2))
    if n:
        sess.ctx.kv_read(h, 0, n, k, v, sess.stream, layer=layer)
    torch.cuda.synchronize()
    return k, v


def stored(x, dtype):
    """float64 -> the storage type's values, by way of 32 bits."""
    x = np.asarray(x).astype(np.float32)
    return synth.to_f32(synth.bf16_round(x)) if dtype == "bf16" else x


def check_turned(got, x, pos, freq, layout, mag, dtype):
    want = lc.turn(f64(x), pos, freq, layout, mag)
    size = mag * np.abs(f64(x)).max()
    far = max(1.0, float(np.abs(np.asarray(pos, np.float64)).max()))
    tol = torch.finfo(TYPES[dtype]).eps / 2 * 1.001 * np.abs(want) + 2 * size * (far * 2.0**-51 + 1e-12) + (1e-38 if dtype == "f32" else 1e-37)
    assert (np.abs(f64(got) - want) <= tol).all()
    half = 2 * len(freq)
    assert torch.equal(got[..., half:].cpu(), x[..., half:].cpu())          # what does not turn is moved as it is


def check_out(out, ref, q, K, V, scale, dtype):
    D = K.shape[-1]
    e = D * 2.0**-24 * (np.abs(q).max(0).max(0) @ np.abs(K).max(0).max(0)) * scale
    tol = 2 * (e + 2.0**-22 + 2.0**-17) * np.abs(V).max()
    err = np.abs(f64(out) - ref)
    assert np.isfinite(f64(out)).all() and err.max() <= tol, (err.max(), tol)
    assert np.linalg.norm(err) <= 1e-5 * np.linalg.norm(ref)                # and far less over many


def check_bounds(sess, files):
    for layer in range(sess.n_layers):
        for h in files:
            k, _ = read(sess, h, layer)
            pages = sess.ctx.kv_pages(h)
            n = sess.ctx.kv_bounded(h)
            want = lc.page_bounds(f64(k))[:n]
            assert np.array_equal(f64(sess.bounds[layer][pages[:n]]), want)


# ---- rope ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hq,hkv,n,layout,dims,kw", [
    ("bf16", 32, 8, 1, "halves", 128, {}), ("bf16", 8, 8, 3, "interleaved", 128, dict(factor=4.0)), ("f32", 8, 8, 64, "halves", 64, dict(magnitude=1.3)),
    ("f32", 8, 1, 17, "interleaved", 64, {}), ("bf16", 4, 1, 33, "halves", 64, dict(original_len=4096, factor=8.0)), ("bf16", 5, 5, 9, "halves", 2, {}),
    ("bf16", 3, 3, 70, "halves", 20, {}), ("bf16", 2, 1, 5, "interleaved", 20, {}), ("f32", 2, 2, 31, "halves", 26, {}), ("f32", 16, 2, 12, "interleaved", 6, {}),
    ("bf16", 32, 8, 2047, "halves", 128, {}), ("bf16", 32, 8, 2049, "interleaved", 96, {}), ("f32", 6, 3, 2050, "halves", 48, {}), ("bf16", 64, 8, 2051, "halves", 126, {}),
    ("f32", 7, 7, 2048, "halves", 62, {})])
@pytest.mark.parametrize("far", [40, 1 << 20, (1 << 31) - 1])
def test_turned_rows(dtype, hq, hkv, n, layout, dims, kw, far):
    print(f"[case] rope {dtype} {hq}/{hkv} n={n} {layout} {dims} {kw} far={far}", flush=True)
    sess = session(dtype, hq, hkv, 4, bounds=False)
    g, r = torch.Generator().manual_seed(n + dims), np.random.default_rng(n)
    pos = r.integers(-far if n % 2 else 0, far, n, endpoint=True)
    q, k = rows(g, n, hq, DIM[dtype], dtype=dtype), rows(g, n, hkv, DIM[dtype], dtype=dtype)
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    rope = binding.make_rope(layout, dims, 500000.0, **kw)
    freq = lc.frequencies(dims, 500000.0, **{x: y for x, y in kw.items() if x != "magnitude"})
    mag = kw.get("magnitude", 1.0)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    sess.ctx.rope_rows(rope, p, q, qo, k, ko, sess.stream)
    check_turned(qo, q, pos, freq, layout, mag, dtype)
    check_turned(ko, k, pos, freq, layout, mag, dtype)
    q2, k2 = q.clone(), k.clone()                                           # in place, and one of the two alone
    sess.ctx.rope_rows(rope, p, q2, q2, k2, k2, sess.stream)
    only = torch.empty_like(k)
    sess.ctx.rope_rows(rope, p, None, None, k, only, sess.stream)
    assert torch.equal(q2, qo) and torch.equal(k2, ko) and torch.equal(only, ko)
    sess.ctx.rope_rows(rope, p, q, q2, None, None, sess.stream)
    assert torch.equal(q2, qo)
    sess.close()


def test_no_rows_and_rows_that_are_not_finite():
    sess = session("bf16", 4, 2, 4, bounds=False)
    rope, p = binding.make_rope(dims=64), torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    sess.ctx.rope_rows(rope, p[:0], torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda"), None, None, sess.stream)
    sess.ctx.rope_rows(rope, p, None, None, None, None, sess.stream)
    k = rows(torch.Generator().manual_seed(1), 2, 2, 128, dtype="bf16")
    k[0, 1, 3] = float("inf")
    k[1, 0, 100] = float("nan")                                             # in the part that does not turn
    ko = torch.empty_like(k)
    sess.ctx.rope_rows(rope, p, None, None, k, ko, sess.stream)
    bad = ~torch.isfinite(ko)
    want = torch.zeros_like(bad)
    want[0, 1, 3] = want[0, 1, 35] = want[1, 0, 100] = True
    assert torch.equal(bad, want)
    sess.close()


def test_rope_is_recorded_and_replayed():
    sess = session("bf16", 8, 8, 4, bounds=False)
    g = torch.Generator().manual_seed(3)
    q, k = rows(g, 40, 8, 128, dtype="bf16"), rows(g, 40, 8, 128, dtype="bf16")
    p = torch.arange(40, dtype=torch.int32, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rope = binding.make_rope()
    sess.ctx.profile_enable(0xff)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sess.ctx.rope_rows(rope, p, q, qo, k, ko, sess.stream)
    for i in range(3):
        q.copy_(rows(g, 40, 8, 128, dtype="bf16"))
        p.add_(100)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(q)
        sess.ctx.rope_rows(rope, p, q, want, None, None, sess.stream)
        torch.cuda.synchronize()
        assert torch.equal(want, qo)
    sess.close()


def test_calls_that_cannot_be_recorded_say_so_and_change_nothing():
    sess = session("bf16", 8, 8, 16)
    f = sess.ctx.kv_open(None)
    sess.ctx.plan_append([f], [20])
    x = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((1, 8, 128), device="cuda")
    torch.cuda.synchronize()
    graph, codes = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        x.add_(1)
        for call in (lambda: sess.ctx.kv_append_rope([f], [1], None, x, x, None, sess.stream), lambda: sess.ctx.kv_bounds([f], sess.stream),
                     lambda: sess.ctx.pred_sparse([f], [1], binding.make_sparse(4), x, x, x, out, None, sess.stream),
                     lambda: sess.ctx.pred_begin_sparse([f], [1], binding.make_sparse(4), sess.stream)):
            try:
                call()
                codes.append(0)
            except binding.SymError as e:
                codes.append(e.code)
    assert codes == [binding.SYM_EINVAL] * 4 and sess.ctx.kv_len(f) == 20 and sess.ctx.kv_bounded(f) == 0
    sess.close()


# ---- append and bounds -----------------------------------------------------------------------------------

# runs travel with the arguments up to 128 of them; pages completed from any slot, by one token or many, in one call or several
@pytest.mark.parametrize("dtype,hkv,before,new,layers", [
    ("bf16", 8, [0], [1], 1), ("bf16", 8, [15], [1], 1), ("f32", 8, [0, 15, 16, 31], [16, 17, 1, 33], 1), ("bf16", 1, [7], [300], 1), ("bf16", 3, [5, 0], [11, 64], 2),
    ("f32", 2, [1] * 64, [31] * 64, 1), ("bf16", 2, [9] * 127 + [0], [1] * 128, 1), ("bf16", 2, [9] * 128 + [0], [1] * 129, 1), ("bf16", 5, [0], [2048], 1),
    ("bf16", 5, [0], [2049], 1), ("f32", 12, [3], [2060], 3), ("bf16", 16, [100], [5], 1)])
@pytest.mark.parametrize("layout,dims", [("halves", 0), ("interleaved", 50), ("halves", 36), (None, 0)])
def test_rotated_append(dtype, hkv, before, new, layers, layout, dims):
    print(f"[case] append {dtype} {hkv} {before[:4]} {new[:4]} x{len(new)} layers={layers} {layout} {dims}", flush=True)
    D = DIM[dtype]
    n_pages = sum(-(-(a + b) // P) for a, b in zip(before, new)) + 4
    sess = session(dtype, hkv, hkv, n_pages, layers)
    g = torch.Generator().manual_seed(sum(new))
    files = [sess.ctx.kv_open(None) for _ in new]
    old = []
    for h, n in zip(files, before):
        old.append((rows(g, layers, n, hkv, D, dtype=dtype), rows(g, layers, n, hkv, D, dtype=dtype)))
        if n:
            sess.ctx.kv_append(h, n, *old[-1], sess.stream)
    sess.ctx.kv_bounds(files, sess.stream)
    T = sum(new)
    k, v = rows(g, layers, T, hkv, D, dtype=dtype), rows(g, layers, T, hkv, D, dtype=dtype)
    rope = binding.make_rope(layout, dims) if layout else None
    index = torch.from_numpy(np.concatenate([np.arange(a, a + b) for a, b in zip(before, new)]).astype(np.int32)).cuda()
    pos = index * 3 + 1 if rope is not None and len(new) % 2 else None
    sess.ctx.kv_append_rope(files, new, rope, k, v, pos, sess.stream)
    turned = k.clone()
    if rope is not None:
        for layer in range(layers):
            sess.ctx.rope_rows(rope, index if pos is None else pos, None, None, k[layer], turned[layer], sess.stream)
    for layer in range(layers):
        t = 0
        for h, n, m, (ko, vo) in zip(files, before, new, old):
            got_k, got_v = read(sess, h, layer)
            assert torch.equal(got_k, torch.cat([ko[layer], turned[layer, t:t + m]])) and torch.equal(got_v, torch.cat([vo[layer], v[layer, t:t + m]]))
            t += m
    assert [sess.ctx.kv_bounded(h) for h in files] == [(a + b) // P for a, b in zip(before, new)]
    check_bounds(sess, files[:9])
    sess.close()


def test_append_to_shared_pages_copies_before_it_completes_them():
    sess = session("bf16", 8, 8, 64)
    g = torch.Generator().manual_seed(5)
    root = sess.ctx.kv_open(None)
    k, v = rows(g, 1, 31, 8, 128, dtype="bf16"), rows(g, 1, 31, 8, 128, dtype="bf16")
    sess.ctx.kv_append_rope([root], [31], None, k, v, None, sess.stream)
    kids = [sess.ctx.kv_fork(root) for _ in range(5)]
    assert [sess.ctx.kv_bounded(h) for h in kids] == [1] * 5
    n = [1, 2, 1, 17, 1]
    k2, v2 = rows(g, 1, sum(n), 8, 128, dtype="bf16"), rows(g, 1, sum(n), 8, 128, dtype="bf16")
    sess.ctx.kv_append_rope(kids, n, None, k2, v2, None, sess.stream)
    t = 0
    for h, m in zip(kids, n):
        got_k, got_v = read(sess, h)
        assert torch.equal(got_k, torch.cat([k[0], k2[0, t:t + m]])) and torch.equal(got_v, torch.cat([v[0], v2[0, t:t + m]]))
        t += m
    assert torch.equal(read(sess, root)[0], k[0])
    assert [sess.ctx.kv_bounded(h) for h in kids] == [2, 2, 2, 3, 2]
    check_bounds(sess, kids + [root])
    # a sharer that sees fewer tokens of the page than the copies do appends in place last
    a = sess.ctx.kv_fork(kids[3])
    sess.ctx.kv_truncate([kids[3]], [40])
    m = [3, 9]
    k3, v3 = rows(g, 1, 12, 8, 128, dtype="bf16"), rows(g, 1, 12, 8, 128, dtype="bf16")
    whole = read(sess, a)[0]
    sess.ctx.kv_append_rope([a, kids[3]], m, None, k3, v3, None, sess.stream)
    assert torch.equal(read(sess, a)[0], torch.cat([whole, k3[0, :3]])) and torch.equal(read(sess, kids[3])[0], torch.cat([whole[:40], k3[0, 3:]]))
    assert sess.ctx.kv_bounded(kids[3]) == 3
    check_bounds(sess, kids + [root, a])
    sess.close()


@pytest.mark.parametrize("dtype,hkv,lens,layers", [("bf16", 8, [0, 1, 15, 16, 17, 300], 1), ("f32", 3, [4100], 2), ("bf16", 1, [16 * 256], 1), ("f32", 8, [16 * 257, 40], 1), ("bf16", 5, [100] * 60, 3)])
def test_bounds_of_pages(dtype, hkv, lens, layers):
    print(f"[case] bounds {dtype} {hkv} {lens[:6]} layers={layers}", flush=True)
    n_pages = sum(-(-n // P) for n in lens) + 3
    order = np.random.default_rng(1).permutation(n_pages).astype(np.int32)
    sess = session(dtype, hkv, hkv, n_pages, layers, order)
    g = torch.Generator().manual_seed(sum(lens))
    files = [sess.ctx.kv_open(None) for _ in lens]
    for h, n in zip(files, lens):
        if n:
            sess.ctx.kv_append(h, n, rows(g, layers, n, hkv, DIM[dtype], dtype=dtype), rows(g, layers, n, hkv, DIM[dtype], dtype=dtype), sess.stream)
            torch.cuda.synchronize()
    assert [sess.ctx.kv_bounded(h) for h in files] == [0] * len(files)
    sess.ctx.kv_bounds(files + files[:1], sess.stream)
    torch.cuda.synchronize()
    assert [sess.ctx.kv_bounded(h) for h in files] == [n // P for n in lens]
    check_bounds(sess, files)
    used = torch.zeros(n_pages, dtype=torch.bool)
    for h, n in zip(files, lens):
        used[sess.ctx.kv_pages(h)[:n // P]] = True
    assert torch.isnan(sess.bounds[:, ~used.cuda()]).all()                  # nothing else is written
    sess.close()


def test_bounds_of_keys_that_are_not_finite():
    sess = session("bf16", 2, 2, 8)
    f = sess.ctx.kv_open(None)
    k = rows(torch.Generator().manual_seed(2), 1, 48, 2, 128, dtype="bf16")
    k[0, 3, 0, 5], k[0, 9, 0, 5] = float("inf"), float("-inf")
    k[0, 20, 1, 127] = float("nan")
    sess.ctx.kv_append(f, 48, k, k, sess.stream)
    sess.ctx.kv_bounds([f], sess.stream)
    torch.cuda.synchronize()
    got = sess.bounds[0][sess.ctx.kv_pages(f)].float().cpu()
    pages = k[0].float().cpu().view(3, 16, 2, 128)
    assert torch.equal(torch.nan_to_num(got, nan=777.0), torch.nan_to_num(torch.stack([pages.amin(1), pages.amax(1)], 2), nan=777.0))
    assert torch.isnan(got[1, 1, :, 127]).all()
    sess.close()


# ---- sparse preds ----------------------------------------------------------------------------------------

def make_files(sess, lens, g, spread=0.7):
    s, L = sess.shape, sess.n_layers
    files = []
    for n in lens:
        files.append(sess.ctx.kv_open(None))
        if n:
            shared = torch.randn((L, -(-n // P), 1, s.n_kv_heads, s.head_dim), generator=g).expand(-1, -1, P, -1, -1).reshape(L, -1, s.n_kv_heads, s.head_dim)[:, :n]
            k = (torch.randn((L, n, s.n_kv_heads, s.head_dim), generator=g) + spread * shared).to(TYPES[s.dtype]).cuda()
            sess.ctx.kv_append(files[-1], n, k, rows(g, L, n, s.n_kv_heads, s.head_dim, dtype=s.dtype), sess.stream)
            torch.cuda.synchronize()
    return files


def run_sparse(sess, files, new, sp, rope=None, freq=None, layout="halves", layers=None, dense=(), g=None, pos=None, picked=True):
    """One batch, checked: appended rows, bounds, pages read, outputs."""
    s, ctx, L = sess.shape, sess.ctx, sess.n_layers
    g = g or torch.Generator().manual_seed(sum(new))
    T, D = sum(new), s.head_dim
    before = [ctx.kv_len(h) for h in files]
    q, k, v = rows(g, L, T, s.n_q_heads, D, dtype=s.dtype), rows(g, L, T, s.n_kv_heads, D, dtype=s.dtype), rows(g, L, T, s.n_kv_heads, D, dtype=s.dtype)
    out = torch.full((L, T, s.n_q_heads, D), float("nan"), device="cuda")
    pick = torch.full((L, T, s.n_kv_heads, sp.budget), -7, dtype=torch.int32, device="cuda") if picked else None
    q0, k0 = q.clone(), k.clone()
    if L == 1:
        ctx.pred_sparse(files, new, sp, q[0], k[0], v[0], out[0], pick[0] if picked else None, sess.stream)
    else:
        ctx.pred_begin_sparse(files, new, sp, sess.stream)
        for layer in (layers or range(L)):
            if layer in dense:
                ctx.pred_layer(layer, q[layer], k[layer], v[layer], out[layer], sess.stream)
            else:
                ctx.pred_layer_sparse(layer, q[layer], k[layer], v[layer], out[layer], pick[layer] if picked else None, sess.stream)
    torch.cuda.synchronize()
    assert torch.equal(q, q0) and torch.equal(k, k0)
    index = np.concatenate([np.arange(n, n + m) for n, m in zip(before, new)])
    at = index if pos is None else pos.cpu().numpy()
    for layer in range(L):
        t = 0
        for h, n, m in zip(files, before, new):
            assert ctx.kv_len(h) == n + m
            K, V = read(sess, h, layer)
            qs, ks = f64(q[layer, t:t + m]), f64(k[layer, t:t + m])
            if rope is not None and layer not in dense:
                qs, ks = (stored(lc.turn(x, at[t:t + m], freq, layout, rope.magnitude), s.dtype).astype(np.float64) for x in (qs, ks))
            assert np.array_equal(f64(K[n:]), ks) and torch.equal(V[n:], v[layer, t:t + m])
            budget = 1 << 30 if layer in dense else sp.budget
            ref, pages = lc.sparse_attention(qs, f64(K), f64(V), n, budget, sp.first, sp.last)
            if picked and layer not in dense:
                want = np.full((m, s.n_kv_heads, sp.budget), -1)
                for i in range(m):
                    for x in range(s.n_kv_heads):
                        want[i, x, :len(pages[i][x])] = pages[i][x]
                assert np.array_equal(pick[layer, t:t + m].cpu().numpy(), want)
            if layer not in dense:
                check_out(out[layer, t:t + m], ref, qs, f64(K), f64(V), 1 / np.sqrt(D), s.dtype)
            else:
                assert (np.abs(f64(out[layer, t:t + m]) - ref) <= 2e-3 * np.maximum(1, np.abs(ref))).all()
            t += m
    if not L > 1 or layers is None:
        assert [ctx.kv_bounded(h) for h in files] == [ctx.kv_len(h) // P for h in files]
        check_bounds(sess, files)
    return out


@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 8, 8), ("bf16", 8, 4), ("bf16", 32, 8), ("bf16", 16, 2), ("bf16", 8, 1), ("f32", 3, 3), ("f32", 4, 2), ("f32", 4, 1), ("f32", 16, 2)])
@pytest.mark.parametrize("budget,first,last", [(1, 0, 1), (3, 1, 2), (8, 1, 2), (20, 0, 1), (64, 2, 4)])
def test_sparse_decode(dtype, hq, hkv, budget, first, last):
    print(f"[case] sparse {dtype} {hq}/{hkv} budget {budget} {first} {last}", flush=True)
    lens = [0, 1, 15, 16, 47, 16 * budget - 1, 16 * budget, 700, 1111]
    sess = session(dtype, hq, hkv, sum(-(-n // P) + 3 for n in lens))
    g = torch.Generator().manual_seed(budget + hq)
    files = make_files(sess, lens, g)
    rope = binding.make_rope("interleaved" if budget == 8 else "halves", DIM[dtype] // 2 if budget == 3 else 0, factor=2.0)
    freq = lc.frequencies(rope.dims or DIM[dtype], factor=2.0)
    for step in range(3):                      # the first call finds no bounds, the others what it left
        use = rope if step else None
        run_sparse(sess, files, [1] * len(files), binding.make_sparse(budget, first, last, rope=use), use, freq, "interleaved" if budget == 8 else "halves", g=g)
    sess.close()


@pytest.mark.parametrize("dtype,hq,hkv,lens,new,budget", [("bf16", 32, 8, [700, 0, 33, 250], [5, 40, 3, 1], 6), ("f32", 8, 8, [300, 15], [17, 9], 5), ("bf16", 8, 1, [130], [100], 4),
                                                          ("bf16", 64, 8, [90, 1000], [4, 2], 7), ("f32", 16, 2, [63], [66], 3)])
def test_sparse_drafts_and_chunks(dtype, hq, hkv, lens, new, budget):
    # every token chooses for itself; pages that an earlier token of the call completes are among the choice of a later one
    print(f"[case] sparse chunk {dtype} {hq}/{hkv} {lens} {new}", flush=True)
    sess = session(dtype, hq, hkv, sum(-(-(n + 3 * m) // P) + 2 for n, m in zip(lens, new)))
    g = torch.Generator().manual_seed(sum(lens))
    files = make_files(sess, lens, g)
    rope = binding.make_rope()
    for _ in range(2):
        run_sparse(sess, files, new, binding.make_sparse(budget, 1, 1, rope=rope), rope, lc.frequencies(DIM[dtype]), g=g)
    sess.close()


# most scores a token of each variant of the choice, the line of every one; one wavefront's 32 pages of scores
@pytest.mark.parametrize("pages", [5, 34, 35, 36, 67, 258, 259, 260, 515, 1026, 1027, 1100])
def test_number_of_scores(pages):
    sess = session("bf16", 2, 1, pages + 4)
    g = torch.Generator().manual_seed(pages)
    files = make_files(sess, [16 * pages - 3], g)
    run_sparse(sess, files, [1], binding.make_sparse(min(9, pages - 1), 1, 1), g=g)
    sess.close()


@pytest.mark.parametrize("pages", [514, 515, 2050, 2051, 4098, 4099, 8194, 8195, 16386, 16387, 17000])
def test_number_of_scores_of_long_files(pages):
    # fp32 choice as the library documents it, computed by torch on the file's own bounds
    sess = session("bf16", 1, 1, pages + 4, poison=False)
    g = torch.Generator(device="cuda").manual_seed(pages)
    f = sess.ctx.kv_open(None)
    sess.ctx.plan_append([f], [16 * pages - 1])
    pool = sess.pool.view(torch.bfloat16).view(-1, 2, 2, 16, 64)
    pool.copy_(torch.randn(pool.shape, generator=g, device="cuda", dtype=torch.bfloat16))
    q = torch.randn((1, 1, 128), generator=g, device="cuda", dtype=torch.bfloat16)
    k, out = torch.zeros_like(q), torch.empty((1, 1, 128), device="cuda")
    pick = torch.empty((1, 1, min(700, pages - 100)), dtype=torch.int32, device="cuda")
    sess.ctx.pred_sparse([f], [1], binding.make_sparse(pick.shape[2], 1, 1), q, k, k, out, pick, sess.stream)
    torch.cuda.synchronize()
    b = sess.bounds[0, torch.tensor(sess.ctx.kv_pages(f), device="cuda"), 0].double()
    score = ((b[:, 1] * q[0, 0].double().clamp(min=0)).sum(-1) + (b[:, 0] * q[0, 0].double().clamp(max=0)).sum(-1)).float()[1:-1]
    want = torch.sort(torch.sort(score, dim=0, descending=True, stable=True).indices[:pick.shape[2] - 2]).values + 1
    assert pick[0, 0].tolist() == [0] + want.tolist() + [pages - 1]
    sess.close()


def test_equal_scores_take_the_lowest_indices_and_nan_comes_first():
    sess = session("f32", 2, 2, 64)
    f = sess.ctx.kv_open(None)
    n = 16 * 40
    k = torch.zeros((1, n, 2, 64))
    k[:, :, 1] = torch.arange(n)[None, :, None].div(16, rounding_mode="floor") % 3 - 1.0
    k[0, 16 * 30 + 5, 0, 7] = float("nan")
    k[0, 16 * 35 + 5, 0, 0] = float("inf")                      # 0 * inf in the score of a query with a zero there
    v = torch.ones((1, n, 2, 64))
    sess.ctx.kv_append(f, n, k.cuda(), v.cuda(), sess.stream)
    q = torch.ones((1, 2, 64))
    q[0, 0] = 0.0
    pick = torch.empty((1, 2, 6), dtype=torch.int32, device="cuda")
    out = torch.empty((1, 2, 64), device="cuda")
    new = torch.zeros((1, 2, 64), device="cuda")
    sess.ctx.pred_sparse([f], [1], binding.make_sparse(6, 1, 1), q.cuda(), new, new, out, pick, sess.stream)
    torch.cuda.synchronize()
    assert pick[0, 0].tolist() == [0, 1, 2, 30, 35, 40]
    assert pick[0, 1].tolist() == [0, 2, 5, 8, 11, 40]
    assert torch.isnan(out[0, 0]).all() and torch.isfinite(out[0, 1]).all()
    sess.close()


def test_values_that_are_not_finite_reach_the_outputs_that_see_them():
    for dtype, hq, hkv in (("bf16", 4, 1), ("bf16", 8, 1), ("f32", 4, 1)):
        sess = session(dtype, hq, hkv, 16)
        f = sess.ctx.kv_open(None)
        D = DIM[dtype]
        g = torch.Generator().manual_seed(4)
        k, v = 0.1 * torch.randn((1, 100, 1, D), generator=g), torch.randn((1, 100, 1, D), generator=g)
        v[0, 3, 0, 1], v[0, 20, 0, 2], v[0, 99, 0, 3] = float("inf"), float("nan"), float("-inf")
        sess.ctx.kv_append(f, 100, k.to(TYPES[dtype]).cuda(), v.to(TYPES[dtype]).cuda(), sess.stream)
        q, new = torch.randn((1, hq, D), generator=g).to(TYPES[dtype]).cuda(), torch.zeros((1, 1, D), dtype=TYPES[dtype], device="cuda")
        out = torch.empty((1, hq, D), device="cuda")
        sess.ctx.pred_sparse([f], [1], binding.make_sparse(8, 1, 1), q, new, new, out, None, sess.stream)
        o = out[0].cpu()
        assert (o[:, 1] == float("inf")).all() and torch.isnan(o[:, 2]).all() and (o[:, 3] == float("-inf")).all()
        o[:, 1:4] = 0
        assert torch.isfinite(o).all()
        sess.close()


def test_steps_over_layers_sparse_and_dense():
    # a model whose first layer attends to everything: prompt by dense preds, then steps with both kinds of layers; forks, drafts rolled back
    sess = session("bf16", 8, 2, 400, layers=3)
    g = torch.Generator().manual_seed(8)
    files = make_files(sess, [200, 37, 450], g)
    rope = binding.make_rope()
    freq = lc.frequencies(128)
    sp = binding.make_sparse(6, 1, 2, rope=rope, dense_layers=True)
    for step, new in enumerate([[1, 1, 1], [4, 1, 2], [1, 30, 1], [1, 1, 1]]):
        run_sparse(sess, files, new, sp, rope, freq, layers=[2, 0, 1] if step == 1 else None, dense=(0,), g=g)
        if step == 1:
            sess.ctx.kv_truncate(files, [n - 3 for n in map(sess.ctx.kv_len, files)])
            files.append(sess.ctx.kv_fork(files[2]))
            files.pop(1)
    only = binding.make_sparse(6, 1, 2, rope=rope)
    run_sparse(sess, files, [1, 1, 2], only, rope, freq, g=g)
    sess.ctx.pred_begin_sparse(files, [1, 1, 1], only, sess.stream)
    x, o = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8, 128), device="cuda")
    for code, call in [(binding.SYM_EINVAL, lambda: sess.ctx.pred_layer(0, x, x, x, o, sess.stream)), (binding.SYM_EINVAL, lambda: sess.ctx.pred_layer_sparse(3, x, x, x, o, None, sess.stream)),
                       (binding.SYM_EBUSY, lambda: sess.ctx.kv_append_rope([files[0]], [1], None, x, x, None, sess.stream)), (binding.SYM_EBUSY, lambda: sess.ctx.kv_bounds(files, sess.stream)),
                       (binding.SYM_EBUSY, lambda: sess.ctx.bounds_attach(None)), (binding.SYM_EBUSY, lambda: sess.ctx.pred_begin_sparse([files[0]], [1], only, sess.stream))]:
        with pytest.raises(binding.SymError) as e:
            call()
        assert e.value.code == code
    sess.ctx.pred_layer_sparse(1, x, x[:, :2].contiguous(), x[:, :2].contiguous(), o, None, sess.stream)
    with pytest.raises(binding.SymError) as e:
        sess.ctx.pred_layer_sparse(1, x, x[:, :2].contiguous(), x[:, :2].contiguous(), o, None, sess.stream)
    assert e.value.code == binding.SYM_EBUSY
    had = [sess.ctx.kv_bounded(h) for h in files]
    sess.ctx.pred_end()
    assert [sess.ctx.kv_bounded(h) for h in files] == had          # the abandoned layers' rows are not there
    with pytest.raises(binding.SymError) as e:
        sess.ctx.pred_layer_sparse(0, x, x, x, o, None, sess.stream)
    assert e.value.code == binding.SYM_EINVAL
    sess.close()


def test_files_that_came_by_other_calls():
    # extracted, merged, offloaded and restored pages have no bounds, or their old place's: the pred computes what is missing
    sess = session("bf16", 8, 2, 400)
    g = torch.Generator().manual_seed(9)
    a, b = make_files(sess, [500, 333], g)
    run_sparse(sess, [a, b], [1, 1], binding.make_sparse(5, 1, 1), g=g)
    c = sess.ctx.kv_extract(a, np.arange(0, 501, 2), sess.stream)
    d = sess.ctx.kv_merge([b, a], sess.stream)
    sess.ctx.kv_offload([a], sess.stream)
    sess.ctx.kv_offload([b], sess.stream)
    e = make_files(sess, [200], g)[0]                            # takes the pages that were freed
    run_sparse(sess, [c, d, e], [1, 1, 1], binding.make_sparse(5, 1, 1), g=g)
    sess.ctx.kv_restore([b, a], sess.stream)
    run_sparse(sess, [a, b, c, d, e], [1, 20, 1, 3, 1], binding.make_sparse(5, 1, 1), g=g)
    sess.close()


def test_long_scattered_files_one_part_of_the_list_to_each_of_many_workgroups():
    # few rows: the list is cut into parts that the merge kernel joins; an odd budget, parts that do not divide evenly
    for dtype, hq, hkv, budget in (("bf16", 16, 2, 97), ("f32", 4, 1, 131), ("bf16", 4, 1, 255)):
        sess = session(dtype, hq, hkv, 700, order=np.random.default_rng(2).permutation(700).astype(np.int32))
        g = torch.Generator().manual_seed(budget)
        files = make_files(sess, [9001], g)
        for _ in range(2):
            run_sparse(sess, files, [1], binding.make_sparse(budget, 3, 5), g=g)
        sess.close()


def test_positions_of_the_caller():
    sess = session("bf16", 8, 2, 64)
    g = torch.Generator().manual_seed(11)
    files = make_files(sess, [100, 60], g)
    rope = binding.make_rope(base=500000.0, factor=8.0, original_len=8192, magnitude=1.1)
    freq = lc.frequencies(128, 500000.0, 8.0, 8192)
    pos = torch.tensor([100000, 7, 8], dtype=torch.int32, device="cuda")
    run_sparse(sess, files, [1, 2], binding.make_sparse(4, 1, 1, rope=rope, positions=pos), rope, freq, g=g, pos=pos)
    sess.close()


def test_a_pool_that_is_full_changes_nothing():
    sess = session("bf16", 2, 2, 4)
    g = torch.Generator().manual_seed(12)
    f = make_files(sess, [50], g)[0]
    x, o = torch.zeros((20, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((20, 2, 128), device="cuda")
    before = (sess.ctx.kv_len(f), sess.ctx.kv_pages(f), sess.ctx.free_pages(), sess.ctx.kv_bounded(f))
    for call in (lambda: sess.ctx.kv_append_rope([f], [20], binding.make_rope(), x, x, None, sess.stream),
                 lambda: sess.ctx.pred_sparse([f], [20], binding.make_sparse(2), x, x, x, o, None, sess.stream)):
        with pytest.raises(binding.SymError) as e:
            call()
        assert e.value.code == binding.SYM_ENOSPC
    sess.ctx.test_fail_staging(1)
    with pytest.raises(binding.SymError):
        sess.ctx.pred_sparse([f], [1], binding.make_sparse(2), x, x, x, o, None, sess.stream)
    assert (sess.ctx.kv_len(f), sess.ctx.kv_pages(f), sess.ctx.free_pages(), sess.ctx.kv_bounded(f)) == before
    run_sparse(sess, [f], [14], binding.make_sparse(2), g=g)
    sess.close()


@pytest.mark.parametrize("dtype,hq,hkv,new", [("bf16", 8, 2, [6, 21, 1]), ("f32", 4, 1, [5, 2, 18]), ("bf16", 16, 2, [1, 1, 1]), ("bf16", 3, 3, [4, 4, 4])])
def test_several_tokens_of_files_with_many_scores(dtype, hq, hkv, new):
    # more pages than a workgroup scores for itself: up to four tokens share the pass over the bounds, also across a page's end
    sess = session(dtype, hq, hkv, 1800)
    g = torch.Generator().manual_seed(sum(new) + hq)
    files = make_files(sess, [9010, 60, 8700], g)
    rope = binding.make_rope()
    for budget in (40, 7):
        run_sparse(sess, files, new, binding.make_sparse(budget, 1, 2, rope=rope), rope, lc.frequencies(DIM[dtype]), g=g)
    sess.close()


@pytest.mark.parametrize("budget", [2100, 2260])
def test_lists_longer_than_a_workgroup_holds(budget):
    # 2200 pages: chosen from, and read whole; every token's list is cut into two parts at least
    sess = session("f32", 2, 1, 2300)
    g = torch.Generator().manual_seed(budget)
    files = make_files(sess, [35200 - 2], g)
    run_sparse(sess, files, [3], binding.make_sparse(budget, 2, 3), g=g)
    sess.close()


def small_context(hq, hkv, n_pages, workspace_bytes):
    cfg = binding.make_config(hq, hkv, 128, P, "bf16", n_pages, device=0, decode_waves=1)
    pool = torch.zeros(n_pages * binding.page_bytes(cfg), dtype=torch.uint8, device="cuda")
    ws = torch.empty(workspace_bytes, dtype=torch.uint8, device="cuda")
    cfg.pool, cfg.workspace, cfg.workspace_bytes = pool.data_ptr(), ws.data_ptr(), workspace_bytes
    ctx = binding.Context(cfg)
    ctx.bounds_attach(torch.empty(binding.bounds_bytes(cfg), dtype=torch.uint8, device="cuda"))
    return ctx, (pool, ws)


def test_a_small_workspace_takes_the_rows_a_few_at_a_time():
    # 70 tokens of one file of 700 pages: 2 kv heads x 700 scores, 5.6 KB a token; a page in the middle of a slab is completed
    g = torch.Generator().manual_seed(21)
    k, v = rows(g, 1, 11200, 2, 128, dtype="bf16"), rows(g, 1, 11200, 2, 128, dtype="bf16")
    q, kn, vn = rows(g, 70, 4, 128, dtype="bf16"), rows(g, 70, 2, 128, dtype="bf16"), rows(g, 70, 2, 128, dtype="bf16")
    st = torch.cuda.current_stream().cuda_stream
    got = []
    for size in (64 << 20, 160 << 10, 120 << 10):
        ctx, keep = small_context(4, 2, 720, size)
        f = ctx.kv_open(None)
        # the append reads its runs from the staging buffer, not from the workspace
        ctx.kv_append_rope([f], [11200], None, k, v, None, st)
        out, pick = torch.empty((70, 4, 128), device="cuda"), torch.empty((70, 2, 30), dtype=torch.int32, device="cuda")
        launches = ctx.get_stats()["kernel_launches"]
        ctx.pred_sparse([f], [70], binding.make_sparse(30, 1, 1, rope=binding.make_rope()), q, kn, vn, out, pick, st)
        torch.cuda.synchronize()
        got.append((out, pick, ctx.get_stats()["kernel_launches"] - launches))
        del keep
        ctx.close()
    assert got[0][2] == 3 and got[1][2] > 3 and got[2][2] > got[1][2]
    for out, pick, _ in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(pick, got[0][1])
    ctx, keep = small_context(4, 2, 720, 78 << 10)      # 70 turned query rows, the lists (5 KB) and no room for one token's scores
    f = ctx.kv_open(None)
    ctx.plan_append([f], [11200])
    before = (ctx.kv_len(f), ctx.kv_pages(f), ctx.free_pages())
    with pytest.raises(binding.SymError) as e:
        ctx.pred_sparse([f], [70], binding.make_sparse(30, 1, 1, rope=binding.make_rope()), q, kn, vn, got[0][0], None, st)
    assert e.value.code == binding.SYM_ENOSPC and (ctx.kv_len(f), ctx.kv_pages(f), ctx.free_pages()) == before
    ctx.close()


@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 8, 2), ("f32", 8, 1)])
def test_reading_every_page_is_a_dense_pred_of_turned_rows(dtype, hq, hkv):
    # the calls as a model makes them: prompt by a rotated append, one step on turned rows by the dense pred, the same step sparse
    sess, other = session(dtype, hq, hkv, 64), session(dtype, hq, hkv, 64)
    g = torch.Generator().manual_seed(31)
    D = DIM[dtype]
    rope, n, new = binding.make_rope("interleaved", factor=4.0, original_len=1024), [300, 31], [1, 3]
    k, v = rows(g, 1, sum(n), hkv, D, dtype=dtype), rows(g, 1, sum(n), hkv, D, dtype=dtype)
    q, kn, vn = rows(g, 4, hq, D, dtype=dtype), rows(g, 4, hkv, D, dtype=dtype), rows(g, 4, hkv, D, dtype=dtype)
    outs = []
    for s in (sess, other):
        files = [s.ctx.kv_open(None) for _ in n]
        s.ctx.kv_append_rope(files, n, rope, k, v, None, s.stream)
        out = torch.empty((4, hq, D), device="cuda")
        if s is sess:
            pos = torch.tensor([300, 31, 32, 33], dtype=torch.int32, device="cuda")
            qt, kt = torch.empty_like(q), torch.empty_like(kn)
            s.ctx.rope_rows(rope, pos, q, qt, kn, kt, s.stream)
            s.ctx.pred_batch(files, new, qt, kt, vn, out, s.stream)
        else:
            s.ctx.pred_sparse(files, new, binding.make_sparse(99, 1, 1, rope=rope), q, kn, vn, out, None, s.stream)
        torch.cuda.synchronize()
        outs.append((out, [read(s, h) for h in files]))
    assert all(torch.equal(a, b) for x, y in zip(outs[0][1], outs[1][1]) for a, b in zip(x, y))
    # the dense pred rounds the weights of several tokens to 11 bits: its own bar
    assert ((outs[0][0] - outs[1][0]).abs() <= 2e-3 * outs[1][0].abs().clamp(min=1)).all()
    for s in (sess, other):
        s.close()


def test_calls_on_a_stream_of_their_own():
    sess = session("bf16", 8, 2, 80)
    g = torch.Generator().manual_seed(41)
    files = make_files(sess, [600, 90], g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rope = binding.make_rope()
    with torch.cuda.stream(side):
        for _ in range(3):
            run_sparse(sess, files, [1, 2], binding.make_sparse(6, 1, 1, rope=rope), rope, lc.frequencies(128), g=g)
    torch.cuda.current_stream().wait_stream(side)
    sess.close()


def test_pages_beyond_32_bits_of_bytes():
    # the files' pages are the last of a pool of 72 GB, their bounds at the end of a buffer of 4.5 GB
    n_pages = 1_100_000
    order = np.arange(n_pages, dtype=np.int32)[::-1].copy()
    sess = session("bf16", 16, 8, n_pages, order=order, poison=False, bounds=False)
    sess.bounds = torch.empty((1, n_pages, 8, 2, 128), dtype=torch.bfloat16, device="cuda")
    sess.ctx.bounds_attach(sess.bounds)
    g = torch.Generator().manual_seed(51)
    files = make_files(sess, [500, 60], g)
    assert min(sess.ctx.kv_pages(files[0])) > 1_000_000
    rope = binding.make_rope()
    run_sparse(sess, files, [1, 17], binding.make_sparse(6, 1, 1, rope=rope), rope, lc.frequencies(128), g=g)
    k = rows(g, 1, 40, 8, 128, dtype="bf16")
    sess.ctx.kv_append_rope(files, [1, 39], None, k, k, None, sess.stream)
    sess.ctx.kv_bounds(files, sess.stream)
    torch.cuda.synchronize()
    check_bounds(sess, files)
    sess.close()


def test_forks_of_one_prompt():
    # eight branches of a shared prefix, each with a tail of its own, one token each: pages and bounds of the prefix are shared
    sess = session("bf16", 8, 2, 200)
    g = torch.Generator().manual_seed(61)
    root = make_files(sess, [405], g)[0]
    sess.ctx.kv_bounds([root], sess.stream)
    kids = [sess.ctx.kv_fork(root) for _ in range(8)]
    rope = binding.make_rope()
    for new in ([1] * 8, [12] + [1] * 7, [1] * 8):
        run_sparse(sess, kids, new, binding.make_sparse(7, 1, 2, rope=rope), rope, lc.frequencies(128), g=g)
    sess.close()


@pytest.mark.parametrize("dtype,hq,hkv,layout,dims,lens", [("bf16", 8, 1, "halves", 0, [8991, 20, 8300]), ("bf16", 8, 4, "interleaved", 36, [8300]), ("f32", 4, 2, "halves", 16, [8815, 8400]),
                                                           ("f32", 3, 3, "interleaved", 64, [8303]), ("bf16", 2, 2, "halves", 24, [8400]), ("bf16", 16, 8, "halves", 0, [8400] * 4)])
@pytest.mark.parametrize("given", [False, True])
def test_steps_over_layers_of_files_with_many_scores(dtype, hq, hkv, layout, dims, lens, given):
    # later steps find all bounds there: their appends and scores may go together (files that complete a page, one with nothing to score;
    # 24 elements are halves that a lane does not hold, and four files of eight heads have too many scores for that)
    print(f"[case] layers, many scores {dtype} {hq}/{hkv} {layout} {dims} {lens} {given}", flush=True)
    sess = session(dtype, hq, hkv, sum(-(-n // P) + 2 for n in lens), layers=2)
    g = torch.Generator().manual_seed(len(lens))
    files = make_files(sess, lens, g)
    rope = binding.make_rope(layout, dims, base=50000.0, magnitude=1.25)
    for _ in range(3):
        pos = torch.tensor([n + 70001 for n in map(sess.ctx.kv_len, files)], dtype=torch.int32, device="cuda") if given else None
        run_sparse(sess, files, [1] * len(files), binding.make_sparse(9, 1, 2, rope=rope, positions=pos), rope, lc.frequencies(dims or DIM[dtype], 50000.0), layout, g=g, pos=pos)
    sess.close()


@pytest.mark.parametrize("dtype,hq,hkv,lens,new", [("bf16", 8, 8, [16 * 130, 16 * 700, 16 * 1500 + 7], [11, 12, 13]), ("bf16", 8, 4, [16 * 2045], [66]), ("bf16", 4, 2, [16 * 2049], [130]),
                                                   ("f32", 4, 4, [16 * 300, 16 * 1030], [40, 30]), ("f32", 16, 2, [16 * 2300, 50], [100, 40])])
def test_many_rows_with_many_scores(dtype, hq, hkv, lens, new):
    # more rows and heads than compute units: the attention scores up to 2048 pages itself, beyond them not
    print(f"[case] many rows, many scores {dtype} {hq}/{hkv} {lens} {new}", flush=True)
    sess = session(dtype, hq, hkv, sum(-(-(n + m) // P) + 2 for n, m in zip(lens, new)))
    files = make_files(sess, lens, torch.Generator().manual_seed(len(lens)))
    run_sparse(sess, files, new, binding.make_sparse(7, 1, 2))
    sess.close()


@pytest.mark.parametrize("pages", [400, 1900])
def test_one_long_file_among_many_short_ones(pages):
    # many rows, of which few have pages to score
    sess = session("bf16", 16, 8, pages + 200)
    g = torch.Generator().manual_seed(pages)
    files = make_files(sess, [16 * pages - 3] + list(range(1, 80, 2)), g)
    for _ in range(2):
        run_sparse(sess, files, [1] * len(files), binding.make_sparse(20, 1, 2), g=g)
    sess.close()


@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 1, 1), ("bf16", 8, 1), ("bf16", 2, 2), ("f32", 1, 1), ("f32", 4, 1)])
@pytest.mark.parametrize("budget", [70, 300])
def test_short_files_beside_long_ones(dtype, hq, hkv, budget):
    # the list of a long file goes in parts, of which a short file's row has pages for a few or for one
    print(f"[case] short beside long {dtype} {hq}/{hkv} {budget}", flush=True)
    lens = [0, 5, 16, 40, 16 * 420 + 1, 16 * 64]
    sess = session(dtype, hq, hkv, sum(-(-n // P) + 2 for n in lens), order=np.arange(sum(-(-n // P) + 2 for n in lens), dtype=np.int32)[::-1].copy())
    g = torch.Generator().manual_seed(budget)
    files = make_files(sess, lens, g)
    for _ in range(2):
        run_sparse(sess, files, [1] * len(files), binding.make_sparse(budget, 1, 2), g=g)
    sess.close()
