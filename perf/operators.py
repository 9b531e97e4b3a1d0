"""Rotary positions, rotated appends, page bounds and sparse preds: the work to be measured, with its plain form.

A case is one pass through one of the library's operators for long contexts, on files that are already there.

Kinds of cases
  rope    the query and key rows of `tokens` new tokens turned to their positions, U{0..far}
  append  U{new_lo..new_hi} tokens appended to each of `lips` files of U{lo..hi} tokens, keys turned on the way to
          their pages, bounds of the pages that they complete written
  bounds  the bounds (elementwise minimum and maximum of the keys) of every full page of `lips` files of U{lo..hi} tokens
  sparse  `lips` files of U{lo..hi} tokens, U{new_lo..new_hi} new tokens each, through `layers` attention layers: the new rows
          turned and appended, every new token and kv head attends to at most `budget` pages: the first `first`, the
          last `last`, and those between of the highest score
Everywhere: `layout` "halves", "interleaved" or "none" (rows arrive turned), `dims` of a head that turn, `base`, `factor` and `orig` of the
scaling for long contexts, `mag`; `scatter`: pages of a file in random places of the pool; `lens`: seed of lengths and positions.

The cache is the documented page layout, [page][kv head][K, V][row half][16 tokens][half a row]; page p of layer l is page
l * pages + p.  A pass leaves the files as long as it found them.
"""
import math
import random

import numpy as np
import torch

own = False
P = 16          # tokens per page


def listed():
    turned = dict(layout="halves", dims=128, base=500000.0, factor=8.0, orig=8192, mag=1.0)
    plain = dict(layout="halves", dims=128, base=10000.0, factor=1.0, orig=0, mag=1.0)
    return [
        # A decode step's rows of a loaded server: launch latency.
        dict(name="rope_64_rows", kind="rope", dtype="bf16", hq=32, hkv=8, tokens=64, far=131072, lens=1, **turned),
        # Prompt chunks of a server's full batch.
        dict(name="rope_16384_rows", kind="rope", dtype="bf16", hq=32, hkv=8, tokens=16384, far=131072, lens=2, **turned),
        # fp32 storage, neighbours paired, three quarters of the head turned, an odd number of rows.
        dict(name="rope_f32_part", kind="rope", dtype="f32", hq=8, hkv=8, tokens=1559, far=4096, lens=3, layout="interleaved", dims=48, base=10000.0, factor=4.0, orig=0, mag=1.1),
        # One token for each of 64 files: every sixteenth completes a page.
        dict(name="append_64x1", kind="append", dtype="bf16", hq=32, hkv=8, lips=64, lo=512, hi=4096, new_lo=1, new_hi=1, scatter=False, lens=4, **turned),
        # A document's rows brought into the cache.
        dict(name="append_doc", kind="append", dtype="bf16", hq=32, hkv=8, lips=1, lo=0, hi=0, new_lo=6000, new_hi=9000, scatter=False, lens=5, **plain),
        # Bounds of one short file, fp32 storage.
        dict(name="bounds_f32_1", kind="bounds", dtype="f32", hq=8, hkv=8, lips=1, lo=300, hi=700, scatter=False, lens=6),
        # Bounds of a server's files that were stored by a prompt's dense attention.
        dict(name="bounds_64", kind="bounds", dtype="bf16", hq=32, hkv=8, lips=64, lo=512, hi=4096, scatter=True, lens=7),
        # The smallest sparse pred: one fp32 file, rows that arrive turned.
        dict(name="sparse_f32_1", kind="sparse", dtype="f32", hq=8, hkv=8, lips=1, lo=1500, hi=2500, new_lo=1, new_hi=1, layers=1, budget=32, first=1, last=2,
             scatter=False, lens=8, layout="none", dims=64, base=10000.0, factor=1.0, orig=0, mag=1.0),
        # The decode batch of a loaded server: 64 files of 512..4096 tokens, 1024 tokens read of each.
        dict(name="sparse_64", kind="sparse", dtype="bf16", hq=32, hkv=8, lips=64, lo=512, hi=4096, new_lo=1, new_hi=1, layers=1, budget=64, first=1, last=2,
             scatter=False, lens=9, **turned),
        # Long contexts on a 70B-shaped layer, pages scattered.
        dict(name="sparse_long_g8", kind="sparse", dtype="bf16", hq=64, hkv=8, lips=8, lo=32768, hi=131072, new_lo=1, new_hi=1, layers=1, budget=256, first=1, last=4,
             scatter=True, lens=10, **turned),
        # One user's long file through the attention layers of a model.
        dict(name="sparse_1x8_layers", kind="sparse", dtype="bf16", hq=32, hkv=8, lips=1, lo=20000, hi=40000, new_lo=1, new_hi=1, layers=8, budget=128, first=1, last=4,
             scatter=False, lens=11, **turned),
        # Drafts and short chunks being verified, ragged.
        dict(name="sparse_chunks", kind="sparse", dtype="bf16", hq=32, hkv=8, lips=8, lo=1000, hi=8000, new_lo=2, new_hi=33, layers=1, budget=48, first=1, last=4,
             scatter=False, lens=12, **turned),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, evenly spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "append", "bounds", "sparse", "sparse", "sparse", "long"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D = 128 if dtype == "bf16" else 64
    hkv = rng.choice([1, 2, 4, 8, 8])
    c = dict(dtype=dtype, hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 8]), lens=rng.randrange(1, 1 << 30))
    turn = dict(layout=rng.choice(["halves", "interleaved"]), dims=rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)]), base=rng.choice([10000.0, 500000.0, 1e6]),
                factor=rng.choice([1.0, 4.0, 8.0]), orig=rng.choice([0, 4096, 8192]), mag=rng.choice([1.0, 1.0, 1.2]))
    if kind == "rope":
        c.update(kind="rope", tokens=_log(rng, 1, 8192), far=_log(rng, 16, 1 << 20), **turn)
    elif kind == "append":
        new, lips = _log(rng, 1, 4096), _log(rng, 1, 64)
        new = max(1, min(new, 8192 // lips))
        c.update(kind="append", lips=lips, lo=0, hi=rng.choice([0, 1000, 4000]), new_lo=max(1, new // 2), new_hi=new, scatter=rng.random() < 0.3, **turn)
    elif kind == "bounds":
        lo = _log(rng, 1, 2048)
        c.update(kind="bounds", lips=_log(rng, 1, 64), lo=lo, hi=2 * lo, scatter=rng.random() < 0.3)
    else:
        if kind == "long":
            lo, lips, new, layers = _log(rng, 16384, 65536), _log(rng, 1, 4), 1, 1
        else:
            lo, lips, new, layers = _log(rng, 16, 8192), _log(rng, 1, 48), rng.choice([1, 1, 1, _log(rng, 2, 24)]), rng.choice([1, 1, 3])
            lips = max(1, min(lips, 80000 // (lo * layers), 96 // (new * layers)))
        rows = lips * new * layers
        budget = max(4, min(_log(rng, 4, 256), 24000 // (rows * c["hq"] // hkv), 4500 // rows))
        first, last = rng.randint(0, 2), rng.randint(1, 2)
        if rng.random() < 0.2:
            turn["layout"] = "none"
        c.update(kind="sparse", lips=lips, lo=lo, hi=2 * lo, new_lo=max(1, new // 2), new_hi=new, layers=layers, budget=budget, first=first, last=last,
                 scatter=kind == "long" or rng.random() < 0.3, **turn)
    return c


# ---- what a case consists of ------------------------------------------------------------------

def _dim(case):
    return 128 if case["dtype"] == "bf16" else 64


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _files(case):
    """Lengths of the files, and new tokens of each."""
    r = random.Random(case["lens"])
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["lips"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) if "new_lo" in case else 0 for _ in lens]
    return lens, new


def _tables(case):
    """Pages of the pool, the order in which pages are given out, and every file's pages with the new tokens in it: all files as
    they are first, then what the new tokens need, file by file."""
    lens, new = _files(case)
    before, after = [-(-n // P) for n in lens], [-(-(n + m) // P) for n, m in zip(lens, new)]
    used, pages = sum(after), sum(after) + 2
    if case.get("scatter"):
        pages += pages // 4
    order = np.random.Generator(np.random.PCG64(case["lens"])).permutation(pages) if case.get("scatter") else np.arange(pages)
    start, extra = np.concatenate([[0], np.cumsum(before)]), sum(before) + np.concatenate([[0], np.cumsum(np.array(after) - np.array(before))])
    tables = [np.concatenate([order[start[i]:start[i + 1]], order[extra[i]:extra[i + 1]]]) for i in range(len(lens))]
    assert sum(map(len, tables)) == used
    return pages, order.astype(np.int32), tables


def _positions(case):
    r = np.random.Generator(np.random.PCG64(case["lens"]))
    return r.integers(0, case["far"], case["tokens"]).astype(np.int32)


def _inputs(case, seed):
    """The cache (keys: a part that a page's tokens share, a few large channels, noise) and the rows of the new tokens."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    D, H, t, layers = _dim(case), case["hkv"], _type(case), case.get("layers", 1)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=t)  # noqa: E731
    got = {}
    if case["kind"] == "rope":
        n = case["tokens"]
        got.update(q=randn(n, case["hq"], D), k=randn(n, H, D))
        return got
    pages = _tables(case)[0] * layers
    pool = randn(pages, H, 2, 2, P, D // 2)
    pool[:, :, 0] += 0.7 * randn(pages, H, 2, 1, D // 2)
    pool[:, :, 0] += 2.0 * (torch.rand((1, H, 2, 1, D // 2), generator=g, device="cuda") < 0.05).to(t)
    got["pool"] = pool
    T = sum(_files(case)[1])
    if T:
        got.update(k=randn(layers, T, H, D), v=randn(layers, T, H, D))
    if case["kind"] == "sparse":
        got["q"] = randn(layers, T, case["hq"], D)
    return got


def _bounds_of(pool, at):
    """[len(at), Hkv, 2, D]: smallest and largest element of the keys of pages `at`."""
    k = pool[:, :, 0][at]                                        # [pages, Hkv, row half, 16, half a row]
    return torch.stack([k.amin(3).flatten(2), k.amax(3).flatten(2)], 2)


def prepare(case, seed):
    x = _inputs(case, seed)
    st = dict(case=case, **x)
    dev = lambda a, t=torch.int64: torch.as_tensor(np.asarray(a), device="cuda", dtype=t)  # noqa: E731
    layers, kind = case.get("layers", 1), case["kind"]
    sparse = kind == "sparse"
    if kind == "rope":
        st.update(pos=dev(_positions(case), torch.int32), q_out=torch.empty_like(x["q"]), k_out=torch.empty_like(x["k"]))
        sess_pages, order, tables, lens, new = 4, None, [], [0], [0]
    else:
        lens, new = _files(case)
        sess_pages, order, tables = _tables(case)
        full = np.concatenate([t[:n // P] for t, n in zip(tables, lens)] + [np.zeros(0, np.int64)]).astype(np.int64)
        at = dev(np.concatenate([full + i * sess_pages for i in range(layers)]))
        st["bounds"] = torch.zeros((layers * sess_pages, case["hkv"], 2, _dim(case)), dtype=_type(case), device="cuda")
        if kind == "bounds":
            st["full"] = at
        else:
            st["bounds"][at] = _bounds_of(x["pool"], at)         # the files' pages have theirs from earlier steps
            T = sum(new)
            pos = np.concatenate([np.arange(n, n + m) for n, m in zip(lens, new)])
            page = np.concatenate([t[np.arange(n, n + m) // P] for t, n, m in zip(tables, lens, new)])
            shift = np.repeat(np.arange(layers) * sess_pages, T)
            done = np.concatenate([t[n // P:(n + m) // P] for t, n, m in zip(tables, lens, new)])
            st.update(at_pos=dev(np.tile(pos, layers)), at_page=dev(np.tile(page, layers) + shift), at_slot=dev(np.tile(pos % P, layers)),
                      done=dev(np.concatenate([done + i * sess_pages for i in range(layers)])))
            if sparse:
                most = max(map(len, tables))
                table = np.zeros((len(tables), most), np.int64)
                for i, t in enumerate(tables):
                    table[i, :len(t)] = t
                file = np.repeat(np.arange(len(tables)), new)
                st.update(table=dev(np.concatenate([table[file] + i * sess_pages for i in range(layers)])), out=torch.empty_like(x["q"], dtype=torch.float32))
    if case.get("layout", "none") != "none":
        st["angle"] = dev(_frequencies(case), torch.float64)
    if own:
        st.update(_session(case, st, sess_pages, order, lens, new))
    torch.cuda.synchronize()
    return st


def _session(case, st, pages, order, lens, new):
    """The library's side: a context over the pool, its files, the settings of the calls."""
    from paper_2510_25412_amd import binding, driver, synth
    kind, layers = case["kind"], case.get("layers", 1)
    shape = synth.Shape(case["hq"], case["hkv"], _dim(case), P, case["dtype"])
    sess = driver.HipSession(shape, pages, order, "cuda:0", max_lips=max(len(lens), 1), max_tokens=max(sum(new), 64),
                             max_entries=sum(-(-(n + m) // P) + 1 for n, m in zip(lens, new)) + 64, n_layers=layers)
    ctx, got = sess.ctx, dict(sess=sess, ctx=sess.ctx)
    if case.get("layout", "none") != "none":
        got["rope"] = binding.make_rope(layout=case["layout"], dims=case["dims"], base=case["base"], factor=case["factor"], original_len=case["orig"],
                                        low_turns=1.0, high_turns=32.0, magnitude=case["mag"])
    if kind == "rope":
        return got
    pool = sess.pool.view(_type(case)).view(st["pool"].shape)
    pool.copy_(st["pool"])
    kv = np.array([ctx.kv_open(None) for _ in lens], np.int32)
    some = [i for i, n in enumerate(lens) if n]
    if some:
        ctx.plan_append(kv[some], [lens[i] for i in some])       # the files' pages; their rows lie in the pool already
    ctx.bounds_attach(st["bounds"])
    if some and kind != "bounds":
        ctx.kv_bounds(kv, sess.stream)
    got.update(pool=pool, kv=kv, n=np.array(new, np.int32), lengths=np.array(lens, np.int64))
    if kind == "sparse":
        got["sparse"] = binding.make_sparse(case["budget"], case["first"], case["last"], rope=got.get("rope"))
    return got


def _frequencies(case):
    """Radians per position of every pair."""
    f = case["base"] ** (-np.arange(0, case["dims"], 2, dtype=np.float64) / case["dims"])
    if case["orig"] == 0:
        return f / case["factor"]
    turns = case["orig"] * f / (2 * math.pi)
    keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    return f * (keep + (1.0 - keep) / case["factor"])


# ---- the plain form ---------------------------------------------------------------------------

def _turn(case, x, pos, freq):
    """Rows x [n, heads, D] turned to positions pos [n]; in 64 bits (angles of far positions; a key that rounds to its neighbour in the
    storage type shows in fp32 outputs), rounded to the storage type."""
    if case["layout"] == "none":
        return x
    angle = pos.double()[:, None, None] * freq
    c, s = case["mag"] * torch.cos(angle), case["mag"] * torch.sin(angle)
    y, R = x.double(), case["dims"]
    if case["layout"] == "halves":
        a, b = y[..., :R // 2], y[..., R // 2:R]
        z = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        z = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([z, y[..., R:]], -1).to(x.dtype)


def _append(st):
    """The new rows at their slots, and bounds for the pages that became full."""
    case, pool = st["case"], st["pool"]
    H, D = case["hkv"], _dim(case)
    k = _turn(case, st["k"].reshape(-1, H, D), st["at_pos"], st.get("angle"))
    pool[st["at_page"], :, 0, :, st["at_slot"]] = k.view(-1, H, 2, D // 2)
    pool[st["at_page"], :, 1, :, st["at_slot"]] = st["v"].reshape(-1, H, 2, D // 2)
    st["bounds"][st["done"]] = _bounds_of(pool, st["done"])


def _sparse(st):
    case, pool, table = st["case"], st["pool"], st["table"]
    H, D, G = case["hkv"], _dim(case), case["hq"] // case["hkv"]
    rows, most = table.shape
    _append(st)
    q = _turn(case, st["q"].reshape(-1, case["hq"], D), st["at_pos"], st.get("angle")).view(rows, H, G, D)
    seen = st["at_pos"] + 1
    pages = (seen + P - 1) // P
    # scores: what no sum of the group's logits with a key of the page exceeds
    up, down = q.double().clamp(min=0).sum(2), q.double().clamp(max=0).sum(2)                    # [rows, Hkv, D]
    b = st["bounds"][table].double()                                                             # [rows, pages, Hkv, 2, D]
    score = ((b[..., 1, :] * up[:, None]).sum(-1) + (b[..., 0, :] * down[:, None]).sum(-1)).float().transpose(1, 2)
    index = torch.arange(most, device="cuda")
    always = (index < case["first"]) | (index >= pages[:, None] - case["last"])
    score = torch.where(always[:, None], math.inf, score)
    score = torch.where((index >= pages[:, None])[:, None], -math.inf, score)
    kept = min(case["budget"], most)
    pick = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :kept]               # [rows, Hkv, kept]
    pid = table[:, None].expand(rows, H, most).gather(-1, pick)
    head = torch.arange(H, device="cuda")[None, :, None]
    k, v = (pool[pid, head, x].transpose(3, 4).reshape(rows, H, kept * P, D).float() for x in (0, 1))
    token = (pick[..., None] * P + torch.arange(P, device="cuda")).flatten(-2)
    s = torch.matmul(q.float(), k.transpose(-1, -2).contiguous()) / math.sqrt(D)
    s = torch.where((token < seen[:, None, None])[:, :, None], s, -math.inf)
    w = torch.exp(s - s.amax(-1, keepdim=True))
    st["out"].copy_((torch.matmul(w, torch.where((token < seen[:, None, None])[..., None], v, 0.0)) / w.sum(-1, keepdim=True)).view(st["out"].shape))


def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if own:
        ctx, stream = st["ctx"], st["sess"].stream
        if kind == "rope":
            ctx.rope_rows(st["rope"], st["pos"], st["q"], st["q_out"], st["k"], st["k_out"], stream)
        elif kind == "append":
            ctx.kv_append_rope(st["kv"], st["n"], st["rope"], st["k"], st["v"], None, stream)
            ctx.kv_truncate(st["kv"], st["lengths"])
        elif kind == "bounds":
            ctx.kv_bounds(st["kv"], stream)
        else:
            if case["layers"] == 1:
                ctx.pred_sparse(st["kv"], st["n"], st["sparse"], st["q"], st["k"], st["v"], st["out"], None, stream)
            else:
                ctx.pred_begin_sparse(st["kv"], st["n"], st["sparse"], stream)
                for i in range(case["layers"]):
                    ctx.pred_layer_sparse(i, st["q"][i], st["k"][i], st["v"][i], st["out"][i], None, stream)
            ctx.kv_truncate(st["kv"], st["lengths"])
    elif kind == "rope":
        st["q_out"], st["k_out"] = (_turn(case, st[x], st["pos"], st["angle"]) for x in "qk")
    elif kind == "append":
        _append(st)
    elif kind == "bounds":
        st["bounds"][st["full"]] = _bounds_of(st["pool"], st["full"])
    else:
        _sparse(st)
    if kind == "rope":
        return {"q": st["q_out"], "k": st["k_out"]}
    if kind == "bounds":
        return {"bounds": st["bounds"]}
    return {"pool": st["pool"], "bounds": st["bounds"], **({"out": st["out"]} if kind == "sparse" else {})}


# ---- the definition in 64 bits ----------------------------------------------------------------

def _turned(case, x, pos):
    """x [n, heads, D] in 64 bits, every pair a complex number times m e^(i angle)."""
    x = x.double().clone()
    if case["layout"] == "none":
        return x
    R = case["dims"]
    for i, f in enumerate(_frequencies(case)):
        a, b = (i, i + R // 2) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full((len(pos), 1), case["mag"], dtype=torch.float64, device="cuda"), torch.as_tensor(pos * f, device="cuda")[:, None])
        x[..., a], x[..., b] = z.real, z.imag
    return x


def exact(case, seed):
    x, kind = _inputs(case, seed), case["kind"]
    if kind == "rope":
        pos = _positions(case).astype(np.float64)
        return {"q": _turned(case, x["q"], pos), "k": _turned(case, x["k"], pos)}
    D, H, layers, G = _dim(case), case["hkv"], case.get("layers", 1), case["hq"] // case["hkv"]
    lens, new = _files(case)
    pages, _, tables = _tables(case)
    pool, rows = x["pool"], lambda p, kv: p[:, :, kv].permute(0, 3, 1, 2, 4).reshape(-1, H, D)  # noqa: E731
    bounds = torch.zeros((layers * pages, H, 2, D), dtype=torch.float64, device="cuda")
    out = torch.zeros((layers, sum(new), case["hq"], D), dtype=torch.float64, device="cuda") if kind == "sparse" else None
    for layer in range(layers):
        t = 0
        for table, n, m in zip(tables, lens, new):
            if not len(table):
                continue
            at = torch.as_tensor(table + layer * pages, device="cuda")
            pos = np.arange(n, n + m, dtype=np.float64)
            if m:
                k, v = rows(pool[at], 0), rows(pool[at], 1)
                k[n:n + m] = _turned(case, x["k"][layer, t:t + m], pos).to(k.dtype)              # the cache holds rounded keys
                v[n:n + m] = x["v"][layer, t:t + m]
                pool[at] = torch.stack([k, v], 1).view(len(table), P, 2, H, 2, D // 2).permute(0, 3, 2, 4, 1, 5)
            full = (n + m) // P
            keys = rows(pool[at], 0).double().view(-1, P, H, D)
            bounds[at[:full]] = torch.stack([keys[:full].amin(1), keys[:full].amax(1)], 2)
            for i in range(m if kind == "sparse" else 0):
                seen = n + i + 1
                count = -(-seen // P)
                q = _turned(case, x["q"][layer, t + i:t + i + 1], pos[i:i + 1]).to(_type(case)).double()[0].view(H, G, D)
                take = torch.ones((H, count), dtype=torch.bool, device="cuda")
                if count > case["budget"]:
                    lo, hi = case["first"], count - case["last"]
                    b = bounds[at[lo:hi]]                                                        # [pages, Hkv, 2, D]
                    score = torch.maximum(q[None] * b[:, :, None, 0], q[None] * b[:, :, None, 1]).sum((-1, -2)).float()
                    take[:, lo:hi] = False
                    order = torch.sort(score, dim=0, descending=True, stable=True).indices[:case["budget"] - case["first"] - case["last"]]
                    take[:, lo:hi] = take[:, lo:hi].scatter(1, order.t(), True)
                w = torch.repeat_interleave(take, P, 1)[:, :seen]                                # [Hkv, tokens]
                k, v = (rows(pool[at[:count]], kv)[:seen].double() for kv in (0, 1))
                s = (q[None] * k[:, :, None]).sum(-1).permute(1, 2, 0) / math.sqrt(D) if G * seen < 40000 else torch.stack([torch.mv(k[:, h], q[h, j]) for h in range(H) for j in range(G)]).view(H, G, seen) / math.sqrt(D)
                p = torch.softmax(s.masked_fill(~w[:, None], -math.inf), -1)
                out[layer, t + i] = torch.stack([torch.mm(p[h], v[:, h].contiguous()) for h in range(H)]).view(case["hq"], D)
            t += m
    if kind == "bounds":
        return {"bounds": bounds}
    return {"pool": pool.double() if pool.numel() < 1 << 29 else None, "bounds": bounds, **({"out": out} if kind == "sparse" else {})}


def work(case):
    H, D, kind = case["hkv"], _dim(case), case["kind"]
    row = 256                                                    # bytes of a head's row, of either type
    if kind == "rope":
        return {"bytes": 2 * case["tokens"] * (case["hq"] + H) * row, "flops": 3 * case["tokens"] * (case["hq"] + H) * case["dims"]}
    lens, new = _files(case)
    if kind == "bounds":
        full = sum(n // P for n in lens)
        return {"bytes": max(1, full) * H * (P * row + 2 * row), "flops": 2 * full * H * P * D}
    done = sum((n + m) // P - n // P for n, m in zip(lens, new))
    held = sum(n % P for n, m in zip(lens, new) if (n + m) // P > n // P)
    appended = sum(new) * 4 * H * row + done * H * 2 * row + held * H * row
    if kind == "append":
        return {"bytes": appended, "flops": 3 * sum(new) * H * case["dims"]}
    scored = kept = score_pairs = pairs = 0
    for n, m in zip(lens, new):
        last = -(-(n + m) // P)
        if last > case["budget"]:
            scored += last - case["first"] - case["last"]        # bounds are read once for the tokens of a file
        for i in range(m):
            c = -(-(n + i + 1) // P)
            k = min(c, case["budget"])
            kept += k
            pairs += (k - 1) * P + (n + i) % P + 1
            score_pairs += max(0, c - case["first"] - case["last"]) if c > case["budget"] else 0
    T, es = sum(new), 4 if case["dtype"] == "f32" else 2
    if max(new) > 1:                                             # new tokens of a file may choose the same pages
        kept = min(kept, sum(-(-(n + m) // P) for n, m in zip(lens, new)))
    return {"bytes": case["layers"] * (appended + scored * H * 2 * row + kept * H * 2 * P * row + T * case["hq"] * D * (es + 4)),
            "flops": case["layers"] * (4 * case["hq"] * D * pairs + 4 * H * D * score_pairs)}
