"""Beam search beside the cache - selection, state rows, files - and the pool's page copies: the work to be measured, with its plain form.

A case is one pass through one operator, on inputs and files that are already there.

Kinds of cases
  select    logits [rows, vocab] of `groups` requests with U{beams_lo..beams_hi} beams each: of every request the `best` continuations (beam,
            token) of largest score, score = beam's score + log softmax.  `first`: share of requests at their first step, where only
            one beam lives; `mask`: share of rows with a grammar, whose rows allow 0, 20, half or all but 20 of the tokens
  states    rows of `arrays` arrays [outer][rows][width] of `kind_of` values, row r becomes the row of its parent, in place
  reorder   files of `groups` requests of U{beams_lo..beams_hi} beams, a prompt of U{lo..hi} tokens that a request's beams share and U{0..own_hi} tokens of
            their own: beams that lost take over the file of one that survives, last pages copied at once
  fork      `groups` files of U{lo..hi} tokens forked U{beams_lo..beams_hi} times each, last pages copied at once; the forks are removed again
  withdraw  the lower half of the pool emptied into the upper half, and back: `lips` files of U{lo..hi} tokens, `full` of the half in use
Everywhere: `layers` of the pool; `scatter`: pages of a file in random places; `lens`: seed of lengths, parents and masks' kinds.

The cache is the documented page layout, [page][kv head][K, V][row half][16 tokens][half a row]; page p of layer l is page
l * pages + p.  Parents are such that a second pass leaves what the first one made.
"""
import math
import random

import numpy as np
import torch

own = False
P = 16          # tokens per page


def listed():
    kv = dict(dtype="bf16", hq=32, hkv=8)
    return [
        # One user's search of four beams: launch latency.
        dict(name="select_1x4", kind="select", dtype="bf16", groups=1, beams_lo=4, beams_hi=4, vocab=32768, best=8, first=0.0, mask=0.0, lens=1),
        # A loaded server's step, four beams each, a large vocabulary.
        dict(name="select_64x4", kind="select", dtype="bf16", groups=64, beams_lo=4, beams_hi=4, vocab=131072, best=8, first=0.1, mask=0.0, lens=2),
        # Requests of different widths, some with grammars, rows that begin at odd addresses.
        dict(name="select_grammar", kind="select", dtype="f16", groups=24, beams_lo=1, beams_hi=8, vocab=100003, best=16, first=0.1, mask=0.6, lens=3),
        # fp32 logits, wide searches.
        dict(name="select_f32_wide", kind="select", dtype="f32", groups=64, beams_lo=16, beams_hi=16, vocab=65537, best=32, first=0.0, mask=0.0, lens=4),
        # Token histories and lengths of one user's beams.
        dict(name="states_1x4", kind="states", kind_of="i32", groups=1, beams_lo=4, beams_hi=4, arrays=2, outer=1, width=517, lens=27),
        # Recurrent states of a server's beams through eight layers.
        dict(name="states_64x4", kind="states", kind_of="bf16", groups=64, beams_lo=2, beams_hi=6, arrays=2, outer=8, width=16384, lens=6),
        # Four beams of one user, eight layers.
        dict(name="reorder_1x4", kind="reorder", groups=1, beams_lo=4, beams_hi=4, lo=1500, hi=2500, own_hi=100, layers=8, scatter=False, lens=7, **kv),
        # A server's beams.
        dict(name="reorder_64x4", kind="reorder", groups=64, beams_lo=4, beams_hi=4, lo=512, hi=4096, own_hi=200, layers=4, scatter=True, lens=8, **kv),
        # One prompt sampled eight times, fp32 storage.
        dict(name="fork_f32_1x8", kind="fork", dtype="f32", hq=8, hkv=8, groups=1, beams_lo=8, beams_hi=8, lo=300, hi=700, layers=1, scatter=False, lens=9),
        # Prompts that become beams.
        dict(name="fork_32x8", kind="fork", groups=32, beams_lo=4, beams_hi=12, lo=512, hi=4096, layers=8, scatter=False, lens=10, **kv),
        # A small pool lent and taken back.
        dict(name="withdraw_1", kind="withdraw", dtype="bf16", hq=8, hkv=2, lips=1, lo=500, hi=1000, full=1.0, layers=1, scatter=False, lens=11),
        # Half of a server's pool lent to another use and taken back, pages all over it.
        dict(name="withdraw_64", kind="withdraw", lips=64, lo=512, hi=4096, full=0.7, layers=2, scatter=True, lens=12, **kv),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, evenly spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["select", "select", "select", "states", "reorder", "fork", "withdraw"])
    c = dict(kind=kind, lens=rng.randrange(1, 1 << 30))
    if kind == "withdraw":
        dtype, hkv = rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 4, 8])
        lo, layers = _log(rng, 1, 2048), rng.choice([1, 1, 2, 3])
        lips = max(1, min(_log(rng, 1, 64), 150000 // (lo * layers)))
        return dict(c, dtype=dtype, hkv=hkv, hq=hkv * rng.choice([1, 4]), lips=lips, lo=lo, hi=2 * lo, full=rng.choice([1.0, 0.9, 0.5]), layers=layers, scatter=rng.random() < 0.6)
    lo = rng.choice([1, 2, 4, 4, 8, _log(rng, 1, 32)])
    c.update(groups=_log(rng, 1, max(1, 256 // lo)), beams_lo=lo, beams_hi=min(64, rng.choice([lo, lo, 2 * lo])))
    rows = c["groups"] * c["beams_hi"]
    if kind == "select":
        vocab = min(_log(rng, 2, 131072), 60_000_000 // rows)
        return dict(c, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), vocab=vocab, best=min(128, rng.choice([1, lo, 2 * lo, 2 * lo, _log(rng, 1, 128)])),
                    first=rng.choice([0.0, 0.0, 0.3, 1.0]), mask=rng.choice([0.0, 0.0, 0.5, 1.0]))
    if kind == "states":
        kind_of, outer, arrays = rng.choice(["bf16", "i32", "f32", "i8"]), rng.choice([1, 1, 4, 8]), rng.randint(1, 4)
        return dict(c, kind_of=kind_of, arrays=arrays, outer=outer, width=min(_log(rng, 1, 65536), max(1, 60_000_000 // (rows * outer * arrays))))
    dtype, hkv, layers = rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 5])
    lo = min(_log(rng, 1, 4096), max(1, 200000 // (c["groups"] * layers)))
    c.update(dtype=dtype, hkv=hkv, hq=hkv * rng.choice([1, 4]), lo=lo, hi=2 * lo, layers=layers, scatter=rng.random() < 0.4)
    return dict(c, own_hi=rng.choice([1, 20, 100])) if kind == "reorder" else c


# ---- what a case consists of ------------------------------------------------------------------

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32, "i8": torch.int8}


def _dim(case):
    return 128 if case["dtype"] == "bf16" else 64


def _beams(case):
    """Beams of each request, and the seeded numbers that follow."""
    r = np.random.Generator(np.random.PCG64(case["lens"]))
    return r.integers(case["beams_lo"], case["beams_hi"] + 1, case["groups"]).astype(np.int32), r


def _parents(beams, r):
    """Per row the beam of its request whose state it takes: those that survive keep theirs."""
    got = []
    for b in beams:
        keeps = r.random(b) < 0.6
        keeps[r.integers(0, b)] = True
        got.append(np.where(keeps, np.arange(b), r.choice(np.flatnonzero(keeps), b)))
    return np.concatenate(got).astype(np.int32)


def _files(case):
    """Every file's pages as they are before the call, its tokens, the order in which pages are given out, and the pool's pages."""
    kind, tables, lens, used = case["kind"], [], [], 0
    if kind == "withdraw":
        r = np.random.Generator(np.random.PCG64(case["lens"]))
        lens = r.integers(case["lo"], case["hi"] + 1, case["lips"])
        used = int((-(-lens // P)).sum())
        half = max(used, int(round(used / case["full"])))
        place = r.permutation(half)[:used] if case["scatter"] else np.arange(used)
        at = np.concatenate([[0], np.cumsum(-(-lens // P))])
        return [place[at[i]:at[i + 1]] for i in range(len(lens))], lens, np.arange(2 * half), 2 * half
    beams, r = _beams(case)
    for b in beams:
        n = int(r.integers(case["lo"], case["hi"] + 1))
        prompt = np.arange(used, used + n // P)                     # full pages, shared by the request's beams
        used += len(prompt)
        if kind == "fork":
            rest = np.arange(used, used + (n % P > 0))
            used += len(rest)
            tables.append(np.concatenate([prompt, rest]))
            lens.append(n)
            continue
        more = int(r.integers(0, case["own_hi"] + 1))               # beams of a request are equally long
        mine = -(-(n % P + more) // P)
        for i in range(b):
            tables.append(np.concatenate([prompt, np.arange(used, used + mine)]))
            lens.append(n + more)
            used += mine
    pages = used + int(beams.sum()) + 2
    order = r.permutation(pages) if case["scatter"] else np.arange(pages)
    return [order[t] for t in tables], np.array(lens), order, pages


def _copies(case):
    """(source page, destination page, filled slots) of the copies of a pass, in order."""
    tables, lens, order, pages = _files(case)
    if case["kind"] == "withdraw":
        half, used = pages // 2, np.sort(np.concatenate(tables))
        there = half + np.arange(len(used))
        filled = np.full(pages, P)
        for t, n in zip(tables, lens):
            filled[t[-1]] = (n - 1) % P + 1
        return used, there, filled[used]
    rank = np.empty(pages, np.int64)
    rank[order] = np.arange(pages)
    beams, r = _beams(case)
    if case["kind"] == "fork":
        take = np.repeat(np.arange(len(beams)), beams)
        taken = np.concatenate(tables)
    else:
        first = np.repeat(np.concatenate([[0], np.cumsum(beams)[:-1]]), beams)
        src = _reordered(case) + first
        take = src[src != np.arange(len(src))]
        taken = np.concatenate([tables[i] for i in sorted(set(src))])
    free = np.setdiff1d(np.arange(pages), taken)
    free = free[np.argsort(rank[free])]
    take = take[lens[take] % P != 0]
    return np.array([tables[i][-1] for i in take], np.int64), free[:len(take)], lens[take] % P


def _reordered(case):
    return _parents(_beams(case)[0], np.random.Generator(np.random.PCG64(case["lens"] + 1)))


def _allowed(case, seed, rows):
    """Bits [rows][words] of the tokens that a row allows, or None; kind of every row: 0 none, 1 twenty, 2 half, 3 all but twenty, 4 all."""
    if not case["mask"]:
        return None, None
    r = np.random.Generator(np.random.PCG64([case["lens"], 2]))
    kind = np.where(r.random(rows) < case["mask"], r.integers(0, 4, rows), 4)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    V = case["vocab"]
    some = torch.randint(0, V, (rows, 20), generator=g, device="cuda")
    half = torch.rand((rows, V), generator=g, device="cuda") < 0.5
    k = torch.as_tensor(kind, device="cuda")[:, None]
    few = torch.zeros((rows, V), dtype=torch.bool, device="cuda").scatter_(1, some, True)
    bits = (k == 4) | ((k == 1) & few) | ((k == 2) & half) | ((k == 3) & ~few)
    bits = torch.nn.functional.pad(bits, (0, -V % 32)).view(rows, -1, 32).long()
    return (bits << torch.arange(32, device="cuda")).sum(-1).to(torch.int32), kind      # (two's complement: the low 32 bits)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind in ("select", "states"):
        beams, r = _beams(case)
        rows = int(beams.sum())
    if kind == "select":
        t, V = TYPES[case["dtype"]], case["vocab"]
        x = torch.randn((rows, V), generator=g, device="cuda").mul_(2.0)
        x += 6.0 * (torch.rand((rows, V), generator=g, device="cuda") < 8.0 / V)        # the tokens that a model has in mind
        scores = -30.0 * torch.rand((rows,), generator=g, device="cuda")
        row, dead = 0, torch.zeros(rows, dtype=torch.bool)
        for b in beams:                                                                 # at the first step one beam lives
            if r.random() < case["first"]:
                dead[row + 1:row + b] = True
            row += b
        allowed, _ = _allowed(case, seed, rows)
        return dict(logits=x.to(t), scores=torch.where(dead.cuda(), -math.inf, scores), allowed=allowed)
    if kind == "states":
        t, s = TYPES[case["kind_of"]], (case["outer"], rows, case["width"])
        make = (lambda: torch.randn(s, generator=g, device="cuda", dtype=t)) if t.is_floating_point else (lambda: torch.randint(-100, 100, s, generator=g, device="cuda", dtype=t))
        return dict(states=[make() for _ in range(case["arrays"])])
    pages = _files(case)[3]
    return dict(pool=torch.randn((case["layers"], pages, case["hkv"] * 4, P, _dim(case) // 2), generator=g, device="cuda", dtype=TYPES[case["dtype"]]))


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    dev = lambda a, t=torch.int64: torch.as_tensor(np.asarray(a), device="cuda", dtype=t)  # noqa: E731
    kind = case["kind"]
    if kind in ("select", "states"):
        beams, r = _beams(case)
        first = np.concatenate([[0], np.cumsum(beams)])
        st["beams"] = beams
    if kind == "select":
        G, K = case["groups"], case["best"]
        most = int(beams.max())
        at = first[:-1, None] + np.arange(most)
        st.update(row=dev(np.where(np.arange(most) < beams[:, None], at, 0)), there=dev(np.arange(most) < beams[:, None], torch.bool),
                  best=torch.empty((G, K), device="cuda"), parent=torch.empty((G, K), dtype=torch.int32, device="cuda"), token=torch.empty((G, K), dtype=torch.int32, device="cuda"))
    elif kind == "states":
        parents = _reordered(case)
        st.update(parents=dev(parents, torch.int32), row=dev(parents + np.repeat(first[:-1], beams)))
    else:
        src, dst, filled = _copies(case)
        st.update(src=dev(src), dst=dev(dst), within=dev(np.arange(P) < np.asarray(filled)[:, None], torch.bool))
    if own:
        st.update(_session(case, st))
    torch.cuda.synchronize()
    return st


def _session(case, st):
    """The library's side: a context (over the pool), its files, what the calls are given."""
    from paper_2510_25412_amd import binding, driver, synth
    kind = case["kind"]
    if kind in ("select", "states"):
        sess = driver.HipSession(synth.Shape(8, 8, 128, P, "bf16"), 4, None, "cuda:0", max_lips=1, max_tokens=64, max_entries=64)
        got = dict(sess=sess, ctx=sess.ctx)
        if kind == "select":
            got["scratch"] = torch.empty(binding.beam_scratch_bytes(st["beams"], case["vocab"], case["best"]), dtype=torch.uint8, device="cuda")
        else:
            got["plan"] = binding.make_states([(x, x, 1) for x in st["states"]])
        return got
    tables, lens, order, pages = _files(case)
    shape = synth.Shape(case["hq"], case["hkv"], _dim(case), P, case["dtype"])
    sess = driver.HipSession(shape, pages, order.astype(np.int32), "cuda:0", max_lips=max(64, len(lens)), max_tokens=1024, max_entries=pages + 64, n_layers=case["layers"])
    ctx, got = sess.ctx, dict(sess=sess, ctx=sess.ctx)
    pool = sess.pool.view(TYPES[case["dtype"]]).view(st["pool"].shape)
    pool.copy_(st["pool"])
    got["pool"] = pool
    if kind == "withdraw":
        _lay(ctx, tables, lens)
        got["half"] = pages // 2
        return got
    if kind == "fork":
        kv = np.array([ctx.kv_open(None) for _ in lens], np.int32)
        some = np.flatnonzero(lens)
        ctx.plan_append(kv[some], lens[some])                    # the files' pages; their rows lie in the pool already
        got["parents"] = np.repeat(kv, _beams(case)[0])
        return got
    beams, _ = _beams(case)
    kv, row = [], 0
    for b in beams:                                              # full pages of the prompt, then each beam's own
        shared = 0
        while shared < len(tables[row]) and b > 1 and tables[row][shared] == tables[row + 1][shared]:
            shared += 1
        if b == 1:
            shared = len(tables[row])
        top = ctx.kv_open(None)
        if min(shared * P, lens[row]):
            ctx.plan_append([top], [min(shared * P, lens[row])])
        mine = [top] + [ctx.kv_fork(top) for _ in range(b - 1)]
        for h in mine:
            if lens[row] > shared * P:
                ctx.plan_append([h], [lens[row] - shared * P])
        kv += mine
        row += b
    got["kv"] = np.array(kv, np.int32)
    first = np.repeat(np.concatenate([[0], np.cumsum(beams)[:-1]]), beams)
    got["take"] = (_reordered(case) + first).astype(np.int32)
    return got


def _lay(ctx, tables, lens):
    """Files whose pages lie where `tables` says, in a pool that gives pages out in their order: a file of each page, joined."""
    hold = []
    for _ in range(max(int(t.max()) for t in tables) + 1):
        hold.append(ctx.kv_open(None))
        ctx.plan_append([hold[-1]], [P])
    for t, n in zip(tables, lens):
        ctx.kv_truncate([ctx.kv_merge([hold[p] for p in t])], [int(n)])      # whole pages: referenced, in the file's order
    for h in hold:
        ctx.kv_remove(h)


# ---- the plain form ---------------------------------------------------------------------------

def _select(st):
    """Per row the best tokens and the normaliser, then the best of a request's rows; 64 bits: which is chosen hangs on comparisons."""
    case, x = st["case"], st["logits"].float()
    V, K = case["vocab"], case["best"]
    if st["allowed"] is not None:
        bit = (st["allowed"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bit.flatten(1)[:, :V] == 1, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x.double() - top.double())
    base = st["scores"].double() - (top[:, 0].double() + torch.log(e.sum(-1)))
    kept = min(K, V)
    value, token = torch.sort(x, dim=-1, descending=True, stable=True)
    score = base[:, None] + value[:, :kept].double()
    score = torch.where(torch.isfinite(score), score, -math.inf)
    rows = st["row"]                                                                             # [groups, most beams]
    score = torch.where(st["there"][..., None], score[rows], -math.inf).flatten(1)
    score, at = torch.sort(score, dim=-1, descending=True, stable=True)
    found = min(K, score.shape[1])
    score, at = score[:, :found], at[:, :found]
    none = score == -math.inf
    st["best"].fill_(-math.inf)
    st["parent"].fill_(-1)
    st["token"].fill_(-1)
    st["best"][:, :found] = score.float()
    st["parent"][:, :found] = torch.where(none, -1, at // kept).int()
    st["token"][:, :found] = torch.where(none, -1, token[:, :kept][rows].flatten(1).gather(1, at)).int()


def _copy(pool, src, dst, within):
    """Filled slots of pages src to pages dst, in every layer."""
    pool[:, dst] = torch.where(within[None, :, None, :, None], pool[:, src], pool[:, dst])


def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if own:
        ctx, stream = st["ctx"], st["sess"].stream
        if kind == "select":
            ctx.beam_select(st["beams"], case["best"], st["logits"], st["scores"], st["best"], st["parent"], st["token"], st["scratch"], st["allowed"], stream)
        elif kind == "states":
            ctx.beam_states(st["beams"], st["parents"], st["plan"], stream)
        elif kind == "reorder":
            ctx.kv_reorder(st["kv"], st["take"], True, stream)
        elif kind == "fork":
            ctx.kv_remove_batch(ctx.kv_fork_batch(st["parents"], True, stream))
        else:
            half = st["half"]
            ctx.pool_withdraw(0, half, stream)
            ctx.pool_return(0, half)
            ctx.pool_withdraw(half, half, stream)
            ctx.pool_return(half, half)
    elif kind == "select":
        _select(st)
    elif kind == "states":
        st["states"] = [x[:, st["row"]] for x in st["states"]]
    else:
        _copy(st["pool"], st["src"], st["dst"], st["within"])
        if kind == "withdraw":                                   # back, to the lowest places; the filled slots of the next pass lie there too
            back = torch.arange(len(st["src"]), device="cuda")
            _copy(st["pool"], st["dst"], back, st["within"])
            st["src"] = back
    if kind == "select":
        return {"scores": st["best"], "parents": st["parent"], "tokens": st["token"]}
    return {"states": st["states"]} if kind == "states" else {"pool": st["pool"]}


# ---- the definition in 64 bits ----------------------------------------------------------------

def exact(case, seed):
    """Scores of a request's choices, every beam's whole distribution at hand; what is moved, one row or page after the other."""
    x, kind = _inputs(case, seed), case["kind"]
    if kind == "states":
        first, at = np.cumsum(_beams(case)[0]), np.arange(sum(_beams(case)[0]))
        first = np.concatenate([[0], first])[np.searchsorted(first, at, side="right")]
        took = [s.double() for s in x["states"]]
        for s, t in zip(x["states"], took):
            for row, parent in enumerate(_reordered(case)):
                t[:, row] = s[:, int(first[row]) + int(parent)]
        return {"states": took} if took[0].is_floating_point() else None
    if kind != "select":
        pool = x["pool"]
        if pool.numel() > 1 << 31:
            return None
        lists = [_copies(case)]
        if kind == "withdraw":
            lists.append((lists[0][1], np.arange(len(lists[0][1])), lists[0][2]))
        for pages in lists:
            old = pool[:, torch.as_tensor(np.asarray(pages[0]), device="cuda")]
            for i, (_, d, n) in enumerate(zip(*pages)):
                pool[:, int(d), :, :int(n)] = old[:, i, :, :int(n)]
        return {"pool": pool.double()}
    beams, _ = _beams(case)
    V, K = case["vocab"], case["best"]
    best = torch.full((case["groups"], K), -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for i, b in enumerate(beams):
        y = x["logits"][row:row + b].double()
        if x["allowed"] is not None:
            word = x["allowed"][row:row + b].long() & 0xffffffff
            v = torch.arange(V, device="cuda")
            y = y.masked_fill((word[:, v // 32] >> (v % 32)) % 2 == 0, -math.inf)
        p = torch.log_softmax(y, -1) + x["scores"][row:row + b, None].double()
        p = torch.nan_to_num(p, nan=-math.inf).flatten().sort(descending=True).values[:K]
        best[i, :len(p)] = p
        row += b
    return {"scores": best, "parents": None, "tokens": None}


def work(case):
    kind = case["kind"]
    if kind == "select":
        beams, r = _beams(case)
        V, rows, es = case["vocab"], int(beams.sum()), 4 if case["dtype"] == "f32" else 2
        live = np.ones(rows, bool)
        row = 0
        for b in beams:
            if r.random() < case["first"]:
                live[row + 1:row + b] = False
            row += b
        seen = np.full(rows, V)
        if case["mask"]:
            m = np.random.Generator(np.random.PCG64([case["lens"], 2]))
            masked = m.random(rows) < case["mask"]
            which = np.where(masked, m.integers(0, 4, rows), 4)
            seen = np.array([0, min(V, 20), V // 2, max(0, V - 20), V])[which]
        n = int(seen[live].sum())
        return {"bytes": n * es + (int(live.sum()) * -(-V // 32) * 4 if case["mask"] else 0) + rows * 4 + case["groups"] * case["best"] * 12, "flops": 4 * n + 1}
    if kind == "states":
        beams, _ = _beams(case)
        parents, first = _reordered(case), np.repeat(np.concatenate([[0], np.cumsum(beams)[:-1]]), beams)
        changed = parents != np.arange(len(parents)) - first
        read = len(set((parents + first)[changed]))
        return {"bytes": max(4, (read + int(changed.sum())) * case["arrays"] * case["outer"] * case["width"] * TYPES[case["kind_of"]].itemsize + 4 * len(parents)), "flops": 0}
    src, _, filled = _copies(case)
    slots = sum({int(s): int(f) for s, f in zip(src, filled)}.values()) + int(np.sum(filled))      # read once, however many take it
    return {"bytes": max(4, (2 if kind == "withdraw" else 1) * slots * case["hkv"] * 512 * case["layers"]), "flops": 0}
