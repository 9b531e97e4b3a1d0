"""Retrieval-augmented-generation workload of the paper's section 5 as a driver of the library:
a population of identical LIPs, each answering one request about a topic whose document (3000
tokens in the paper, 100 documents) must be in its KV file before the answer is decoded.  The
LIP logic is the paper's prompt caching: the KV files of the `retain` most requested topics are
kept and forked for every later request of the topic (the paper keeps the caches of its 20 most
popular topics and drops the rest); other topics are prefilled from scratch and
their file is removed with the request.  Topic popularity is skewed by a Pareto index (smaller
index = a few topics get most requests).

Everything that touches K/V runs through the C ABI (kv_open / kv_fork / kv_remove, pred batches
on the GPU); the firing times of the batches come from the library's controller (section 4.4).
Time is virtual: requests arrive by a seeded Poisson process, and every fired batch advances the
clock by its measured wall time (host work + GPU, synchronised), so throughput and latency are
those of a server that does nothing but this path.  Only attention is computed (no weights on
this path): Q/K/V rows are slices of fixed seeded random arrays, and sampled tokens do not exist.
With `beams` > 1 an answer is searched for with that many beams: the document's file is forked for each, every step's
preds are followed by the choice among their continuations (logits: slices of a fixed seeded random array), and the
beams' scores, tokens and files follow it.
Host logic and argument marshalling only; none of the method's arithmetic.
"""
import math
import time
from collections import deque
from dataclasses import dataclass

import numpy as np

from . import binding, synth


@dataclass
class RagConfig:
    n_docs: int = 100
    doc_tokens: int = 3000
    answer_tokens: int = 32
    retain: int = 20
    pareto_index: float = 1.0
    rate_per_s: float = 2000.0          # request arrivals (Poisson)
    n_requests: int = 400
    prefill_chunk: int = 512            # a document enters its file in pred calls of this many tokens
    max_batch: int = 64
    max_wait_us: float = 300.0
    seed: int = 2025
    beams: int = 1                      # of an answer; > 1: a pred call of an answer is as many rows
    vocab: int = 32768                  # of the logits that beams choose from


def topic_probabilities(n_docs, pareto_index, rng):
    """Request probability of every topic: weights drawn from a Pareto distribution with the given
    index (heavy tail for a small index), normalised."""
    w = rng.pareto(pareto_index, size=n_docs) + 1.0
    return w / w.sum()


class _Lip:
    __slots__ = ("rid", "topic", "arrival", "fid", "to_prefill", "to_decode", "hit", "beams")


class RagDriver:
    """sess: a driver.HipSession whose pool, workspace (max_lips >= max_batch * beams, max_tokens >=
    max_batch * max(prefill_chunk, beams)) are large enough.  trace=True records every file operation and batch
    (and keeps the outputs) so that the run can be replayed on the CPU model."""

    def __init__(self, sess, cfg, trace=False, timer=None):
        import torch
        self.torch = torch
        self.sess, self.cfg = sess, cfg
        self.timer = timer or binding.BatchTimer(cfg.max_batch, cfg.max_wait_us)
        s = sess.shape
        self.max_rows = cfg.max_batch * max(cfg.prefill_chunk, cfg.beams, 1)
        st = np.random.SeedSequence(cfg.seed).spawn(4)
        self.rng = np.random.Generator(np.random.PCG64(st[0]))
        # fixed seeded rows; a batch with T new tokens uses rows [0, T) of each
        self.q_host = synth._normal(st[1], (self.max_rows, s.n_q_heads, s.head_dim), s.dtype)
        self.k_host = synth._normal(st[2], (self.max_rows, s.n_kv_heads, s.head_dim), s.dtype)
        self.v_host = synth._normal(st[3], (self.max_rows, s.n_kv_heads, s.head_dim), s.dtype)
        from .driver import to_device
        self.q, self.k, self.v = (to_device(a, sess.device) for a in (self.q_host, self.k_host, self.v_host))
        self.out = torch.empty((self.max_rows, s.n_q_heads, s.head_dim), dtype=torch.float32, device=sess.device)
        if cfg.beams > 1:
            rows, B = cfg.max_batch * cfg.beams, cfg.beams
            g = torch.Generator().manual_seed(cfg.seed)
            self.logits = (2.0 * torch.randn((rows, cfg.vocab), generator=g)).to(sess.device, torch.bfloat16)
            # of every request: its beams' scores (at first they are one and the same) and tokens
            self.scores = torch.full((cfg.n_requests, B), -math.inf, device=sess.device)
            self.scores[:, 0] = 0.0
            self.tokens = torch.full((cfg.n_requests * B, cfg.answer_tokens), -1, dtype=torch.int32, device=sess.device)
            self.every = np.full(min(cfg.max_batch, cfg.n_requests), B, np.int32)
            self.nth = torch.arange(len(self.every), device=sess.device)
            self.best = [torch.empty(rows, dtype=t, device=sess.device) for t in (torch.float32, torch.int32, torch.int32)]
            self.scratch = torch.empty(max(binding.beam_scratch_bytes(self.every[:n], cfg.vocab, B) for n in range(1, len(self.every) + 1)),
                                       dtype=torch.uint8, device=sess.device)
        self.trace = [] if trace else None
        self.outputs = [] if trace else None
        self.next_fid = 0
        self.h = {}                      # file id -> handle

    # ---- file operations (recorded when tracing) ----------------------------------
    def _open(self):
        fid = self.next_fid
        self.next_fid += 1
        self.h[fid] = self.sess.ctx.kv_open(None)
        if self.trace is not None:
            self.trace.append(("open", fid))
        return fid

    def _fork(self, parent):
        fid = self.next_fid
        self.next_fid += 1
        self.h[fid] = self.sess.ctx.kv_fork(self.h[parent])
        if self.trace is not None:
            self.trace.append(("fork", fid, parent))
        return fid

    def _remove(self, fid):
        self.sess.ctx.kv_remove(self.h.pop(fid))
        if self.trace is not None:
            self.trace.append(("remove", fid))

    def _spread(self, parent):
        """A fork of the file for every beam, last pages their own."""
        fids = list(range(self.next_fid, self.next_fid + self.cfg.beams))
        self.next_fid += len(fids)
        self.h.update(zip(fids, map(int, self.sess.ctx.kv_fork_batch([self.h[parent]] * len(fids), True, self.sess.stream))))
        if self.trace is not None:
            self.trace.append(("fork_batch", fids, [parent] * len(fids)))
        return fids

    def _remove_all(self, fids):
        self.sess.ctx.kv_remove_batch([self.h.pop(f) for f in fids])
        if self.trace is not None:
            self.trace.append(("remove_batch", list(fids)))

    def _choose(self, lips):
        """A step of these requests' searches: the best continuations of their beams, whose scores, tokens and files follow them."""
        torch, ctx, B, n, stream = self.torch, self.sess.ctx, self.cfg.beams, len(lips), self.sess.stream
        rid, at = torch.tensor([[lip.rid for lip in lips], [self.cfg.answer_tokens - lip.to_decode for lip in lips]], device=self.sess.device)
        best, beam, token = (x[:n * B] for x in self.best)
        ctx.beam_select(self.every[:n], B, self.logits[:n * B], self.scores[rid].flatten(), best, beam, token, self.scratch, None, stream)
        self.scores[rid] = best.view(n, B)
        of_request = self.tokens.view(-1, B, self.cfg.answer_tokens)
        tokens = of_request[rid]                             # this batch's alone, whatever the run's length
        rows = tokens.flatten(0, 1)
        ctx.beam_states(self.every[:n], beam, binding.make_states([(rows, rows, 0)]), stream)
        tokens[self.nth[:n], :, at] = token.view(n, B)
        of_request[rid] = tokens
        files = [f for lip in lips for f in lip.beams]
        sources = beam.cpu().numpy()
        sources = np.where(sources < 0, -1, sources + np.repeat(np.arange(n) * B, B))
        ctx.kv_reorder([self.h[f] for f in files], sources, True, stream)
        if self.trace is not None:
            self.trace.append(("reorder", files, sources.tolist()))

    # ---- the run -------------------------------------------------------------------
    def run(self):
        cfg, torch = self.cfg, self.torch
        probs = topic_probabilities(cfg.n_docs, cfg.pareto_index, self.rng)
        arrivals = np.cumsum(self.rng.exponential(1e6 / cfg.rate_per_s, size=cfg.n_requests))   # microseconds
        topics = self.rng.choice(cfg.n_docs, size=cfg.n_requests, p=probs)
        counts = np.zeros(cfg.n_docs, np.int64)
        cache = {}                       # topic -> file id of the retained document KV
        calls = deque()                  # pending pred calls: (lip, n_tokens), oldest first
        stream = self.sess.stream
        now, k = 0.0, 0
        done, lat, batches, busy = 0, [], [], 0.0
        hits = steps = prefilled = 0

        def submit(lip, t):
            n = min(cfg.prefill_chunk, lip.to_prefill) if lip.to_prefill > 0 else 1
            calls.append((lip, n))
            self.timer.arrive(t)

        def admit(t, rid):
            nonlocal hits
            lip = _Lip()
            lip.rid, lip.topic, lip.arrival = rid, int(topics[rid]), t
            counts[lip.topic] += 1
            lip.to_decode, lip.beams = cfg.answer_tokens, None
            if lip.topic in cache:       # prompt cache hit: share the document's pages
                lip.to_prefill, lip.hit = 0, True
                if cfg.beams > 1:
                    lip.fid, lip.beams = None, self._spread(cache[lip.topic])
                else:
                    lip.fid = self._fork(cache[lip.topic])
                hits += 1
            else:
                lip.fid, lip.to_prefill, lip.hit = self._open(), cfg.doc_tokens, False
            submit(lip, t)

        def retain_after_prefill(lip):
            """The document is in lip.fid: keep it if the topic is among the `retain` most requested."""
            if lip.topic in cache or cfg.retain <= 0:
                return
            if len(cache) >= cfg.retain:
                coldest = min(cache, key=lambda t: (counts[t], t))
                if counts[coldest] >= counts[lip.topic]:
                    return
                self._remove(cache.pop(coldest))
            cache[lip.topic] = lip.fid                    # the prefilled file becomes the cached one
            lip.fid = self._fork(lip.fid)                 # the request continues on a fork

        while done < cfg.n_requests:
            while k < cfg.n_requests and arrivals[k] <= now:
                admit(float(arrivals[k]), k)
                k += 1
            fire = self.timer.decide(now, True)
            if fire == 0:
                nxt = min(float(arrivals[k]) if k < cfg.n_requests else math.inf, self.timer.next_deadline())
                assert nxt < math.inf and nxt > now, "scheduler waits with nothing to wait for"
                now = nxt
                continue
            self.timer.fired(fire)
            batch = [calls.popleft() for _ in range(fire)]
            fids, nt = [], []
            for lip, n in batch:
                fids += lip.beams or [lip.fid]
                nt += [n] * (len(lip.beams) if lip.beams else 1)
            kv = [self.h[f] for f in fids]
            T = sum(nt)
            t0 = time.perf_counter()
            self.sess.ctx.pred_batch(kv, nt, self.q, self.k, self.v, self.out, stream)
            if self.trace is not None:
                self.trace.append(("pred", fids, nt))
            searching = [lip for lip, _ in batch if lip.beams]
            if searching:
                self._choose(searching)
            torch.cuda.current_stream(self.sess.device).synchronize()
            dt = (time.perf_counter() - t0) * 1e6
            if self.trace is not None:
                self.outputs.append(self.out[:T].cpu().numpy().copy())
            now += dt
            busy += dt
            self.timer.done(fire, dt)
            batches.append(fire)
            steps += fire
            for lip, n in batch:
                if lip.to_prefill > 0:
                    lip.to_prefill -= n
                    prefilled += n
                    if lip.to_prefill == 0:
                        retain_after_prefill(lip)
                        if cfg.beams > 1:
                            lip.beams = self._spread(lip.fid)
                            self._remove(lip.fid)
                else:
                    lip.to_decode -= 1
                if lip.to_prefill == 0 and lip.to_decode == 0:
                    if lip.beams:
                        self._remove_all(lip.beams)
                    else:
                        self._remove(lip.fid)
                    lat.append(now - lip.arrival)
                    done += 1
                else:
                    submit(lip, now)
        self.cache = cache
        lat = np.array(lat)
        return dict(requests=done, seconds=now / 1e6, requests_per_s=done / (now / 1e6), lip_steps_per_s=steps / (now / 1e6),
                    pred_calls=steps, batches=len(batches), mean_batch=float(np.mean(batches)), hit_rate=hits / max(done, 1),
                    latency_ms_mean=float(lat.mean() / 1e3), latency_ms_p50=float(np.percentile(lat, 50) / 1e3),
                    latency_ms_p95=float(np.percentile(lat, 95) / 1e3), gpu_busy_frac=busy / now, tokens_prefilled=prefilled,
                    cached_topics=len(cache), scheduler=self.timer.state())

    def close(self):
        for fid in list(self.h):
            self.sess.ctx.kv_remove(self.h.pop(fid))
        self.timer.close()
