"""Beams beside the cache, as defined (test infrastructure, CPU only): the choice of a search step in 64 bits, and the file
system's batched forks, reordering and withdrawn pages on top of its state model.

Score of token v after beam b: score_b + x_bv - log sum exp over what row b allows.  Not finite: no choice.  Of equal scores the lower
beam, then the lower token.

Reordering: file i holds afterwards what file from[i] held before.  With `own_last` the copies that the files' next appends would make are made at
once: of files whose partly filled last page has several references, those that took something first, in order, then the others.
Withdrawing pages: what is in use moves, lowest page first, to the free page of lowest rank outside; the pages leave the free set.
"""
import heapq

import numpy as np

from .kvfs_model import EBADF, EBUSY, EINVAL, ENOSPC, KVError, KVFSModel


def select(logits, scores, beams, n_best, allowed=None):
    """logits [rows, vocab], scores [rows]; allowed [rows, vocab] truth values.  Returns scores (float64), beams, tokens [groups, n_best]."""
    x = np.asarray(logits, np.float64)
    groups, row = len(beams), 0
    best, beam, token = np.full((groups, n_best), -np.inf), np.full((groups, n_best), -1), np.full((groups, n_best), -1)
    for g, n in enumerate(beams):
        found = []
        for b in range(n):
            v = np.arange(x.shape[1]) if allowed is None else np.flatnonzero(allowed[row + b])
            y = x[row + b, v]
            if len(y) and np.isfinite(scores[row + b]) and not np.isnan(y).any() and y.max() < np.inf and y.max() > -np.inf:
                lse = np.log(np.exp(y - y.max()).sum())              # from the largest: of far values nothing is lost
                order = np.lexsort((v, -y))[:n_best]
                found += [(-(float(scores[row + b]) + ((y[i] - y.max()) - lse)), b, -y[i], v[i]) for i in order if y[i] > -np.inf]
        for k, (s, b, _, v) in enumerate(sorted(found)[:n_best]):
            best[g, k], beam[g, k], token[g, k] = -s, b, v
        row += n
    return best, beam, token


class BeamFiles(KVFSModel):
    """The state model with the batched calls.  Calls that copy return (source, destination, slots) triples."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.gone = set()                          # withdrawn pages

    def kv_fork_batch(self, parents, own_last):
        files = [self._file(h, usable=True) for h in parents]
        if own_last and sum(f.length % self.P != 0 for f in files) > self.free_pages():
            raise KVError(ENOSPC)
        new, copies = [], []
        for h in parents:
            new.append(self.kv_fork(h))
            if own_last:
                copies += self._own(new[-1])
        return new, copies

    def _own(self, h):
        f = self._file(h)
        r = f.length % self.P
        if r == 0 or self.refcount[f.pages[-1]] == 1:
            return []
        if not self.free_ranks:
            raise KVError(ENOSPC)
        src = f.pages[-1]
        f.pages[-1] = self._alloc()
        self.refcount[src] -= 1
        return [(src, f.pages[-1], r)]

    def kv_reorder(self, kv, sources, own_last):
        files = [self._file(h, usable=True) for h in kv]
        if any(s < -1 or s >= len(kv) for s in sources):
            raise KVError(EINVAL)
        if len({id(f) for f in files}) < len(files):
            raise KVError(EBUSY)
        before = self.refcount.copy(), list(self.free_ranks), [(list(f.pages), f.length) for f in files]
        takes = [i for i, s in enumerate(sources) if s not in (-1, i)]
        forks = {i: self.kv_fork(kv[sources[i]]) for i in takes}            # what each is to hold, while all are as they were
        for i in takes:
            fork = self._file(forks[i])
            self._release_pages(files[i])
            files[i].pages, files[i].length = fork.pages, fork.length
            del self.handles[forks[i]]
        copies = []
        try:
            if own_last:
                for i in takes + [i for i in range(len(kv)) if i not in takes]:
                    copies += self._own(kv[i])
        except KVError:
            self.refcount, self.free_ranks = before[0], before[1]
            for f, (pages, length) in zip(files, before[2]):
                f.pages, f.length = pages, length
            raise
        return copies

    def kv_remove_batch(self, kv):
        files = [self._file(h) for h in kv]
        if len({id(f) for f in files}) < len(files):
            raise KVError(EBUSY)
        for h in kv:
            self.kv_remove(h)

    def pool_withdraw(self, first, n):
        if first < 0 or n < 0 or first + n > self.n_pages or any(p in self.gone for p in range(first, first + n)):
            raise KVError(EINVAL)
        inside = {int(self.rank[p]) for p in range(first, first + n)}
        used = [p for p in range(first, first + n) if self.refcount[p] > 0]
        outside = [r for r in self.free_ranks if r not in inside]
        if len(used) > len(outside):
            raise KVError(ENOSPC)
        self.gone |= set(range(first, first + n))
        self.free_ranks = outside
        heapq.heapify(self.free_ranks)
        files, copies = list({id(f): f for f in list(self.handles.values()) + list(self.names.values())}.values()), []
        for p in used:
            q, slots = int(self.order[heapq.heappop(self.free_ranks)]), 0
            self.refcount[q], self.refcount[p] = self.refcount[p], 0
            for f in files:
                for i, e in enumerate(f.pages):
                    if e == p:
                        f.pages[i] = q
                        slots = max(slots, min(self.P, f.length - i * self.P))
            if p in self.waiters:
                self.waiters[q] = self.waiters.pop(p)
            copies.append((p, q, slots))
        return copies

    def pool_return(self, first, n):
        if first < 0 or n < 0 or first + n > self.n_pages or any(p not in self.gone for p in range(first, first + n)):
            raise KVError(EINVAL)
        for p in range(first, first + n):
            self.gone.discard(p)
            heapq.heappush(self.free_ranks, int(self.rank[p]))
