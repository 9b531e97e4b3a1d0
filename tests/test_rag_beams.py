"""The steps of the RAG driver's searches (CPU only) on a stand-in for the library's calls: what they hand over is the batch's, however
many requests a run has, and every request's scores, tokens and files follow its beams."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import beams as oracle
from paper_2510_25412_amd import binding, rag, synth


class StandIn:
    """The calls of a step, carried out on the host as the header defines them."""

    def __init__(self):
        self.rows_moved, self.reorders = [], []

    def beam_select(self, beams, best, logits, scores, best_scores, best_beams, best_tokens, scratch, allowed, stream):
        assert len(beams) <= 65536 and logits.shape[0] == sum(beams) == scores.numel() and scores.is_contiguous()
        assert scratch.numel() >= binding.beam_scratch_bytes(beams, logits.shape[1], best)
        s, b, t = oracle.select(logits.double().numpy(), scores.double().numpy(), beams, best)
        for out, v in ((best_scores, s), (best_beams, b), (best_tokens, t)):
            assert out.is_contiguous() and out.numel() == v.size
            out.view(v.shape).copy_(torch.from_numpy(v))

    def beam_states(self, beams, parents, plan, stream):
        rows = int(np.sum(beams))
        assert len(beams) <= 65536 and parents.dtype == torch.int32 and parents.is_contiguous() and parents.numel() == rows == plan._rows
        self.rows_moved.append(rows)
        first = np.repeat(np.cumsum(beams) - beams, beams)
        width = np.repeat(beams, beams)
        for s in plan[:plan._n]:
            read = [C.string_at(s.src + r * s.row_stride, s.row_bytes) for r in range(rows)]
            for r, p in enumerate(parents.tolist()):
                if 0 <= p < width[r]:
                    C.memmove(s.dst + r * s.row_stride, read[first[r] + p], s.row_bytes)

    def kv_reorder(self, kv, sources, own_last, stream):
        assert own_last
        self.reorders.append((list(kv), [int(s) for s in sources]))


class Session:
    device, stream = torch.device("cpu"), None

    def __init__(self):
        self.shape, self.ctx = synth.Shape(8, 2, 128, 16, synth.BF16), StandIn()


@pytest.mark.parametrize("n_requests,beams,answer", [(5, 3, 4), (300, 2, 3), (70000, 2, 3)])
def test_a_step_moves_the_rows_of_its_batch(n_requests, beams, answer):
    cfg = rag.RagConfig(n_requests=n_requests, answer_tokens=answer, prefill_chunk=1, max_batch=4, beams=beams, vocab=37, seed=3)
    sess = Session()
    d = rag.RagDriver(sess, cfg)
    r = np.random.default_rng(n_requests)
    live = [0, n_requests // 2, n_requests - 1, 1]
    told = {rid: ([[] for _ in range(beams)], np.full(beams, -np.inf)) for rid in live}
    lips = {}
    for rid in live:
        told[rid][1][0] = 0.0
        lip = lips[rid] = rag._Lip()
        lip.rid, lip.to_decode, lip.beams = rid, answer, [rid * beams + i for i in range(beams)]
        for f in lip.beams:
            d.h[f] = f
    logits = d.logits.double().numpy()
    while any(lip.to_decode for lip in lips.values()):
        batch = [lips[rid] for rid in r.permutation([rid for rid in live if lips[rid].to_decode])[:int(r.integers(1, 5))]]
        before = len(sess.ctx.rows_moved)
        d._choose(batch)
        assert sess.ctx.rows_moved[before:] == [len(batch) * beams]
        moved = []
        for i, lip in enumerate(batch):
            said, scores = told[lip.rid]
            s, b, t = oracle.select(logits[i * beams:(i + 1) * beams], scores, [beams], beams)
            told[lip.rid] = [(said[p] if p >= 0 else said[k]) + [tok] for k, (p, tok) in enumerate(zip(b[0], t[0]))], s[0].astype(np.float32).astype(np.float64)
            moved += [int(p) + i * beams if p >= 0 else -1 for p in b[0]]
            lip.to_decode -= 1
        assert sess.ctx.reorders[-1] == ([f for lip in batch for f in lip.beams], moved)
    tokens = d.tokens.view(n_requests, beams, answer)
    for rid in live:
        assert tokens[rid].tolist() == told[rid][0]
        assert d.scores[rid].tolist() == told[rid][1].tolist()
    others = torch.ones(n_requests, dtype=torch.bool)
    others[live] = False
    assert (tokens[others] == -1).all() and (d.scores[others][:, 0] == 0).all()
    d.timer.close()
