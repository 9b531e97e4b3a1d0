"""Sparse preds in workspaces that hold few parts of a token's list: the same pages, and outputs as exact as with many parts.

Tolerance.  A logit is a sum of D products in fp32, each step off by half a step of the running sum: sqrt(D) 2^-25 of its size, rms, 3.4e-7 for
logits of about 1; a weight takes that and 2^-23 from the exponential, and the outputs, relative to their norm, what the weights take: 4e-7.  The bar is
1e-6 of the norm over all outputs; adding up more or fewer parts changes a sum of a few dozen terms by 2^-24 of it each."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import longcontext as lc
from paper_2510_25412_amd import binding

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DIM = {"bf16": 128, "f32": 64}


@pytest.mark.parametrize("dtype,hq,hkv,sizes", [("bf16", 4, 2, (256, 64, 44, 40)), ("bf16", 8, 1, (512, 164, 150)), ("f32", 4, 1, (256, 64, 52, 44, 40)), ("bf16", 2, 2, (128, 40, 28))])
def test_fewer_parts(dtype, hq, hkv, sizes):
    D, t, pages, budget = DIM[dtype], TYPES[dtype], 700, 300
    g = torch.Generator().manual_seed(hq)
    randn = lambda *s: torch.randn(s, generator=g).to(t).cuda()  # noqa: E731
    n = 16 * pages - 5
    k, v, q, kn, vn = randn(1, n, hkv, D), randn(1, n, hkv, D), randn(1, hq, D), randn(1, hkv, D), randn(1, hkv, D)
    K, V = (torch.cat([a[0], b]).double().cpu().numpy() for a, b in ((k, kn), (v, vn)))
    ref, chosen = lc.sparse_attention(q.double().cpu().numpy(), K, V, n, budget, 1, 1)
    st = torch.cuda.current_stream().cuda_stream
    outs = []
    for kb in sizes:
        cfg = binding.make_config(hq, hkv, D, 16, dtype, pages + 8, device=0, decode_waves=1)
        pool = torch.zeros((pages + 8) * binding.page_bytes(cfg), dtype=torch.uint8, device="cuda")
        ws = torch.full(((kb << 10) + 4096,), 0x5a, dtype=torch.uint8, device="cuda")            # what lies behind stays
        cfg.pool, cfg.workspace, cfg.workspace_bytes = pool.data_ptr(), ws.data_ptr(), kb << 10
        ctx = binding.Context(cfg)
        ctx.bounds_attach(torch.empty(binding.bounds_bytes(cfg), dtype=torch.uint8, device="cuda"))
        f = ctx.kv_open(None)
        ctx.kv_append_rope([f], [n], None, k, v, None, st)
        out, pick = torch.full((1, hq, D), float("nan"), device="cuda"), torch.empty((1, hkv, budget), dtype=torch.int32, device="cuda")
        ctx.pred_sparse([f], [1], binding.make_sparse(budget, 1, 1), q, kn, vn, out, pick, st)
        torch.cuda.synchronize()
        assert pick[0].tolist() == chosen[0] and (ws[kb << 10:] == 0x5a).all()
        err = np.linalg.norm(out.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        print(f"[case] {dtype} {hq}/{hkv} {kb} KB: {err:.2e}", flush=True)
        assert err <= 1e-6
        outs.append(out.clone())
        ctx.close()
    assert not all(torch.equal(o, outs[0]) for o in outs[1:])                                    # the parts are not the same ones
