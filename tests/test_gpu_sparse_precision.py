"""How exact the outputs of sparse preds are: full fp32 weights for every number of heads to a group.

Tolerances.  A logit is a sum of D products in fp32, D steps each off by at most 2^-24 of sum |q k|: e = D 2^-24 max sum |q k| scale, at most.  A
weight is off by e and by 2^-22 (exponential, running maximum), its sum and the products' sums by n 2^-24, relative; an output by twice that of the
largest |v|.  Over all outputs the steps are independent of each other: sqrt(D) 2^-25 a logit of size 1, 3.4e-7, and 2^-23 from the
exponential: 4e-7 of their norm, bar 1e-6.  Weights of 16 bits are off by 2^-17 on average, all to one side: 4e-6 to 8e-6."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import longcontext as lc
from paper_2510_25412_amd import binding, driver, synth

BAR = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DIM = {"bf16": 128, "f32": 64}


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("n,D", [(60, 128), (1000, 128), (5000, 64)])
def test_weights_of_sixteen_bits_do_not_pass(n, D):
    # the mistake in the oracle: weights without what the third part of them holds
    r = np.random.default_rng(n)
    q, K, V = r.standard_normal((8, D)), r.standard_normal((n, D)), r.standard_normal((n, D))
    s = q @ K.T / np.sqrt(D)
    w = np.exp(s - s.max(1, keepdims=True))
    cut = (w.astype(np.float32).view(np.uint32) & np.uint32(0xffffff00)).view(np.float32).astype(np.float64)
    full = w.astype(np.float32).astype(np.float64)
    ref = (w / w.sum(1, keepdims=True)) @ V
    error = lambda x: np.linalg.norm((x @ V) / full.sum(1, keepdims=True) - ref) / np.linalg.norm(ref)  # noqa: E731
    assert error(cut) > 2 * BAR and error(full) < BAR / 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 2, 2), ("bf16", 8, 4), ("bf16", 16, 4), ("bf16", 8, 1), ("bf16", 64, 8), ("f32", 2, 2), ("f32", 4, 2), ("f32", 8, 2), ("f32", 16, 2)])
@pytest.mark.parametrize("lens,new,budget", [([1000], 1, 24), ([4000], 1, 200), ([90, 250, 600, 33], 1, 16), ([700, 40], 9, 8)])
def test_outputs_over_all(dtype, hq, hkv, lens, new, budget):
    D, t = DIM[dtype], TYPES[dtype]
    sess = driver.HipSession(synth.Shape(hq, hkv, D, 16, dtype), sum(-(-(n + new) // 16) for n in lens) + 2, None)
    g = torch.Generator().manual_seed(hq + budget)
    randn = lambda *s: torch.randn(s, generator=g).to(t).cuda()  # noqa: E731
    bounds = torch.empty(binding.bounds_bytes(sess.ctx.cfg), dtype=torch.uint8, device="cuda")
    sess.ctx.bounds_attach(bounds)
    files, old = [sess.ctx.kv_open(None) for _ in lens], [(randn(n, hkv, D), randn(n, hkv, D)) for n in lens]
    for h, n, (k, v) in zip(files, lens, old):
        sess.ctx.kv_append(h, n, k, v, sess.stream)
    T = new * len(lens)
    q, k, v, out = randn(T, hq, D), randn(T, hkv, D), randn(T, hkv, D), torch.full((T, hq, D), float("nan"), device="cuda")
    sess.ctx.pred_sparse(files, [new] * len(lens), binding.make_sparse(budget, 1, 2), q, k, v, out, None, sess.stream)
    torch.cuda.synchronize()
    ref, most = [], 0.0
    for i, (n, (ok, ov)) in enumerate(zip(lens, old)):
        at = slice(i * new, (i + 1) * new)
        K, V = f64(torch.cat([ok, k[at]])), f64(torch.cat([ov, v[at]]))
        ref.append(lc.sparse_attention(f64(q[at]), K, V, n, budget, 1, 2)[0])
        e = D * 2.0**-24 * np.sqrt((f64(q[at])**2).sum(-1).max() * (K**2).sum(-1).max()) / np.sqrt(D)
        most = max(most, 2 * (e + 2.0**-22 + 2 * 16 * budget * 2.0**-24) * np.abs(V).max())
    err = f64(out) - np.concatenate(ref)
    print(f"[case] {dtype} {hq}/{hkv} {lens} {new}: {np.linalg.norm(err) / np.linalg.norm(np.concatenate(ref)):.2e} of the norm, {np.abs(err).max() / most:.2e} of the bound", flush=True)
    assert np.isfinite(f64(out)).all() and np.abs(err).max() <= most
    assert np.linalg.norm(err) <= BAR * np.linalg.norm(np.concatenate(ref))
    sess.close()
