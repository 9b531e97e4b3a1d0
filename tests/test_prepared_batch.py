"""A batch whose arguments are marshalled once and that is issued again and again: its arrays (CPU), and its steps against pred_batch (GPU)."""
import ctypes as C

import numpy as np
import pytest

from paper_2510_25412_amd import binding


def int32s(address, n):
    return list((C.c_int32 * n).from_address(address))


@pytest.mark.parametrize("kv,n", [([0, 1, 2], [1, 4, 2]), (np.arange(6, dtype=np.int64)[::2], np.array([3, 1, 1], np.int32)), ([1], [7])])
def test_arrays_are_marshalled_and_kept(kv, n):
    ctx = binding.Context(binding.make_config(8, 2, 128, 16, "bf16", 16))
    for _ in range(6):
        ctx.kv_open(None)
    keep, args = prepared = ctx.prepare_batch(kv, n, 4096, 8192, None, 1 << 20)
    assert args[0] == len(kv) and int32s(args[1], len(kv)) == list(kv) and int32s(args[2], len(kv)) == list(n)
    assert args[3:] == (4096, 8192, None, 1 << 20)
    assert any(x is not None and getattr(x, "ctypes", None) is not None and x.ctypes.data == args[1] for x in keep[:2])
    for _ in range(2):
        with pytest.raises(binding.SymError) as e:
            ctx.pred_prepared(prepared)                # a context without a device
        assert e.value.code == binding.SYM_EINVAL
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 8, 2), ("f32", 4, 4)])
def test_steps_of_a_prepared_batch(dtype, hq, hkv):
    torch = pytest.importorskip("torch")
    from paper_2510_25412_amd import driver, synth
    t, D = (torch.bfloat16, 128) if dtype == "bf16" else (torch.float32, 64)
    shape = synth.Shape(hq, hkv, D, 16, dtype)
    got = []
    for way in ("prepared", "each"):
        g = torch.Generator().manual_seed(7)
        randn = lambda *s: torch.randn(s, generator=g).to(t).cuda()  # noqa: E731
        sess = driver.HipSession(shape, 64, None)
        files, lens, new = [sess.ctx.kv_open(None) for _ in range(3)], [40, 17, 100], [1, 3, 1]
        for h, n in zip(files, lens):
            sess.ctx.kv_append(h, n, randn(n, hkv, D), randn(n, hkv, D), sess.stream)
        q, k, v, out = randn(5, hq, D), randn(5, hkv, D), randn(5, hkv, D), torch.empty((5, hq, D), device="cuda")
        batch = sess.ctx.prepare_batch(files, new, q, k, v, out)
        for step in range(3):
            if way == "prepared":
                sess.ctx.pred_prepared(batch, sess.stream)
            else:
                sess.ctx.pred_batch(files, new, q, k, v, out, sess.stream)
            torch.cuda.synchronize()
            got.append((way, out.clone(), [sess.ctx.kv_len(h) for h in files]))
            for x in (q, k, v):                        # the next step's rows, where the batch expects them
                x.copy_(randn(*x.shape))
        sess.close()
    for (_, a, n), (_, b, m) in zip(got[:3], got[3:]):
        assert n == m and torch.isfinite(a).all() and torch.equal(a, b)
