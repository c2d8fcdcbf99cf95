"""Layers of a model out of the operators on 8-bit rows and those on a paged cache, beside a context whose projections are in 8 bits: a prompt's
keys and values in both caches.

In the first layer both start from the same embeddings, whose norms have the same codes, and multiply them with the same kernels: keys
and values differ by the rotations' arithmetic (some 1e-6 of a pair), which moves a few to the next bf16 number, eps of the value.  Further on
queries and probabilities are rounded to bf16 here and not there, and a row that is off by delta has some of its values on other 8-bit codes,
2^-4 sqrt(8 delta) of the quantised row, which leads from any delta to 0.03 per quantisation: 0.1 for some independent 0.03 in a row."""
import numpy as np
import pytest
import torch

import workloads as wl
from test_gpu_cached import gpu

pytestmark = pytest.mark.gpu
SHAPES = [wl.ModelShape("layers64", 3, 256, 4, 2, 64, 648, 300, 101, dtype=wl.DTYPE_BF16),
          wl.ModelShape("layers128", 2, 512, 14, 2, 128, 1000, 260, 140, dtype=wl.DTYPE_BF16)]
SCHED = wl.Schedule(exit_layer=2, period_k=3, phase=2, scope=wl.SCOPE_STREAM, n_text=1, n_speech=4)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.name)
@pytest.mark.parametrize("chunks", [[39], [20, 1, 18]])
def test_layers_beside_a_context(shape, chunks):
    from paper_2603_09215_amd import scaled
    from paper_2603_09215_amd.binding import Spark, weights_to_device
    c, n = gpu(), sum(chunks)
    raw = wl.make_weights(shape, seed=5, std=0.06, gain_std=0.1)
    prompt = wl.make_prompt(shape, n + 1, seed=6)
    sp = Spark(shape, SCHED, raw, max_batch=1, max_seq_len=64, kv_page_tokens=16)
    sp.scaled_projections()
    sid = sp.seq_open(0)
    sp.prefill(sid, prompt)

    w = weights_to_device(raw)
    nq, nkv, hd, eps = shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.rms_eps
    W = scaled.ScaledWeights
    layers = [dict(qkv=W(torch.cat([w["wq"][i], w["wk"][i], w["wv"][i]])), o=W(w["wo"][i]), gated=W(w["wg"][i], w["wu"][i]), down=W(w["wd"][i]))
              for i in range(shape.n_layers)]
    cache = c.PagedCache.empty(4, nkv, hd, page_tokens=16, layers=shape.n_layers)
    turn, table = c.Rotation(hd, base=shape.rope_base), torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    done = 0
    for rows in chunks:
        batch = c.CachedRows(torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([done + rows], dtype=torch.int32, device="cuda"), table)
        h = w["embed"][torch.from_numpy(np.asarray(prompt[done:done + rows])).long().cuda()].float()
        y = None
        for i, layer in enumerate(layers):
            qkv = scaled.scaled_matmul(scaled.scaled_norm(h, w["attn_norm"][i].contiguous(), eps, y=y), layer["qkv"])
            q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([nq * hd, nkv * hd, nkv * hd], 1))
            q = c.cached_append(q, k, v, cache, batch, layer=i, rotation=turn)
            o = c.cached_attend(q, cache, batch, layer=i)
            y = scaled.scaled_matmul(scaled.scaled_rows(o.flatten(1)), layer["o"])
            a = scaled.scaled_gated(scaled.scaled_norm(h, w["mlp_norm"][i].contiguous(), eps, y=y), layer["gated"])
            y = scaled.scaled_matmul(a, layer["down"])
        done += rows
    pool, pages = cache.pool.cpu().float(), table[0].tolist()
    for i in range(shape.n_layers):
        got, want = np.zeros((2, n, nkv * hd)), np.zeros((2, n, nkv * hd))
        for t in range(n):
            want[:, t] = sp.get_kv(sid, i, t)
            got[:, t] = pool[pages[t // 16], i, :, :, t % 16].reshape(2, -1).numpy()
        if i == 0:
            pair = np.abs(want).reshape(2, n, nkv, 2, hd // 2)
            pair = np.repeat(pair.sum(3, keepdims=True), 2, axis=3).reshape(want.shape)
            assert (np.abs(got - want) <= torch.finfo(torch.bfloat16).eps * np.maximum(np.abs(want), np.abs(got)) + 2e-6 * pair).all()
        else:
            for which in (0, 1):
                assert np.linalg.norm(got[which] - want[which]) <= 0.1 * np.linalg.norm(want[which]), (i, which)
    sp.close()
