"""Passes of every size of a context on 8-bit projections against the same in 64 bits (tests/scaled_model.py): rows by rows,
to what arithmetic leaves, in the logits of steps and in the cache of prompts.  Passes of more than 64 rows hand sums on in
bf16, of at most 1024 rows go through the layers at once, and prompts have buffers of their own beyond 256 rows."""
import numpy as np
import pytest
import torch

import scaled_model as sm
import workloads as wl
from parity_util import say
from test_gpu_scaled_model import SCHED, SHAPES, sb   # noqa: F401 (sb: the fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def models():
    out = {}
    for name, shape in SHAPES.items():
        w = sm.weights(shape, 3)
        out[name] = shape, w, sm.Model(shape, w)
    return out


def batch(sb, model, n, sched, lens, steps, looked_at):   # noqa: F811
    """n sequences in step; the errors of the steps `looked_at`, and the passes' sizes above the exit"""
    shape, weights, plain = model
    sp = sb.Spark(shape, sched, weights, max_batch=n, max_seq_len=64, kv_page_tokens=16)
    sp.scaled_projections()
    prompts = [wl.make_prompt(shape, lens[i % len(lens)], seed=i) for i in range(n)]
    sids = [sp.seq_open(0) for _ in range(n)]
    for sid, p in zip(sids, prompts):
        sp.prefill(sid, p)
    forced = np.stack([wl.make_forced_stream(shape, steps, sched.n_text, sched.n_speech, 0, seed=50 + i) for i in range(n)], axis=1)
    ids, many, errors, uppers, pending = [list(p) for p in prompts], n > sm.FP32_ROWS, [], [], 0
    for st in range(steps):
        _, dep = sp.step(sids, forced[st])
        assert len(set(dep.tolist())) == 1
        pending += 1
        if int(dep[0]) == shape.n_layers:
            uppers.append(n * pending)
            pending = 0
        if st in looked_at:
            for i, sid in enumerate(sids):
                before = len(prompts[i]) - 1          # rows of the prompt's pass
                flags = [False] * before + [many] * (len(ids[i]) - before)
                want = plain.forward(ids[i], flags, flags, sched.exit_layer, int(dep[0]))[0]
                errors.append(float(sm.off(sp.get_logits(sid)[0], want)))
        for i in range(n):
            ids[i].append(int(forced[st, i]))
    sp.close()
    e = torch.tensor(errors).sort()[0]
    say(f"  {shape.name}: {n} sequences, passes above the exit of {uppers}: errors {float(e[0]):.1e}, median {float(e[len(e) // 2]):.1e}, "
        f"{int((e > 1e-4).sum())} of {len(e)} above 1e-4, worst {float(e[-1]):.1e}")
    return errors, uppers


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("n", [1, 8, 40, 64, 65, 70, 130])
def test_steps_of_a_batch(sb, models, name, n):   # noqa: F811
    steps = 6 if n > 8 else 12
    # (pending rows make the pass above the exit larger: none here where it is to stay within 64)
    sched = SCHED if n <= 8 or n > sm.FP32_ROWS else SCHED.replace(period_k=1, phase=0)
    errors, uppers = batch(sb, models[name], n, sched, (1, 2, 3, 4), steps, range(steps))
    assert uppers and all((u > sm.FP32_ROWS) == (n > sm.FP32_ROWS) for u in uppers)
    assert sm.rows_agree(errors)


@pytest.mark.parametrize("name", list(SHAPES))
def test_a_pass_in_two_pieces(sb, models, name):   # noqa: F811
    """200 sequences complete seven rows each: 1024 and 376, the 147th sequence's in both"""
    sched = wl.Schedule(exit_layer=1, period_k=7, phase=6, scope=wl.SCOPE_STREAM, n_text=0, n_speech=7)
    errors, uppers = batch(sb, models[name], 200, sched, (1, 2), 8, (6, 7))
    assert uppers == [1400]
    assert sm.rows_agree(errors[:200]) and sm.rows_agree(errors[200:])
    assert sm.rows_agree(errors[140:155])      # about the piece's end


def prompt_cache(sb, model, length, many, **kw):   # noqa: F811
    shape, weights, plain = model
    sp = sb.Spark(shape, SCHED, weights, max_batch=1, max_seq_len=1280, kv_page_tokens=64, **kw)
    sp.scaled_projections()
    sid, ids = sp.seq_open(0), wl.make_prompt(shape, length, seed=length)
    sp.prefill(sid, ids)
    T = length - 1
    got = [[np.stack(t) for t in zip(*(sp.get_kv(sid, l, p) for p in range(T)))] for l in range(shape.n_layers)]
    _, dep = sp.step([sid])
    logits = sp.get_logits(sid)[0]
    sp.close()
    flags = many[:T] + [False]                 # the prompt's last token is a step of its own
    lg, want = plain.forward(ids, flags, flags, SCHED.exit_layer, int(dep[0]))
    for l in range(shape.n_layers):
        for i, what in enumerate("KV"):
            g, w = torch.from_numpy(got[l][i]).double(), want[l][i][:T].reshape(T, -1)
            e = sm.off(g, w)
            say(f"  {shape.name} prompt {length} layer {l} {what}: median {float(e.median()):.1e}, {int((e > 1e-4).sum())} of {T} above 1e-4, worst {float(e.max()):.1e}")
            if l == 0:    # straight from the embedding: the same numbers but where the rotation's fp32 lies at a middle
                assert float((g != w).double().mean()) <= 0.01
                assert bool(((g - w).abs() <= 2.0 ** -7 * w.abs() + 1e-5).all())
            else:
                assert sm.rows_agree(e), (l, what)
    assert float(sm.off(logits, lg)) <= 0.1


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("length", [61, 65, 66, 200, 257, 700, 1000, 1100])
def test_the_cache_of_a_prompt(sb, models, name, length):   # noqa: F811
    """one pass up to 1024 rows, two of 640 and 459 at the end: all of more than 64 rows but for the first two lengths"""
    prompt_cache(sb, models[name], length, [length - 1 > sm.FP32_ROWS] * length)


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("length", [297, 600])
def test_the_cache_of_a_prompt_in_the_base_buffers(sb, models, name, length):   # noqa: F811
    """no copy of the caller's weights, so passes of 256 rows: a last one of 40, of 87"""
    rows = length - 1
    prompt_cache(sb, models[name], length, [min(256, rows - r // 256 * 256) > sm.FP32_ROWS for r in range(length)], static_scratch=True)
