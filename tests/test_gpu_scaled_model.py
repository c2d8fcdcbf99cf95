"""A context whose projections run in 8 bits (spark_scaled_projections) against the same model in 64 bits: every
projection's rows and weights held as 8-bit rows by tests/scaled_ref.py, all else as in the bf16 model.  Early exits change
nothing else (the cache a step sees is complete in every layer it runs), so one plain causal forward gives every step.

Tolerances, relative 2-norm of a step's logits.  fp32 arithmetic alone leaves some 1e-7.  But a value that it moves by
1e-6 of itself takes another code in one of 1e5 cases, and what follows multiplies that: a row that is off by delta
has delta / 2^-3 of its values on other codes, 2^-4 of each, so the next quantised row is off by 2^-4 sqrt(8 delta), which
leads from any delta to 2^-5 = 0.03 per quantisation.  So single steps may be off by 0.1 (some independent 0.03 along three
layers), the best one must be off by arithmetic alone, 1e-5, where few rows have gone before it, and all are apart from the
bf16 model.  Passes of more than 64 rows round every product to bf16, so there no step is exact."""
import math

import numpy as np
import pytest
import torch

import scaled_ref as ref
import workloads as wl
from parity_util import say

pytestmark = pytest.mark.gpu

SHAPES = {
    "hd64": wl.ModelShape("scaled64", 3, 256, 4, 2, 64, 648, 300, 101, dtype=wl.DTYPE_BF16),
    "hd128": wl.ModelShape("scaled128", 3, 520, 4, 1, 128, 1000, 260, 140, dtype=wl.DTYPE_BF16),
}
SCHED = wl.Schedule(exit_layer=2, period_k=3, phase=2, scope=wl.SCOPE_STREAM, n_text=1, n_speech=4)


@pytest.fixture(scope="module")
def sb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_09215_amd import binding
    binding.load_library()
    return binding


def tensor(a):
    a = np.asarray(a)
    return torch.from_numpy(a.view(np.int16).copy()).view(torch.bfloat16).double() if a.dtype == np.uint16 else torch.from_numpy(a).double()


class Plain:
    """the model in 64 bits; `held`: its projections on 8-bit rows"""

    def __init__(self, shape, weights, held):
        self.s, self.w, self.held = shape, {k: tensor(v) for k, v in weights.items()}, held
        if held:
            for k in ("wq", "wk", "wv", "wo", "wg", "wu", "wd"):
                self.w[k] = torch.stack([self.hold(m) for m in self.w[k]])

    def hold(self, v):
        return ref.values(*ref.quantise(v))[:, :v.shape[1]] if self.held else v

    def norm(self, x, gain):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.s.rms_eps) * gain

    def logits(self, ids, depth):
        s, w = self.s, self.w
        T, hd, nq, nkv = len(ids), s.head_dim, s.n_q_heads, s.n_kv_heads
        inv = torch.tensor([s.rope_base ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float64).float()
        angle = (torch.arange(T).float()[:, None] * inv[None]).double()
        cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

        def rope(x):
            a, b = x[..., :hd // 2], x[..., hd // 2:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        x = w["embed"][torch.as_tensor(ids).long()]
        mask = torch.triu(torch.ones(T, T, dtype=torch.bool), 1)
        for l in range(depth):
            n = self.hold(self.norm(x, w["attn_norm"][l]))
            q, k = rope((n @ w["wq"][l].T).view(T, nq, hd)), rope((n @ w["wk"][l].T).view(T, nkv, hd))
            k, v = ref.to_type(k, torch.bfloat16), ref.to_type((n @ w["wv"][l].T).view(T, nkv, hd), torch.bfloat16)
            out = torch.empty(T, nq, hd, dtype=torch.float64)
            for h in range(nq):
                sc = q[:, h] @ k[:, h // (nq // nkv)].T / math.sqrt(hd)
                out[:, h] = torch.softmax(sc.masked_fill(mask, -math.inf), -1) @ v[:, h // (nq // nkv)]
            x = x + self.hold(out.view(T, nq * hd)) @ w["wo"][l].T
            n = self.hold(self.norm(x, w["mlp_norm"][l]))
            g, u = n @ w["wg"][l].T, n @ w["wu"][l].T
            x = x + self.hold(g * torch.sigmoid(g) * u) @ w["wd"][l].T
        h = x[-1:]
        if depth == s.n_layers:
            return (self.norm(h, w["final_norm"]) @ w["lm_head"].T)[0]
        u = h + h @ w["lens_a"].T + w["lens_b"]
        return (self.norm(u, w["lens_norm"]) @ w["lens_head"].T)[0]


def off(got, want):
    return float((torch.as_tensor(got).double() - want).norm() / want.norm())


def run(sb, shape, prompts, steps, best_within=None):
    weights = wl.make_weights(shape, seed=3, gain_std=0.1)
    plain, full = Plain(shape, weights, True), Plain(shape, weights, False)
    sp = sb.Spark(shape, SCHED, weights, max_batch=len(prompts), max_seq_len=256, kv_page_tokens=16)
    sp.scaled_projections()
    if best_within:   # attention on the matrix units cuts its weights into two bf16 parts, 1e-5 off
        sp.tune("attn_mfma_min_rows", 1 << 20)
    sids = [sp.seq_open(i) for i in range(len(prompts))]
    for sid, p in zip(sids, prompts):
        sp.prefill(sid, p)
    forced = np.stack([wl.make_forced_stream(shape, steps, SCHED.n_text, SCHED.n_speech, i, seed=50 + i) for i in range(len(prompts))], axis=1)
    ids = [list(p) for p in prompts]
    worst, best, nearest_full, depths = 0.0, 1.0, 1.0, set()
    for st in range(steps):
        _, dep = sp.step(sids, forced[st])
        for i, sid in enumerate(sids):
            lg, head = sp.get_logits(sid)
            assert head == dep[i]
            want = plain.logits(ids[i], int(dep[i]))
            worst, best = max(worst, off(lg, want)), min(best, off(lg, want))
            nearest_full = min(nearest_full, off(lg, full.logits(ids[i], int(dep[i]))))
            ids[i].append(int(forced[st, i]))
            depths.add(int(dep[i]))
    sp.close()
    say(f"  {shape.name}: {len(prompts)} sequences x {steps} steps, {best:.2e} to {worst:.2e} from the 8-bit model, at least {nearest_full:.2e} from the bf16 one")
    assert worst <= 0.1, worst
    assert best_within is None or best <= best_within, best
    assert nearest_full > 0.01          # it is the 8-bit model that ran
    assert depths == {SCHED.exit_layer, shape.n_layers}


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("lens", [(1,), (9,), (33,), (5, 20, 1), (3, 4, 5, 6, 7, 8, 9, 10)])
def test_steps_match_the_8_bit_model(sb, name, lens):
    shape = SHAPES[name]
    run(sb, shape, [wl.make_prompt(shape, n, seed=n) for n in lens], 8, 1e-5)


@pytest.mark.parametrize("length", [40, 150])
def test_attention_on_the_matrix_units_and_a_long_prompt_pass(sb, length):
    shape = SHAPES["hd128"]
    run(sb, shape, [wl.make_prompt(shape, length, seed=9)], 5)


def test_on_and_off_again(sb):
    """the caller's weights give the same bits after 8-bit steps as before them, and caches of both kinds mix"""
    shape = SHAPES["hd64"]
    weights = wl.make_weights(shape, seed=3)
    prompt, forced = wl.make_prompt(shape, 12, seed=1), wl.make_forced_stream(shape, 6, 1, 4, 0, seed=2)
    got = []
    for turn in range(2):
        sp = sb.Spark(shape, SCHED, weights, max_batch=1, max_seq_len=64, kv_page_tokens=16)
        if turn:
            sp.scaled_projections()
            other = sp.seq_open(0)
            sp.prefill(other, prompt)
            sp.step([other], forced[:1])
            sp.seq_close(other)
            sp.scaled_projections(False)
        sid = sp.seq_open(0)
        sp.prefill(sid, prompt)
        for st in range(3):
            sp.step([sid], forced[st:st + 1])
        got.append(sp.get_logits(sid)[0])
        if turn:
            sp.scaled_projections()
            sp.step([sid], forced[3:4])
            assert np.isfinite(sp.get_logits(sid)[0]).all()
            assert sp.seq_state(sid)["len"] == 15
        sp.close()
    assert np.array_equal(got[0], got[1])


def test_many_steps_in_one_call(sb):
    """spark_decode on 8-bit projections: the tokens and depths of steps one by one"""
    shape = SHAPES["hd128"]
    weights = wl.make_weights(shape, seed=3)
    out = []
    for chunk in (1, 12):
        sp = sb.Spark(shape, SCHED, weights, max_batch=3, max_seq_len=64, kv_page_tokens=16)
        sp.scaled_projections()
        sids = [sp.seq_open(i) for i in range(3)]
        for i, sid in enumerate(sids):
            sp.prefill(sid, wl.make_prompt(shape, 4 + i, seed=i))
        parts = [sp.decode(chunk, sids) for _ in range(12 // chunk)]
        out.append((np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])))
        sp.close()
    assert np.array_equal(out[0][0], out[1][0]) and np.array_equal(out[0][1], out[1][1])


def test_static_scratch_and_refusals(sb):
    import ctypes as C
    shape = SHAPES["hd64"]
    weights = wl.make_weights(shape, seed=3)
    sp = sb.Spark(shape, SCHED, weights, max_batch=1, max_seq_len=64, kv_page_tokens=16, static_scratch=True)
    size = C.c_size_t()
    assert sp.lib.spark_scaled_model_bytes(C.byref(sp.cfg), C.byref(size)) == 0
    buf = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    assert sp.lib.spark_scaled_projections(sp.handle, buf.data_ptr(), size.value - 1) == -3
    assert sp.lib.spark_scaled_projections(sp.handle, buf.data_ptr() + 8, size.value) == -3
    sp.scaled_projections()
    sid = sp.seq_open(0)
    prompt = wl.make_prompt(shape, 20, seed=1)
    sp.prefill(sid, prompt)
    sp.step([sid])
    assert off(sp.get_logits(sid)[0], Plain(shape, weights, True).logits(list(prompt), shape.n_layers)) <= 0.1
    sp.close()
    tiny = wl.TINY
    sp = sb.Spark(tiny.shape, tiny.schedule, wl.make_weights(tiny.shape, seed=0), max_batch=1, max_seq_len=64, kv_page_tokens=16)
    with pytest.raises(sb.SparkError):
        sp.scaled_projections()
    assert sp.lib.spark_scaled_projections(sp.handle, buf.data_ptr(), size.value) == -1
    sp.close()
