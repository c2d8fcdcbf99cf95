"""What the checks of tests/test_gpu_scaled_passes.py can tell apart, on the CPU: attention and silu off by 1e-5 of themselves pass,
each planted mistake fails."""
import pytest
import torch

import scaled_model as sm
import workloads as wl
from test_gpu_scaled_model import SHAPES

WRONG = ("no rotation", "never in bf16", "queries of zeros", "attention not in 8 bits", "gate and up exchanged", "1 % of down", "the last residual left out")


@pytest.fixture(scope="module", params=list(SHAPES))
def model(request):
    shape = SHAPES[request.param]
    w = sm.weights(shape, 3)
    return shape, w, sm.Model(shape, w)


def test_weights_are_8_bit_rows_as_they_are(model):
    shape, w, plain = model
    for name in sm.PROJECTIONS:
        for m in plain.w[name]:
            assert torch.equal(sm.hold(m), m)
            eights = (torch.nn.functional.pad(m, (0, -m.shape[1] % 8)).view(m.shape[0], -1, 8) != 0).sum(-1)
            assert int(eights.max()) == 1


def short_histories(shape, w, plain, other):
    errors = []
    for s in range(24):
        ids = wl.make_prompt(shape, 2 + s % 6, seed=s)
        many = [True] * len(ids)
        other.gen.manual_seed(s)
        errors.append(float(sm.off(other.forward(ids, many, many, 2)[0], plain.forward(ids, many, many, 2)[0])))
    return errors


def test_steps(model):
    shape, w, plain = model
    assert sm.rows_agree(short_histories(shape, w, plain, sm.Model(shape, w, noise=1e-5)))
    for wrong in WRONG:
        assert not sm.rows_agree(short_histories(shape, w, plain, sm.Model(shape, w, wrong=wrong))), wrong


def test_prompts(model):
    shape, w, plain = model
    T = 300
    ids, many = wl.make_prompt(shape, T, seed=1), [True] * T
    want = plain.forward(ids, many, many, 2)[1]

    def agrees(other):
        got = other.forward(ids, many, many, 2)[1]
        return all(sm.rows_agree(sm.off(got[l][i].reshape(T, -1), want[l][i].reshape(T, -1))) for l in (0, 1, 2) for i in (0, 1))

    assert agrees(sm.Model(shape, w, noise=1e-5))
    for wrong in WRONG[:-1]:   # (no cache entry follows the last residual)
        assert not agrees(sm.Model(shape, w, wrong=wrong)), wrong
