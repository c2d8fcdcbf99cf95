"""What the operators on 8-bit rows write into a given tensor counts as changed, and nothing that a gradient is kept of passes."""
import pytest
import torch

from test_gpu_scaled import BF16, activations, bits, ops, weights   # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu


def test_a_backward_pass_over_a_changed_stream_is_refused(ops):   # noqa: F811
    """h is saved by a product that wants w's gradient, then the norm adds to it in place"""
    h, gain = activations(4, 256, 1).cuda(), torch.ones(256, device="cuda")
    w = torch.ones(256, device="cuda", requires_grad=True)
    loss = (h * w).sum()
    ops.scaled_norm(h, gain, 1e-6, y=torch.ones_like(h))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    h = activations(4, 256, 1).cuda()
    loss, out = (h * w).sum(), torch.empty_like(h)
    ops.scaled_norm(h, gain, 1e-6, y=torch.ones_like(h), h_out=out)   # h stays as it is
    loss.backward()
    assert torch.equal(w.grad, h.sum(0))
    w.grad, loss = None, (h * w).sum()
    ops.scaled_norm(h, gain, 1e-6)                                    # nothing is added to it: h stays too
    loss.backward()
    assert torch.equal(w.grad, h.sum(0))


def test_versions_of_what_is_written(ops):   # noqa: F811
    x, gain = activations(4, 256, 1).cuda(), torch.ones(256, device="cuda")
    rows, act, h_out = ops.ScaledRows.empty(4, 256), ops.ScaledRows.empty(4, 100), torch.empty_like(x)
    w, pair, out = ops.ScaledWeights(weights(100, 256, 1).cuda()), ops.ScaledWeights(weights(100, 256, 2).cuda(), weights(100, 256, 3).cuda()), torch.empty(4, 100, device="cuda")
    for call, written, read in ((lambda: ops.scaled_rows(x, out=rows), (rows.codes, rows.scales), (x,)),
                                (lambda: ops.scaled_norm(x, gain, 1e-6, h_out=h_out, out=rows), (h_out, rows.codes, rows.scales), (x, gain)),
                                (lambda: ops.scaled_norm(x, gain, 1e-6, y=h_out), (x,), (gain, h_out)),
                                (lambda: ops.scaled_norm(x, gain, 1e-6), (), (x, gain)),               # (nothing is added: x stays)
                                (lambda: ops.scaled_norm(x, gain, 1e-6, h_out=x, out=rows), (rows.codes, rows.scales), (x, gain)),
                                (lambda: ops.scaled_matmul(rows, w, out=out), (out,), (rows.codes, rows.scales)),
                                (lambda: ops.scaled_gated(rows, pair, out=act), (act.codes, act.scales), (rows.codes, rows.scales))):
        before = [t._version for t in (*written, *read)]
        call()
        after = [t._version for t in (*written, *read)]
        assert [b - a for a, b in zip(before, after)] == [1] * len(written) + [0] * len(read)


def test_parameters_where_no_graph_is_kept(ops):   # noqa: F811
    """refused under grad mode, taken under no_grad and inference mode, with the results of plain tensors"""
    from paper_2603_09215_amd import SparkError
    x, w = activations(5, 256, 1).cuda(), weights(40, 256, 2).cuda()
    want = ops.scaled_matmul(ops.scaled_rows(x), ops.ScaledWeights(w), dtype=BF16)
    xp, wp = torch.nn.Parameter(x), torch.nn.Parameter(w)
    for call in (lambda: ops.scaled_rows(xp), lambda: ops.ScaledWeights(wp), lambda: ops.ScaledWeights(w, wp),
                 lambda: ops.scaled_norm(x, torch.nn.Parameter(torch.ones(256, device="cuda")), 1e-6, h_out=torch.empty_like(x)),
                 lambda: ops.scaled_matmul(ops.scaled_rows(x), ops.ScaledWeights(w), out=torch.empty(5, 40, device="cuda", requires_grad=True))):
        with pytest.raises(SparkError):
            call()
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            rows = ops.scaled_rows(xp, out=ops.ScaledRows.empty(5, 256))
            assert torch.equal(ops.scaled_matmul(rows, ops.ScaledWeights(wp), out=torch.empty(5, 40, device="cuda", dtype=BF16)), want)
            h = x.clone()
            assert not bool(((bits(ops.scaled_norm(h, torch.ones(256, device="cuda"), 1e-6, y=x).codes) & 127) == 127).any())
            assert torch.equal(h, x + x)
