"""The expert-parallel example: operators on the GPU, their traffic and times
into a trace, the trace simulated.  The routed choices, slots, traffic and
gradients against oracle/moe.py, the simulated times against the oracle's
timeline of the same trace."""

import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import moe as plain
from oracle import timeline

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_expert_parallel_layer():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import expert_parallel as ep
    from paper_2505_01616_amd import moe
    from paper_2505_01616_amd.trace import run_trace

    ranks, per, cols, n = 8, 40, 96, 24
    router = moe.Router(experts=16, top_k=4)
    logits, x, dy, dw = ep.inputs(router, ranks * per, cols, n, seed=3)
    layer = ep.run_layer(router, ranks, logits, x, dy, dw)

    def host(t):
        return t.double().cpu().numpy()

    experts, weights = plain.route(router, host(logits))
    np.testing.assert_array_equal(layer.experts.cpu().numpy(), experts)
    np.testing.assert_allclose(host(layer.weights), weights, rtol=100 * 2.0 ** -24)
    want = plain.dispatch(experts, 16, ranks, per, 99.0, False)      # 96 columns and 3 exponents
    for name, got, w in zip(layer.plan._fields, layer.plan, want):
        np.testing.assert_array_equal(got.cpu().numpy(), w, err_msg=name)
    q, e = plain.save(host(x))
    rows = plain.restore(q, e, cols)
    grads = plain.weight_grad(rows, host(dy), want[0], want[1])
    size = plain.weight_grad(np.abs(rows), np.abs(host(dy)), want[0], want[1])
    # half a step of bfloat16, and the 32-bit sums
    assert (np.abs(host(layer.grads) - grads) <= 2.0 ** -8 * np.abs(grads) + (ranks * per + 8) * 2.0 ** -24 * size).all()
    back = plain.route_backward(router, host(logits), experts, host(dw))
    total = np.abs(host(dw)).sum(1, keepdims=True)
    assert (np.abs(host(layer.dlogits) - back) <= 2.0 ** -8 * np.abs(back) + 300 * 2.0 ** -24 * total).all()

    assert (layer.before > 0).all() and (layer.between > 0).all()
    trace = ep.layer_trace(ranks, want[3], layer.before, layer.between)
    ref = timeline.simulate(trace)
    finish, _, sync, stats = run_trace(trace)
    assert stats["complete"] == 1
    np.testing.assert_allclose(finish, ref.finish, rtol=1e-6)
    assert sync.keys() == ref.stream_sync.keys()
    assert max(sync.values()) > layer.before.max() + layer.between.max()


def test_expert_parallel_example_runs():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "expert_parallel.py")], cwd=ROOT, timeout=110,
                       stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.count("the step takes") == 2 and "equally loaded" in r.stdout
