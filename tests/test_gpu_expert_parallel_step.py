"""The expert-parallel example's step is a layer's: the experts' products of the
forward and the backward pass between its all-to-alls, rows of the width that
travels.  Products against 64 bits, times against the oracle's timelines."""

import numpy as np
import pytest

from oracle import moe as plain
from oracle import timeline

pytestmark = pytest.mark.gpu


def test_both_passes_of_the_layer():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import expert_parallel as ep
    from paper_2505_01616_amd import moe

    ranks, per, cols, n = 8, 40, 96, 24
    router = moe.Router(experts=16, top_k=4)
    logits, x, dy, dw = ep.inputs(router, ranks * per, cols, n, seed=3)
    w = torch.randn((16, n, cols), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(torch.bfloat16)
    layer = ep.run_layer(router, ranks, logits, x, dy, dw, w)

    def host(t):
        return t.double().cpu().numpy()

    rows = plain.restore(*plain.save(host(x)), cols)
    off, token = layer.plan.offsets.tolist(), layer.plan.token_of_slot.cpu().numpy()
    # sums of up to 96 exact products in 32 bits, rounded to bfloat16
    for e in range(16):
        at = np.arange(off[e], off[e + 1])
        we, xe, de = host(w[e]), rows[token[at]], host(dy)[at]
        for got, want, size in ((layer.y, xe @ we.T, np.abs(xe) @ np.abs(we).T), (layer.dx, de @ we, np.abs(de) @ np.abs(we))):
            assert (np.abs(host(got)[at] - want) <= 2.0 ** -8 * np.abs(want) + 200 * 2.0 ** -24 * size).all(), e
    for times in (layer.before, layer.between, layer.back_before, layer.back_between):
        assert times.shape == (ranks,) and (times > 0).all()

    sent = layer.plan.traffic.cpu().numpy() / 99.0          # 96 columns and 3 exponents
    assert sent.sum() == off[-1]
    forward = ep.layer_trace(ranks, sent * 99.0, layer.before, layer.between, back=sent.T * 48.0)
    backward = ep.layer_trace(ranks, sent * 48.0, layer.back_before, layer.back_between, back=sent.T * 192.0)
    want = sum(max(timeline.simulate(t).stream_sync.values()) for t in (forward, backward))
    total, events = ep.simulated_step(layer, sent, 99.0)
    assert abs(total - want) <= 1e-6 * want and events > 0
    wide, _ = ep.simulated_step(layer, sent, 192.0)
    assert wide > total
