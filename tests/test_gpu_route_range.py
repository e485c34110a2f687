"""Routing over the whole range of finite logits, and its weights where scores
are small (moe.py on the HIP kernels) against oracle/moe.py in 64 bits.

Bounds.  u = 2^-24.  A sigmoid score is 1/(1 + exp(-x)): the exponential
carries |x| u and 4 u, the sum and the quotient 2 u; with up to 1024 summands
of a renormalisation, products and 22 u for the sum's order a weight stays
below (2 |x| + 40) u relative, as in tests/test_gpu_operators.py.  A score
below float32's smallest normal number, 2^-126, may count as 0: an error of
2^-126 a score.  A renormalised weight s_j / Z then carries (k + 1) 2^-126 / Z.
"""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import SMALL, STEP, U, gpu, host, near, types  # noqa: F401

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -126


def values(torch, kind):
    """Finite values of the type from -110 to 110: all of a 16-bit type, steps
    of 0.005 in float32."""
    if kind == "f32":
        v = np.linspace(-110, 110, 44001, dtype=np.float32).astype(np.float64)
    else:
        bits = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16)
        v = bits.view(types(torch)[kind]).double().numpy()
        v = v[np.isfinite(v) & (np.abs(v) <= 110)]
    return v


def rows_of(torch, kind, experts, seed):
    """All values in rows: some among ordinary logits, the rest with the
    values next to them (all chosen logits small, or large)."""
    v = values(torch, kind)
    rng = np.random.default_rng(seed)
    mixed = torch.from_numpy(rng.normal(0, 2, (len(v) // 4, experts))).to(types(torch)[kind]).double().numpy()
    mixed[np.arange(len(mixed)), rng.integers(0, experts, len(mixed))] = v[::4][:len(mixed)]
    close = np.sort(v)
    close = close[:len(close) // experts * experts].reshape(-1, experts)
    return np.concatenate([mixed, rng.permuted(close, axis=1)])


def small_scores(r, x, e):
    """(sum of the chosen scores, error of a score) of every row: 2^-126 where
    one of them may have counted as 0."""
    s = plain.scores(r.scores, x)
    p = np.where(e >= 0, np.take_along_axis(s, np.maximum(e, 0), 1), 0.0)
    return p.sum(1, keepdims=True), np.where((p < 2 * TINY).any(1, keepdims=True), TINY, 0.0)


def check_route(torch, moe, r, kind, x, bias):
    t = torch.from_numpy(x).to(types(torch)[kind]).cuda()
    b = None if bias is None else torch.from_numpy(bias).float().cuda()
    e, w = moe.route(r, t, b)
    want_e, want_w = plain.route(r, x, bias)
    keep = ~near(r, x, bias)
    if bias is None and r.group_best > 1:      # scores alone decide, and several count as 0
        keep &= (plain.scores(r.scores, x) < 2 * TINY).sum(1) < 2
    np.testing.assert_array_equal(e.cpu().numpy()[keep], want_e[keep])
    z, off = small_scores(r, x, want_e)
    far = np.abs(np.where(np.isfinite(x), x, 0)).max(1, keepdims=True)
    per = (r.top_k + 1) * off / np.maximum(z, 1e-300) if r.renormalise else off
    bound = (2 * far + 40) * U * want_w + r.scale * per + 1e-37 * r.scale * (not r.renormalise)
    assert (np.abs(host(w) - want_w)[keep] <= bound[keep]).all()
    return want_e


SIGMOID = [dict(experts=8, top_k=3), dict(experts=8, top_k=3, renormalise=False, scale=2.5),
           dict(experts=32, top_k=4, groups=4, groups_kept=2, group_best=2)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("cfg", SIGMOID, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_sigmoid_routing_of_every_logit(gpu, cfg, kind, with_bias):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(scores="sigmoid", **cfg)
    bias = None
    if with_bias:
        bias = (np.random.default_rng(5).permutation(r.experts) * 0.0137 - 0.2).astype(np.float32).astype(np.float64)
    check_route(torch, moe, r, kind, rows_of(torch, kind, r.experts, 3), bias)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cfg", SIGMOID[:2], ids=lambda c: "-".join(str(v) for v in c.values()))
def test_sigmoid_gradient_of_every_logit(gpu, cfg, kind):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(scores="sigmoid", **cfg)
    x = rows_of(torch, kind, r.experts, 4)
    e, _ = plain.route(r, x)
    dw = np.random.default_rng(8).normal(0, 1, (len(x), r.top_k)).astype(np.float32)
    got = moe.route_backward(r, torch.from_numpy(x).to(types(torch)[kind]).cuda(), torch.from_numpy(e).int().cuda(),
                             torch.from_numpy(dw).cuda())
    want = plain.route_backward(r, x, e, dw)
    total = np.abs(dw).sum(1, keepdims=True) * r.scale
    far = np.abs(x).max(1, keepdims=True)
    z, off = small_scores(r, x, e)
    # 1 - p may count as 0 as well
    per = 2 * (r.top_k + 1) * off / np.maximum(z, 1e-300) + TINY if r.renormalise else 2 * TINY
    bound = (4 * far + 100) * U * total + total * per + STEP[kind] * np.abs(want) + SMALL[kind]
    assert (np.abs(host(got) - want) <= bound).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_softmax_routing_of_every_logit(gpu, kind, with_bias, renorm):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(8, 3, "softmax", renorm)
    bias = None
    if with_bias:
        bias = (np.random.default_rng(5).permutation(8) * 0.0137 - 0.2).astype(np.float32).astype(np.float64)
    x = rows_of(torch, kind, 8, 3)
    t = torch.from_numpy(x).to(types(torch)[kind]).cuda()
    e, w = moe.route(r, t, None if bias is None else torch.from_numpy(bias).float().cuda())
    want_e, want_w = plain.route(r, x, bias)
    keep = ~near(r, x, bias)
    np.testing.assert_array_equal(e.cpu().numpy()[keep], want_e[keep])
    far = x.max(1, keepdims=True) - x.min(1, keepdims=True)
    bound = (2 * far + 40) * U * want_w + 2 * TINY
    assert (np.abs(host(w) - want_w)[keep] <= bound[keep]).all()


@pytest.mark.parametrize("scores,level", [("sigmoid", -75.0), ("sigmoid", -86.0), ("softmax", -75.0)])
@pytest.mark.parametrize("scale", [16.0, 1e8, 3e38])
def test_weights_of_small_scores_with_large_factors(gpu, scores, level, scale):  # noqa: F811
    """scale / (sum of the chosen scores) is beyond float32, the weights are
    not."""
    torch, moe = gpu
    r = moe.Router(16, 4, scores, scale=scale)
    x = np.random.default_rng(2).uniform(level - 1, level + 0.5, (64, 16)).astype(np.float32).astype(np.float64)
    x[1] = level
    x[2, 1:] = -np.inf
    check_route(torch, moe, r, "f32", x, None)
