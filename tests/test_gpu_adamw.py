"""The AdamW step (moe.AdamW) against oracle/experts.py in 64 bits.

Bounds, u = 2^-24.  m and v are two products and a sum of values of one sign
(v) or two (m): 4 u of |b1 m| + |c1 g|; the factors' own rounding is in it.
d = m / (r root + eps): r off by half of v's 4 u and its own u (2 u with moments
in 8 bits, whose root may be a unit in the last place off, as the reciprocal),
the sum, product and quotient 4 u: d off by Em / (r root + eps) + 8 u |d|.  p: 3 u of
|p| + |rate d| and rate times d's error.  16-bit results add half a step.
Moments in 8 bits are half a step of a 4-bit number (2^-4 of themselves, or
2^-10 units below the smallest normal one) from the 64-bit value, with what
was said before, and their scales 4 u of themselves plus the same; a root that
would round to zero is one smallest step, 2^-9 units.
"""

import numpy as np
import pytest

from oracle import experts as plain

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
HYPER = dict(lr=2e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_01616_amd import moe
    return torch, moe


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def host(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def state_of(torch, moe, opt, i):
    """(m, v, in 8 bits: m's and the root's unit a code stands for) in 64 bits."""
    s = opt.moments[i]
    n = opt.params[i].numel()
    if opt.bits == 32:
        return host(s.m), host(s.v)
    unit = [np.repeat(host(x), moe.SCALED)[:n] for x in s[2:]]
    value = [plain.FLOAT8[q.view(torch.uint8).cpu().numpy()][:n] for q in s[:2]]
    return value[0] * unit[0], (value[1] * unit[1]) ** 2


def check_step(torch, moe, opt, grads, scale, kind):
    """One step, every tensor against the oracle from the state before it."""
    before = [(host(c if c is not None else p), *state_of(torch, moe, opt, i)) for i, (p, c) in enumerate(zip(opt.params, opt.masters))]
    opt.step(grads, grad_scale=scale)
    t = opt.steps
    b1, b2 = opt.betas
    for i, (p0, m0, v0) in enumerate(before):
        n = len(p0)
        if n == 0:
            continue
        g = host(grads[i])
        p, m, v = plain.adamw(p0, g, m0, v0, t, opt.lr, b1, b2, opt.eps, opt.weight_decay, scale)
        gs = g * scale
        em = 4 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * gs)) + 2.0 ** -149
        ev = 4 * U * v + 2.0 ** -148
        root = (1 - b2 ** t) ** -0.5
        r = np.sqrt(v)
        er = np.minimum(ev / np.maximum(r, 1e-300), np.sqrt(ev)) + (U if opt.bits == 32 else 2 * U) * r
        denominator = r * root + opt.eps
        d = m / denominator
        ed = em / denominator + np.abs(d) * (er * root / denominator + 8 * U)
        rate = opt.lr / (1 - b1 ** t)
        ep = 3 * U * (np.abs(p0) + np.abs(rate * d)) + rate * ed
        got = host(opt.params[i])
        assert np.all(np.abs(got - p) <= ep * 1.01 + HALF[kind] * np.abs(p) + LEAST[kind]), (i, n)
        if opt.masters[i] is not None:
            assert np.all(np.abs(host(opt.masters[i]) - p) <= ep * 1.01)
            assert np.array_equal(host(opt.masters[i].to(opt.params[i].dtype)), got)
        if opt.bits == 32:
            gm, gv = state_of(torch, moe, opt, i)
            assert np.all(np.abs(gm - m) <= em) and np.all(np.abs(gv - v) <= ev)
            continue
        for j, (x, e) in enumerate(((m, em), (r, er))):
            want, scales = plain.narrow(x)
            error = np.concatenate([e, np.zeros(-n % 256)]).reshape(-1, 256)
            got_scales = host(opt.moments[i][2 + j])
            assert np.all(np.abs(got_scales - scales) <= 4 * U * scales + error.max(1) / 448), (i, n, j)
            code = opt.moments[i][j].view(torch.uint8).cpu().numpy()
            got = plain.FLOAT8[code]
            units = error / np.where(scales > 0, scales, np.inf)[:, None] + np.abs(want.reshape(-1, 256)) * 8 * U
            half = np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10)
            if j:
                half = np.where((want > 0) & (want < 2.0 ** -10), 2.0 ** -9, half)
                assert np.all((code[:n] > 0) | (x == 0) | (np.repeat(scales, 256)[:n] == 0))
            assert np.all(np.abs(got - want) <= half + units.reshape(-1)), (i, n, j)
            assert not code[n:].any()


SIZES = [1, 2, 7, 8, 255, 256, 257, 2047, 2049, 4096, 5000, 70001, 0]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind,grad,masters", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False),
                                               ("bf16", "f32", True), ("f16", "f16", True), ("f16", "f32", False)])
def test_steps(gpu, bits, kind, grad, masters):
    """From zeros, several steps, sizes with every remainder, gradients that
    are zero here and there and differ widely."""
    torch, moe = gpu
    rng = np.random.default_rng(1)
    params = [torch.from_numpy(rng.normal(0, 0.1, n)).to(types(torch)[kind]).cuda() for n in SIZES]
    opt = moe.AdamW(params, bits=bits, masters=masters, **HYPER)
    for _ in range(4):
        grads = [torch.from_numpy(rng.normal(0, 1, n) * np.exp(rng.normal(0, 2, n)) * (rng.random(n) > 0.1)).to(types(torch)[grad]).cuda() for n in SIZES]
        check_step(torch, moe, opt, grads, 2.0 ** -6, kind)
    assert opt.steps == 4


def test_many_tensors_at_any_alignment(gpu):
    """More tensors than a launch takes, parts of one array at odd places."""
    torch, moe = gpu
    rng = np.random.default_rng(2)
    sizes = rng.integers(1, 400, 130)
    flat, at, params = torch.from_numpy(rng.normal(0, 1, 130 * 401)).bfloat16().cuda(), 0, []
    before = flat.clone()
    outside = torch.ones_like(flat, dtype=torch.bool)
    for n in sizes:
        params.append(flat[at:at + n])
        outside[at:at + n] = False
        at += int(n) + 1
    g = torch.from_numpy(rng.normal(0, 1, len(flat) + 1)).float().cuda()
    grads = [g[1 + i * 401:1 + i * 401 + n] for i, n in enumerate(sizes)]
    opt = moe.AdamW(params, **HYPER)
    check_step(torch, moe, opt, grads, 1.0, "bf16")
    assert torch.equal(flat[outside], before[outside])


def test_nothing_and_none(gpu):
    torch, moe = gpu
    moe.AdamW([]).step([])
    p = [torch.ones(5, device="cuda", requires_grad=True), torch.ones(3, device="cuda", requires_grad=True)]
    opt = moe.AdamW(p, lr=0.1, weight_decay=0.0)
    (p[1] * 2).sum().backward()
    opt.step()
    assert torch.equal(p[0], torch.ones_like(p[0])) and torch.allclose(p[1], torch.full_like(p[1], 0.9))
    assert not opt.moments[0].m.any() and opt.moments[1].m.any()
    # a graph that has saved a parameter sees that it has changed
    q = torch.ones(3, device="cuda", requires_grad=True)
    y = (q * q).sum()
    moe.AdamW([q]).step([torch.ones_like(q)])
    with pytest.raises(RuntimeError, match="modified"):
        y.backward()


def test_refusals(gpu):
    torch, moe = gpu
    p = torch.ones(8, device="cuda")
    opt = moe.AdamW([p, p])
    with pytest.raises(ValueError, match="twice"):
        opt.step([p.clone(), p.clone()])
    opt = moe.AdamW([p])
    for bad in ([torch.ones(9, device="cuda")], [torch.ones(2, 4, device="cuda")], [torch.ones(8)], [torch.ones(8, device="cuda").double()],
                [torch.ones(16, device="cuda")[::2]], []):
        with pytest.raises(ValueError):
            opt.step(bad)
    q = torch.ones(8, device="cuda", requires_grad=True)
    opt = moe.AdamW([q])
    q.data = torch.ones(4, device="cuda")
    with pytest.raises(ValueError, match="params"):
        opt.step([torch.ones(8, device="cuda")])
    assert opt.steps == 0 and torch.equal(p, torch.ones_like(p))
    with pytest.raises(ValueError):
        moe.AdamW([p], masters=[p.clone()])
    with pytest.raises(ValueError):
        moe.AdamW([p], moments=[moe.Moments(torch.zeros(9, device="cuda"), torch.zeros(8, device="cuda"))])
    with pytest.raises(ValueError):
        moe.AdamW([p], bits=8, moments=[moe.Moments(torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda"))])


@pytest.mark.parametrize("bits", [32, 8])
def test_undefined_gradients_stay_with_their_block(gpu, bits):
    torch, moe = gpu
    p = torch.zeros(1000, device="cuda")
    opt = moe.AdamW([p], bits=bits, **HYPER)
    g = torch.ones(1000, device="cuda")
    g[300], g[999] = float("nan"), float("inf")
    opt.step([g])
    opt.step([torch.ones_like(g)])
    bad = ~torch.isfinite(p)
    hit = torch.zeros_like(bad)
    if bits == 32:
        hit[300] = hit[999] = True
    else:
        hit[256:512] = hit[768:] = True
    # an infinite gradient's step is inf / inf in both
    assert torch.equal(bad, hit)


def test_moments_fall(gpu):
    """In 8 bits a block's moments fall with its largest, though a step of
    0.1% is less than half of theirs: 200 steps without a gradient."""
    torch, moe = gpu
    p = torch.zeros(256, device="cuda")
    opt = moe.AdamW([p], bits=8, betas=(0.9, 0.999))
    opt.step([torch.linspace(0.5, 1.0, 256, device="cuda")])
    v = state_of(torch, moe, opt, 0)[1]
    for _ in range(200):
        opt.step([torch.zeros(256, device="cuda")])
    ratio = state_of(torch, moe, opt, 0)[1] / v
    # the largest exactly but for 200 roundings of the scale and the root
    assert abs(ratio[-1] / 0.999 ** 200 - 1) < 1e-3 and np.all(np.abs(ratio / 0.999 ** 200 - 1) < 2 * 2.0 ** -3)


@pytest.mark.parametrize("bits", [32, 8])
def test_streams_and_graphs(gpu, bits):
    """A captured step counts on with every replay where it is asked to."""
    torch, moe = gpu
    rng = np.random.default_rng(3)
    make = lambda: [torch.from_numpy(rng.normal(0, 1, n)).float().cuda() for n in (300, 5000)]      # noqa: E731
    start, grads = make(), make()
    captured, eager = ([p.clone() for p in start] for _ in range(2))
    one = moe.AdamW(captured, bits=bits, counted=True, **HYPER)
    two = moe.AdamW(eager, bits=bits, **HYPER)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one.step(grads)
    torch.cuda.current_stream().wait_stream(side)
    two.step(grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(grads)
    for turn in range(4):
        for g, new in zip(grads, make()):
            g.copy_(new)
        graph.replay()
        two.step(grads)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            # the factors of a step are worked out on the GPU or on the host:
            # a unit in the last place of each
            assert torch.allclose(a, b, rtol=1e-6, atol=1e-8), turn
    assert int(one.counter[0]) == 5 and two.steps == 5
