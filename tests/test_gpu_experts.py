"""Products of experts with their gradients (moe.gated, moe.product) against
oracle/experts.py in 64 bits.

Bounds.  u = 2^-24, s the half step of the inputs' type relative to the value
(torch.finfo(t).eps / 2: bf16 2^-8, f16 2^-11).  Products of two 16-bit values
are exact in 32 bits; a sum of K of them is off by at most
2 (K + 8) u of the sum of their magnitudes T (a step of the sum may cut instead
of rounding: 2 u).  With E = 2 (K + 8) u T for g and u:
  h = act(g) u:  |act'| <= 1.13, so 1.13 Eg |u| + |act(g)| Eu, plus what act is
    computed with: its exponential's argument rounds (|g| u twice) and the
    function is off by 2^-16 of itself at most (gelu's polynomial 8e-6, the
    reciprocal and exponential a few u): 2^-16 + 4 |g| u of |g u|;
  dg = dh u act'(g), du = dh act(g):  likewise with |act''| <= 1 and act' off by
    (2^-16 + 4 |g| u) (1 + |g|), plus s of themselves for their rounding (and the
    type's smallest half step);
  dx, dW: the sums of those errors with the other factor's magnitudes, plus
    2 (terms + 8) u of the sum of magnitudes.
Every result adds s of itself and the type's smallest half step.
"""

import numpy as np
import pytest

from oracle import experts as plain

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_01616_amd import moe
    return torch, moe


def types(torch):
    return {"bf16": torch.bfloat16, "f16": torch.float16}


def wide(torch, x, dtype, pad=0, skew=0):
    """x on the GPU, its rows inside wider ones that hold NaN, from column
    `skew` on."""
    t = torch.full((x.shape[0], x.shape[1] + pad + skew), float("nan"), dtype=dtype, device="cuda")
    v = t[:, skew:skew + x.shape[1]]
    v.copy_(torch.from_numpy(x))
    return v


def host(t):
    return t.detach().double().cpu().numpy()


def off(terms, top):
    return 2 * (terms + 8) * U * top


def near(got, want, tolerance, what):
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= tolerance)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0].tolist()}: "
                           f"{got[bad][0]} for {want[bad][0]}, {np.broadcast_to(tolerance, bad.shape)[bad][0]} allowed")


def plan(rng, tokens, experts, top_k, drop, by):
    """(offsets, row_of_slot, slots_of_row) of uneven random choices."""
    weight = 1 / (rng.permutation(experts) + 1.0) ** 1.2
    choice = np.stack([rng.choice(experts, top_k, replace=False, p=weight / weight.sum()) for _ in range(tokens)]) if tokens else np.zeros((0, top_k), int)
    choice[rng.random(choice.shape) < drop] = experts
    order = np.argsort(choice.reshape(-1), kind="stable")
    key = choice.reshape(-1)[order]
    offsets = np.searchsorted(key, np.arange(experts + 1)).astype(np.int32)
    if by == "slot":
        return offsets, None, None
    row = np.where(key < experts, order // top_k, -1).astype(np.int32)
    slots = np.full(tokens * top_k, -1, dtype=np.int32)
    slots[order] = np.where(key < experts, np.arange(len(key)), -1)
    return offsets, row, slots.reshape(tokens, top_k)


def check(gpu, kind, act, x, weights, lists, dy=None, pad=0, skew=0, scale=1.0, grads=(True, True)):
    """Runs gated (act) or product (None) and compares everything with the
    oracle; x, weights, dy float64.  Returns the results."""
    torch, moe = gpu
    t = types(torch)[kind]

    def cut(a):
        return torch.from_numpy(a).to(t).double().numpy()

    x, weights = cut(x), [cut(w) for w in weights]
    gx = wide(torch, x, t, pad, skew)
    gw = [torch.from_numpy(w).to(t).cuda() for w in weights]
    offsets, row_of_slot, slots_of_row = (None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in lists)
    if dy is not None:
        gx.requires_grad_(grads[0])
        for w in gw:
            w.requires_grad_(grads[1])
    more = dict(offsets=offsets, row_of_slot=row_of_slot, slots_of_row=slots_of_row)
    got = moe.gated(gx, *gw, activation=act, **more) if act else moe.product(gx, *gw, **more)
    z, top, want = plain.multiply(x, weights, lists[0], lists[1], act)
    K, s, least = x.shape[1], HALF[kind], LEAST[kind]
    e = [off(K, v) for v in top]
    if act:
        a, slope = plain.activation(act, z[0])
        fa = 2.0 ** -16 + 4 * np.abs(z[0]) * U
        err = 1.01 * (1.13 * e[0] * np.abs(z[1]) + np.abs(a) * e[1] + fa * np.abs(z[0] * z[1]))
    else:
        err = e[0]
    near(host(got), want, err * (1 + s) + s * np.abs(want) + least, "result")
    if dy is None:
        return got
    dy = cut(dy)
    gdy = wide(torch, dy, t, pad, skew)
    wanted = ([gx] if grads[0] else []) + (gw if grads[1] else [])
    back = torch.autograd.grad(got, wanted, gdy)
    backs = [back]
    if act:      # g and u computed again, by another kernel where rows are few
        again = moe.gated(gx, *gw, activation=act, recompute=True, **more)
        assert torch.equal(again, got)
        backs.append(torch.autograd.grad(again, wanted, gdy))
    live = plain.used(lists[0], len(weights[0]), lists[1], len(dy), len(x))[:, None]
    dy = np.where(live, dy, 0)
    if act:
        d = [dy * z[1] * slope, dy * a]
        es = e[0] + (2.0 ** -16 + 4 * np.abs(z[0]) * U) * (1 + np.abs(z[0]))
        ed = [1.01 * np.abs(dy) * (e[1] * np.abs(slope) + np.abs(z[1]) * es), 1.01 * np.abs(dy) * (1.13 * e[0] + fa * np.abs(z[0]))]
        ed = [v * (1 + s) + s * np.abs(w) + least * live for v, w in zip(ed, d)]
    else:
        d, ed = [dy], [np.zeros_like(dy)]
    absx, absw = np.abs(x), [np.abs(w) for w in weights]
    dx, dw = plain.gradients(x, weights, d, *lists)
    tx, tw = plain.gradients(absx, absw, [np.abs(v) for v in d], *lists)
    ex, ew = plain.gradients(absx, absw, ed, *lists)
    each = 1 if lists[2] is None else lists[2].shape[1]
    for back in backs:
        if grads[0]:
            bound = ex + off(len(weights) * weights[0].shape[1] + each, tx + ex)
            near(host(back[0]), dx, bound * (1 + s) + s * np.abs(dx) + least, "dx")
        if grads[1]:
            for g, w, t_, e_ in zip(back[-len(weights):], dw, tw, ew):
                near(host(g), w, (e_ + off(len(dy), t_ + e_)) * (1 + s) + s * np.abs(w) + least, "dW")
    return got, back


SHAPES = [  # experts, tokens, top_k, cols, n, dropped, by
    (1, 1, 1, 1, 1, 0.0, "dense"),
    (1, 5, 1, 8, 8, 0.0, "dense"),
    (1, 300, 1, 64, 40, 0.0, "dense"),
    (1, 700, 1, 72, 264, 0.0, "dense"),
    (1, 129, 1, 1000, 33, 0.0, "dense"),
    (2, 1, 1, 128, 128, 0.0, "token"),
    (4, 3, 2, 136, 65, 0.0, "token"),
    (8, 1, 3, 256, 192, 0.0, "slot"),
    (8, 130, 2, 96, 136, 0.1, "token"),
    (3, 700, 2, 192, 320, 0.05, "token"),
    (3, 900, 1, 320, 130, 0.0, "slot"),
    (64, 100, 4, 48, 24, 0.2, "slot"),
    (130, 260, 3, 33, 17, 0.5, "token"),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_products(gpu, kind, act, shape):
    experts, tokens, top_k, cols, n, drop, by = shape
    rng = np.random.default_rng(hash(shape[:5]) % 1000)
    lists = (None, None, None) if by == "dense" else plan(rng, tokens, experts, top_k, drop, by)
    slots = tokens if by == "dense" else tokens * top_k
    x = rng.normal(0, 1, (slots if by == "slot" else tokens, cols)) * np.exp(rng.normal(0, 0.5, cols))
    weights = [rng.normal(0, cols ** -0.5, (experts, n, cols)) for _ in range(2 if act else 1)]
    dy = rng.normal(0, 1, (slots, n))
    for pad, skew in ((0, 0), (8, 0), (3, 0), (7, 1)):
        check(gpu, kind, act, x, weights, lists, dy, pad, skew)


@pytest.mark.parametrize("act", [None, "silu"])
def test_one_gradient(gpu, act):
    """Only the rows' or only the weights' gradient."""
    rng = np.random.default_rng(3)
    lists = plan(rng, 40, 4, 2, 0.1, "token")
    x, dy = rng.normal(0, 1, (40, 64)), rng.normal(0, 1, (80, 48))
    weights = [rng.normal(0, 0.1, (4, 48, 64)) for _ in range(2 if act else 1)]
    check(gpu, "bf16", act, x, weights, lists, dy, grads=(True, False))
    check(gpu, "bf16", act, x, weights, (lists[0], lists[1], None), dy, grads=(False, True))
    torch, moe = gpu
    with pytest.raises(ValueError, match="slots_of_row"):
        check(gpu, "bf16", act, x, weights, (lists[0], lists[1], None), dy)


@pytest.mark.parametrize("act", [None, "gelu"])
@pytest.mark.parametrize("cols", [64, 61])
def test_slots_left_out(gpu, act, cols):
    """Slots before the first expert's and behind the last one's, rows out of
    range, experts without slots; what their gradients and unused rows hold
    reaches nothing."""
    torch, moe = gpu
    rng = np.random.default_rng(4)
    slots, experts, n = 70, 5, 40
    offsets = np.array([3, 3, 20, 20, 41, 66], dtype=np.int32)
    row = rng.integers(0, 30, slots).astype(np.int32)
    row[[0, 5, 19, 50, 69]] = [-1, 30, -7, 2 ** 31 - 1, 4]
    lists = [[] for _ in range(31)]
    for s in range(3, 66):
        if 0 <= row[s] < 30:
            lists[row[s]].append(s)
    each = max(map(len, lists))
    slots_of_row = np.array([v + [-1] * (each - len(v)) for v in lists], dtype=np.int32)
    x = rng.normal(0, 1, (31, cols))
    x[30] = np.nan      # a row that no slot has
    row[5] = 31
    dy = rng.normal(0, 1, (slots, n))
    dy[[0, 1, 5, 19, 50, 66, 69]] = np.nan
    dy[2] = np.inf
    weights = [rng.normal(0, 0.1, (experts, n, cols)) for _ in range(2 if act else 1)]
    y, back = check(gpu, "bf16", act, x, weights, (offsets, row, slots_of_row), dy)
    for s in (0, 1, 2, 5, 19, 50, 66, 69):
        assert not host(y[s]).any()
    assert not host(back[0][30]).any() and not host(back[1][0]).any() and not host(back[1][2]).any()


def test_infinities_stay_where_they_are(gpu):
    """An infinity or a NaN in a row, a weight or a gradient reaches what
    depends on it and nothing else."""
    torch, moe = gpu
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.normal(0, 1, (40, 72))).bfloat16().cuda()
    w = torch.from_numpy(rng.normal(0, 0.1, (2, 24, 72))).bfloat16().cuda()
    offsets = torch.tensor([0, 17, 40], dtype=torch.int32, device="cuda")
    x[20, 3], w[0, 5, 71] = float("inf"), float("nan")
    y = moe.product(x, w, offsets)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[20] = True
    want[:17, 5] = True
    assert torch.equal(bad, want)
    dy = torch.ones_like(y)
    dy[3, 7] = float("inf")
    x.requires_grad_(), w.requires_grad_()
    dx, dw = torch.autograd.grad(moe.product(x, w, offsets), [x, w], dy)
    bad = ~torch.isfinite(dx)
    want = torch.zeros_like(bad)
    want[3] = True
    want[:17, 71] = True
    assert torch.equal(bad, want)
    bad = ~torch.isfinite(dw)
    want = torch.zeros_like(bad)
    want[0, 7] = True
    want[1, :, 3] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_large_gates(gpu, act):
    """Gates far from zero: no overflow on the way, act(g) is g or 0."""
    torch, moe = gpu
    x = torch.tensor([[-3e4], [-200.0], [-30.0], [-5.0], [0.0], [5.0], [30.0], [200.0], [3e4]], dtype=torch.bfloat16, device="cuda")
    one = torch.ones((1, 1), dtype=torch.bfloat16, device="cuda")
    x.requires_grad_()
    y = moe.gated(x, one, one, activation=act)
    dx, = torch.autograd.grad(y, x, torch.ones_like(y))
    g = host(x)[:, 0]
    with np.errstate(over="ignore"):
        a, slope = plain.activation(act, g)
    assert np.allclose(host(y)[:, 0], a * g, rtol=2 ** -8 + 1e-5, atol=1e-30)
    # y = act(g) g; dg and du are rounded before they are added
    want = a + g * slope
    assert np.all(np.abs(host(dx)[:, 0] - want) <= (np.abs(a) + np.abs(g * slope)) * (2 ** -8 + 1e-4) + np.abs(want) * 2 ** -8 + 1e-30)


@pytest.mark.parametrize("act", [None, "silu"])
def test_differences(gpu, act):
    """Gradients against differences of the 64-bit formula."""
    torch, moe = gpu
    rng = np.random.default_rng(6)
    lists = plan(rng, 9, 3, 2, 0.1, "token")
    x = torch.from_numpy(rng.normal(0, 1, (9, 16))).half()
    ws = [torch.from_numpy(rng.normal(0, 0.3, (3, 8, 16))).half() for _ in range(2 if act else 1)]
    dy = rng.normal(0, 1, (18, 8))
    dy = torch.from_numpy(dy).half()
    leaves = [t.cuda().requires_grad_() for t in (x, *ws)]
    at = [torch.from_numpy(a).cuda() for a in lists]
    y = moe.gated(*leaves, *at, activation=act) if act else moe.product(*leaves, *at)
    grads = torch.autograd.grad(y, leaves, dy.cuda())
    values = [t.double().numpy() for t in (x, *ws)]

    def loss(v):
        return float((plain.multiply(v[0], v[1:], lists[0], lists[1], act)[2] * dy.double().numpy()).sum())

    for i, g in enumerate(grads):
        for _ in range(12):
            place = tuple(rng.integers(0, d) for d in values[i].shape)
            step = 1e-4
            up, down = ([v.copy() for v in values] for _ in range(2))
            up[i][place] += step
            down[i][place] -= step
            slope = (loss(up) - loss(down)) / (2 * step)
            # two roundings to 11 bits of at most 16 terms of size ~1, and the
            # differences' own error
            assert abs(float(g[place]) - slope) <= 2 ** -11 * abs(slope) + 2 ** -11 * 16 * 2 + 1e-5


def test_nothing(gpu):
    torch, moe = gpu
    w = torch.ones((2, 8, 16), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.zeros((0, 16), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = moe.gated(x, w, w, none)
    assert y.shape == (0, 8)
    dx, dw = torch.autograd.grad(y, [x, w], y.detach())
    assert dx.shape == (0, 16) and not host(dw).any()
    # slots, but no rows
    row = torch.tensor([0, 1, -1, 3], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    list_ = torch.zeros((0, 2), dtype=torch.int32, device="cuda")
    for y in (moe.product(x, w, offsets, row, list_), moe.gated(x, w, w, offsets, row, list_)):
        assert y.shape == (4, 8) and not host(y).any()
        dx, dw = torch.autograd.grad(y, [x, w], torch.full_like(y, float("nan")))
        assert dx.shape == (0, 16) and not host(dw).any()
    # rows without a slot have a gradient of zero
    x = torch.ones((3, 16), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = moe.product(x, w, offsets[:3] * 0, row[:0], torch.full((3, 1), -1, dtype=torch.int32, device="cuda"))
    assert not host(torch.autograd.grad(y, x, y.detach())[0]).any()


def test_two_dimensional_weights_and_expanded_gradients(gpu):
    torch, moe = gpu
    rng = np.random.default_rng(7)
    x = torch.from_numpy(rng.normal(0, 1, (50, 40))).bfloat16().cuda().requires_grad_()
    w = torch.from_numpy(rng.normal(0, 0.1, (24, 40))).bfloat16().cuda().requires_grad_()
    y = moe.product(x, w)
    y.sum().backward()          # a gradient whose strides are 0
    assert x.grad.shape == x.shape and w.grad.shape == w.shape
    want = host(w).sum(0)
    assert np.allclose(host(x.grad), np.broadcast_to(want, (50, 40)), rtol=2 ** -8 + 1e-5, atol=1e-4)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(moe.product(x, w).float().square().sum(), x, create_graph=True)[0].sum(), w)


def test_offsets_beyond_32_bits(gpu):
    """Rows and weights whose elements' numbers pass 2^32."""
    torch, moe = gpu
    rows, cols, pitch, n = 70000, 64, 65600, 40
    x = torch.zeros((rows, pitch), dtype=torch.bfloat16, device="cuda")[:, :cols]      # 4.6e9 elements
    used = torch.tensor([0, 69999, 65536, 32768, 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[used] = torch.randn((5, cols), generator=g, device="cuda").bfloat16()
    w = torch.randn((n, cols), generator=g, device="cuda").bfloat16()
    y = moe.product(x, w, row_of_slot=used.int())
    want = x[used].double() @ w.double().t()
    assert torch.all((y.double() - want).abs() <= want.abs() * 2 ** -8 + 1e-4)
    del x
    experts, n, cols = 1024, 2048, 2056      # 4.3e9 elements
    w = torch.zeros((experts, n, cols), dtype=torch.bfloat16, device="cuda")
    w[-1] = torch.randn((n, cols), generator=g, device="cuda").bfloat16()
    w[-2] = torch.randn((n, cols), generator=g, device="cuda").bfloat16()
    x = torch.randn((5, cols), generator=g, device="cuda").bfloat16()
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[-2], offsets[-1] = 2, 5
    y = moe.product(x, w, offsets)
    want = torch.cat([x[:2].double() @ w[-2].double().t(), x[2:].double() @ w[-1].double().t()])
    assert torch.all((y.double() - want).abs() <= want.abs() * 2 ** -8 + 2e-2)


def test_streams_and_graphs(gpu):
    """On a stream of their own, and captured with the backward pass and
    replayed with other inputs, with eager work between the replays."""
    torch, moe = gpu
    rng = np.random.default_rng(8)
    lists = [torch.from_numpy(a).cuda() for a in plan(rng, 300, 4, 2, 0.1, "token")]
    make = lambda *s: torch.from_numpy(rng.normal(0, 1, s)).bfloat16().cuda()      # noqa: E731
    x, wg, wu, wd, dy = make(300, 64), make(4, 48, 64), make(4, 48, 64), make(4, 64, 48), make(600, 64)

    def passes(x, wg, wu, wd, dy, offsets, row, list_):
        leaves = [t.detach().requires_grad_() for t in (x, wg, wu, wd)]
        y = moe.product(moe.gated(*leaves[:3], offsets, row, list_), leaves[3], offsets)
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    want = passes(x, wg, wu, wd, dy, *lists)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = passes(x, wg, wu, wd, dy, *lists)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = passes(x, wg, wu, wd, dy, *lists)
    for turn in range(4):
        x.copy_(make(300, 64))
        dy.copy_(make(600, 64))
        if turn == 2:
            for a, b in zip(lists, plan(rng, 300, 4, 2, 0.3, "token")):
                a.copy_(torch.from_numpy(b))
        graph.replay()
        want = passes(x, wg, wu, wd, dy, *lists)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_same_bits(gpu):
    torch, moe = gpu
    rng = np.random.default_rng(9)
    lists = [torch.from_numpy(a).cuda() for a in plan(rng, 2000, 5, 3, 0.1, "token")]
    make = lambda *s: torch.from_numpy(rng.normal(0, 1, s)).bfloat16().cuda().requires_grad_()      # noqa: E731
    x, wg, wu, dy = make(2000, 136), make(5, 72, 136), make(5, 72, 136), make(6000, 72)
    first = None
    for _ in range(3):
        y = moe.gated(x, wg, wu, *lists)
        out = (y, *torch.autograd.grad(y, [x, wg, wu], dy.detach()))
        assert first is None or all(torch.equal(a, b) for a, b in zip(out, first))
        first = out


@pytest.mark.parametrize("cols", [64, 50])
@pytest.mark.parametrize("slots", [50, 700])
def test_outputs_inside_wider_arrays(gpu, cols, slots):
    """The C calls on parts of wider arrays; offsets that decrease or leave the
    array (which callers must not give) write nothing outside the result."""
    torch, moe = gpu
    from paper_2505_01616_amd import netsim as ns
    rng = np.random.default_rng(10)
    experts, n, pad = 4, 72, 5
    make = lambda *s: torch.from_numpy(rng.normal(0, 1, s)).bfloat16().cuda()      # noqa: E731
    x, w, w2 = make(slots, cols), make(experts, n, cols), make(experts, n, cols)
    x8, w8 = moe.quantise(x), moe.quantise(w)
    stream = torch.cuda.current_stream().cuda_stream
    for k, bounds in enumerate(([0, slots // 3, slots // 3, slots - 4, slots - 1], [5, 2, 9 * slots, -3, slots // 2])):
        offsets = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        for op in range(3):
            wide = torch.full((3 * slots, n + pad), 7.0, dtype=torch.bfloat16, device="cuda")
            y = wide[slots:2 * slots, :n]
            tail = (slots, x.data_ptr(), cols, None, offsets.data_ptr())
            if op == 0:
                ns.netsim_experts_product(0, experts, slots, n, cols, ns.BF16, *tail, w.data_ptr(), y.data_ptr(), n + pad, stream)
                want = moe.product(x, w, offsets) if k == 0 else None
            elif op == 1:
                ns.netsim_experts_gated(0, experts, slots, n, cols, ns.BF16, ns.SILU, *tail, w.data_ptr(), w2.data_ptr(), y.data_ptr(),
                                        n + pad, None, None, stream)
                want = moe.gated(x, w, w2, offsets) if k == 0 else None
            else:
                ns.netsim_experts_product8(0, experts, slots, n, cols, slots, x8.q.data_ptr(), x8.scales.data_ptr(), None,
                                           offsets.data_ptr(), w8.q.data_ptr(), w8.scales.data_ptr(), ns.BF16, y.data_ptr(), n + pad, stream)
                want = moe.product8(x8, w8, offsets) if k == 0 else None
            assert want is None or torch.equal(y, want)
            y.fill_(7.0)
            assert bool((wide == 7.0).all()), (k, op)
        if k:
            leaves = [t.detach().requires_grad_() for t in (x, w, w2)]
            torch.autograd.grad(moe.gated(*leaves, offsets), leaves, torch.ones((slots, n), dtype=torch.bfloat16, device="cuda"))
            torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("act", [None, "gelu"])
def test_large_tiles(gpu, kind, act):
    """Sizes that take tiles of 256 (but one matrix's gradients), rows from a list with some
    missing, last tiles and steps of every kind cut short."""
    torch, moe = gpu
    g = torch.Generator(device="cuda").manual_seed(11)
    t = types(torch)[kind]
    experts, slots, rows, n, cols = 3, 14000, 5000, 1288, 1096
    w = [(torch.randn((experts, n, cols), generator=g, device="cuda") * cols ** -0.5).to(t) for _ in range(2 if act else 1)]
    x = torch.randn((rows, cols + 8), generator=g, device="cuda").to(t)[:, :cols]
    dy = torch.randn((slots, n), generator=g, device="cuda").to(t)
    offsets = torch.tensor([3, 9001, 9001, 13990], dtype=torch.int32, device="cuda")
    row = (torch.arange(slots, device="cuda") * 7 % rows).int()
    row[[4000, 9500]] = -1
    at = row.long().clamp(min=0)
    order = torch.argsort(torch.where(row < 0, rows, at), stable=True)[: slots - 2]
    first = torch.searchsorted(at[order], torch.arange(rows, device="cuda"))
    place = torch.arange(slots - 2, device="cuda") - first[at[order]]
    lists = torch.full((rows, 3), -1, dtype=torch.int32, device="cuda")
    lists[at[order], place] = order.int()
    leaves = [v.detach().requires_grad_() for v in (x, *w)]
    more = dict(offsets=offsets, row_of_slot=row, slots_of_row=lists)
    y = moe.gated(*leaves, activation=act, **more) if act else moe.product(*leaves, **more)
    got = (y.detach(), *torch.autograd.grad(y, leaves, dy))
    # the same in 64 bits, expert by expert
    X, W, D = x.double(), [v.double() for v in w], dy.double()
    want = [torch.zeros((slots, n), dtype=torch.float64, device="cuda"), torch.zeros_like(X), *(torch.zeros_like(v) for v in W)]
    bounds = offsets.tolist()
    for e in range(experts):
        s = torch.arange(bounds[e], bounds[e + 1], device="cuda")
        s = s[row[s] >= 0]
        if not len(s):
            continue
        v = [X[at[s]].requires_grad_(), *(u[e].clone().requires_grad_() for u in W)]
        z = v[0] @ v[1].t()
        if act:
            z = torch.nn.functional.gelu(z) * (v[0] @ v[2].t())
        grads = torch.autograd.grad(z, v, D[s])
        want[0][s] = z.detach()
        want[1].index_add_(0, at[s], grads[0])
        for i, d in enumerate(grads[1:]):
            want[2 + i][e] = d
    # a rounding of the result, and of dg and du before it: each at most a half
    # step of every value, so together 2.1 of them in the 2-norm; element by
    # element against the largest, as sums of cancelling terms are off by theirs
    for a, b in zip(got, want):
        a = a.double()
        assert float((a - b).norm() / b.norm()) <= 2.1 * HALF[kind]
        assert float((a - b).abs().max()) <= 2.1 * HALF[kind] * float(b.abs().max())
    zero = torch.zeros_like(row, dtype=torch.bool)
    zero[:3] = zero[13990:] = zero[4000] = zero[9500] = True
    assert not got[0][zero].any() and not got[2][1].any()
