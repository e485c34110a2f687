"""Routing, its gradient, dispatch, activations saved in 8 bits and weight
gradients (moe.py on the HIP kernels) against oracle/moe.py in 64 bits.

Bounds.  u = 2^-24 (float32's half step).  A score exp(d)/Z: d carries |d| u,
the exponential 4 u, a sum of up to 1024 terms over a wave its terms' errors
and 22 u, quotients and products 1 u each; numerator and sum together stay
below (2 |d| + 40) u relative, d the largest distance between two logits that
take part.  Outputs of 16 bits add half a step of their type.  A weight
gradient is a sum of exact products in 32-bit sums: below (slots + 8) u times
the sum of the products' magnitudes.
"""

import numpy as np
import pytest

from oracle import moe as plain

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}    # 8 and 11 significant bits
SMALL = {"f32": 2.0 ** -140, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_01616_amd import moe
    return torch, moe


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def wide(torch, x, dtype, pad):
    """x on the GPU in rows of `pad` more columns that hold NaN."""
    t = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=dtype, device="cuda")
    v = t[:, :x.shape[1]]
    v.copy_(torch.from_numpy(x))
    return v


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------ routing
ROUTERS = [
    dict(experts=1, top_k=1),
    dict(experts=2, top_k=2, renormalise=False),
    dict(experts=8, top_k=2, scores="sigmoid"),
    dict(experts=60, top_k=4, renormalise=False),
    dict(experts=64, top_k=6, groups=8, groups_kept=3, group_best=2),
    dict(experts=64, top_k=8, scores="sigmoid", groups=4, groups_kept=1, scale=2.5),
    dict(experts=65, top_k=7, groups=5, groups_kept=5),
    dict(experts=160, top_k=6, groups=8, groups_kept=3, scale=16.0, renormalise=False),
    dict(experts=256, top_k=8, scores="sigmoid", groups=8, groups_kept=4, group_best=2, scale=2.5),
    dict(experts=257, top_k=32, groups=257, groups_kept=40, group_best=2),
    dict(experts=384, top_k=8, scores="sigmoid", renormalise=False),
    dict(experts=1000, top_k=16, groups=2, groups_kept=1, group_best=2),
    dict(experts=1024, top_k=32, scores="sigmoid"),
]


def near(r, x, bias):
    """Rows in which two computed values that decide the choice differ by less
    than 1e-5 of the largest: their order is not the formula's but rounding's.
    Logits are compared as they are."""
    out = np.zeros(len(x), bool)
    if bias is None and not (r.groups > 1 and r.group_best > 1):
        return out
    for t, row in enumerate(plain.choice_values(r, x, bias)):
        if not (row > -np.inf).any():
            continue
        tol = 1e-5 * np.abs(row[row > -np.inf]).max()
        if r.groups > 1:
            g = np.array(plain.group_values(r, list(row)))
            order = np.argsort(-g, kind="stable")
            if r.groups_kept < r.groups:
                with np.errstate(invalid="ignore"):
                    out[t] |= g[order[r.groups_kept - 1]] - g[order[r.groups_kept]] < tol
            row = row.reshape(r.groups, -1)[order[:r.groups_kept]].reshape(-1)
        v = np.sort(row[row > -np.inf])[::-1][:r.top_k + 1]
        d = v[:-1] - v[1:]
        out[t] |= ((d > 0) & (d < tol)).any()
    return out


def draw_logits(torch, r, tokens, kind, bias, seed):
    """Logits as the type holds them, rows without near values; some with
    experts taken out, an empty one, one of the type's lowest value, one
    with equal values."""
    rng = np.random.default_rng(seed)
    dtype = types(torch)[kind]

    def rounded(a):
        return torch.from_numpy(a).to(dtype).double().numpy()

    x = rounded(rng.normal(0, 2, (tokens, r.experts)))
    if tokens > 4:
        x[1] = -np.inf
        x[2] = float(torch.finfo(dtype).min)
        x[3] = x[3, 0]
        x[4, ::2] = -np.inf
        x[5 % tokens, : r.experts - 1] = -np.inf
    for _ in range(60):
        bad = np.flatnonzero(near(r, x, bias))
        if not len(bad):
            break
        x[bad] = rounded(rng.normal(0, 2, (len(bad), r.experts)))
    keep = ~near(r, x, bias)
    keep[:1] = True
    return x[keep] if keep.sum() > 6 else x


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("cfg", ROUTERS, ids=lambda c: "-".join(str(v) for v in c.values()))
@pytest.mark.parametrize("tokens,pad", [(1, 0), (37, 3)])
def test_route(gpu, cfg, kind, with_bias, tokens, pad):
    torch, moe = gpu
    r = moe.Router(**cfg)
    # biases far apart in steps, so that few rows have near values
    bias = np.random.default_rng(5).permutation(r.experts) * 0.0137 - 0.2 if with_bias else None
    if bias is not None:
        bias = bias.astype(np.float32).astype(np.float64)
    x = draw_logits(torch, r, tokens, kind, bias, 11)
    e, w = moe.route(r, wide(torch, x, types(torch)[kind], pad),
                     None if bias is None else torch.from_numpy(bias).float().cuda())
    want_e, want_w = plain.route(r, x, bias)
    keep = ~near(r, x, bias)
    np.testing.assert_array_equal(e.cpu().numpy()[keep], want_e[keep])
    far = np.where(np.isfinite(x), x, 0)
    far = far.max(1) - far.min(1)
    far[far > 1000] = 0            # the row of lowest values: they are all equal, d = 0
    bound = (2 * far[:, None] + 40) * U * want_w + 1e-37
    assert (np.abs(host(w) - want_w)[keep] <= bound[keep]).all()


def test_route_rows_without_defined_scores(gpu):
    torch, moe = gpu
    x = np.zeros((6, 8))
    x[:] = np.arange(8)
    x[0, 3] = np.nan
    x[1, 2] = np.inf
    x[2, 0] = -np.inf
    x[3] = -np.inf
    x[4, :7] = -np.inf
    logits = torch.from_numpy(x).float().cuda()
    for scores in ("softmax", "sigmoid"):
        for renorm in (False, True):
            r = moe.Router(8, 3, scores, renorm)
            e, w = moe.route(r, logits)
            want_e, want_w = plain.route(r, x)
            np.testing.assert_array_equal(e.cpu().numpy(), want_e)
            np.testing.assert_allclose(host(w), want_w, rtol=60 * U, atol=1e-37)
            assert torch.isnan(w[0]).all() and (e[0] == -1).all()
            assert (e[3] == -1).all() and (w[3] == 0).all()
            assert e[4].tolist() == [7, -1, -1]
    # a bias that is not a number, or takes experts out
    bias = torch.zeros(8, device="cuda")
    bias[5] = float("nan")
    e, w = moe.route(moe.Router(8, 3), logits, bias)
    assert (e[[0, 1, 2, 5]] == -1).all() and torch.isnan(w[5]).all()
    assert e[4].tolist() == [7, -1, -1]     # expert 5 is masked there: its bias does not count
    bias[5] = -float("inf")
    e, _ = moe.route(moe.Router(8, 3), logits, bias)
    assert e[5].tolist() == [7, 6, 4]


def test_route_many_rows(gpu):
    """More rows than a launch's waves, ties throughout (few distinct values)."""
    torch, moe = gpu
    g = torch.Generator().manual_seed(3)
    x = torch.randint(-3, 4, (70001, 48), generator=g).float()
    r = moe.Router(48, 5, renormalise=False)
    e, w = moe.route(r, x.to(torch.bfloat16).cuda())
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(e.cpu().long(), order)
    p = torch.softmax(x.double(), 1).gather(1, order)
    assert ((w.cpu().double() - p).abs() <= 60 * U * p).all()


def test_route_rows_past_32_bit_offsets(gpu):
    """Rows 40,000 apart: the last ones lie beyond 2^31 elements."""
    torch, moe = gpu
    rows, ld = 60000, 40000
    try:
        big = torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda")
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no memory for it")
    x = big[:, :16]
    x[:, 0] = 1.0
    x[-1] = torch.arange(16, device="cuda").to(torch.bfloat16)
    e, _ = moe.route(moe.Router(16, 2), x)
    assert e[-1].tolist() == [15, 14] and e[0].tolist() == [0, 1]
    d = moe.route_backward(moe.Router(16, 2), x, e, torch.ones((rows, 2), device="cuda"))
    assert (d.float().abs() < 1e-6).all()


# --------------------------------------------------------- routing's gradient
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cfg", [c for c in ROUTERS if c.get("groups", 1) in (1, 8)],
                         ids=lambda c: "-".join(str(v) for v in c.values()))
@pytest.mark.parametrize("tokens,pad", [(1, 0), (41, 5)])
def test_route_backward(gpu, cfg, kind, tokens, pad):
    torch, moe = gpu
    r = moe.Router(**cfg)
    x = draw_logits(torch, r, tokens, kind, None, 7)
    tokens = len(x)
    e, _ = plain.route(r, x)
    dw = np.random.default_rng(8).normal(0, 1, (tokens, r.top_k)).astype(np.float32)
    got = moe.route_backward(r, wide(torch, x, types(torch)[kind], pad), torch.from_numpy(e).int().cuda(),
                             torch.from_numpy(dw).cuda())
    want = plain.route_backward(r, x, e, dw)
    far = np.where(np.isfinite(x), x, 0)
    far = far.max(1) - far.min(1)
    far[far > 1000] = 0
    # every term is a product of a score, or of a renormalised one, and of
    # differences of dw: errors relative to the sum of their magnitudes
    s = plain.scores(r.scores, x)
    used = np.where(e >= 0, 1, 0)
    total = (np.abs(dw) * used).sum(1, keepdims=True) * r.scale
    size = np.ones_like(s) if r.renormalise else s
    bound = (4 * far[:, None] + 100) * U * total * size + (STEP[kind] * np.abs(want) + SMALL[kind])
    assert (np.abs(host(got) - want) <= bound).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_backward_against_differences(gpu, scores, renorm):
    """Central differences of the 64-bit weights with step h: their error is
    h^2/6 times a third derivative, which for scores of at most 1 stays below
    8 sum |dw|; h = 1e-3."""
    torch, moe = gpu
    r = moe.Router(12, 3, scores, renorm, scale=1.5)
    rng = np.random.default_rng(2)
    x = rng.normal(0, 1, (5, 12)).astype(np.float32).astype(np.float64)
    e, _ = plain.route(r, x)
    dw = rng.normal(0, 1, (5, 3)).astype(np.float32)
    got = host(moe.route_backward(r, torch.from_numpy(x).float().cuda(), torch.from_numpy(e).int().cuda(),
                                  torch.from_numpy(dw).cuda()))
    h = 1e-3
    for t in range(5):
        total = np.abs(dw[t]).sum() * r.scale
        for c in range(12):
            up, down = x[t].copy(), x[t].copy()
            up[c] += h
            down[c] -= h
            diff = ((plain.weights_of(r, up, e[t]) - plain.weights_of(r, down, e[t])) * dw[t]).sum() / (2 * h)
            assert abs(got[t, c] - diff) <= total * (8 * h * h / 6 + 120 * U)


def test_route_backward_leaves_out_what_is_no_expert(gpu):
    torch, moe = gpu
    x = torch.randn((3, 8), device="cuda")
    e = torch.tensor([[1, -1], [99, -7], [3, 1000000000]], dtype=torch.int32, device="cuda")
    for renorm in (False, True):
        for scores in ("softmax", "sigmoid"):
            r = moe.Router(8, 2, scores, renorm)
            d = moe.route_backward(r, x, e, torch.ones((3, 2), device="cuda"))
            plain_e = np.array([[1, -1], [-1, -1], [3, -1]])
            want = plain.route_backward(r, host(x), plain_e, np.ones((3, 2)))
            assert np.abs(host(d) - want).max() <= 200 * U
            assert (d[1] == 0).all()


# ----------------------------------------------------------------- dispatch
@pytest.mark.parametrize("tokens,k,experts,ranks,per", [
    (1, 1, 1, 1, None), (1, 8, 64, 64, None), (3, 2, 8, 8, 1), (48, 2, 8, 8, None), (63, 1, 7, 7, None),
    (64, 4, 8, 1, None), (1000, 3, 60, 5, None), (1025, 8, 256, 64, None), (2000, 6, 1024, 1024, 3),
    (5000, 32, 96, 3, 4000), (20000, 8, 16, 16, None), (9001, 2, 1000, 10, 2**40),
])
@pytest.mark.parametrize("once", [False, True])
def test_dispatch(gpu, tokens, k, experts, ranks, per, once):
    torch, moe = gpu
    rng = np.random.default_rng(tokens + k)
    # a few hot experts, some choices missing, some out of range
    e = np.minimum((rng.random((tokens, k)) ** 3 * experts).astype(np.int32), experts - 1)
    e[rng.random((tokens, k)) < 0.05] = -1
    e[rng.random((tokens, k)) < 0.01] = experts + 5
    got = moe.dispatch(torch.from_numpy(e).cuda(), experts, ranks=ranks, tokens_per_rank=per, row_bytes=1056.0,
                       once_per_rank=once)
    per = per or -(-tokens // ranks)
    want = plain.dispatch(e, experts, ranks, per, 1056.0, once)
    for name, g, w in zip(got._fields, got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)


def test_dispatch_of_nothing(gpu):
    torch, moe = gpu
    d = moe.dispatch(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 16, ranks=4, row_bytes=8.0)
    assert d.offsets.tolist() == [0] * 17 and d.token_of_slot.numel() == 0 and (d.traffic == 0).all()
    d = moe.dispatch(torch.full((1000, 4), -1, dtype=torch.int32, device="cuda"), 16, ranks=4, row_bytes=8.0)
    assert (d.offsets == 0).all() and (d.token_of_slot == -1).all() and (d.slot_of_choice == -1).all()
    assert (d.traffic == 0).all()


# ------------------------------------------------------------- saved in 8 bits
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pad", [(0, 5, 0), (1, 1, 0), (3, 31, 0), (2, 32, 1), (5, 33, 0), (77, 1000, 3),
                                           (130, 256, 0), (9, 4097, 8)])
def test_save(gpu, rows, cols, pad, kind):
    torch, moe = gpu
    rng = np.random.default_rng(rows * 7 + cols)
    x = rng.normal(0, 1, (rows, cols)) * np.exp(rng.normal(0, 2, (1, cols)))
    x[rng.random(x.shape) < 0.1] = 0
    dtype = types(torch)[kind]
    if rows > 4:
        lim = torch.finfo(dtype)
        x[0] = 0
        x[1] = lim.max
        x[2] = lim.smallest_normal / 4        # subnormal
        x[3, 0] = lim.min
        x[4] = np.nan
        x[4, cols // 2:] = 1.0
        x[3, -1] = np.inf
    x = torch.from_numpy(x).to(dtype).double().numpy()
    t = wide(torch, x, dtype, pad)
    s = moe.save(t)
    q, e = plain.save(x)
    np.testing.assert_array_equal(s.q.cpu().numpy(), q)
    np.testing.assert_array_equal(s.exponents.cpu().numpy(), e)
    back = moe.restore(s, dtype)
    want = plain.restore(q, e, cols)
    got = host(back)
    assert back.shape == (rows, cols)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    np.testing.assert_array_equal(got[ok], want[ok])      # no type rounds what it saved
    step = np.repeat(np.exp2(e.astype(np.float64)), 32, axis=1)[:, :cols]
    assert (np.abs(got - x)[ok] <= step[ok]).all()
    if kind != "f32":
        full = host(moe.restore(s, torch.float32))
        np.testing.assert_array_equal(full[ok], want[ok])


# ------------------------------------------------------------ weight gradient
def grad_case(rng, tokens, k, experts, n, cols, empty=0.05):
    e = np.minimum((rng.random((tokens, k)) ** 3 * experts).astype(np.int64), experts - 1)
    e[rng.random((tokens, k)) < empty] = -1
    off, token, _, _ = plain.dispatch(e, experts, 1, max(1, tokens), 0.0, False)
    x = rng.normal(0, 1, (tokens, cols)) * np.exp(rng.normal(0, 1, (1, cols)))
    return off, token, plain.save(x)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,k,experts,n,cols,pad", [
    (1, 1, 1, 1, 1, 0), (1, 2, 4, 33, 65, 0), (5, 2, 3, 128, 128, 0), (64, 2, 2, 130, 97, 6), (100, 3, 7, 16, 1000, 0),
    (333, 2, 5, 200, 264, 8), (700, 4, 64, 65, 40, 1), (3000, 2, 2, 72, 136, 0),
])
def test_weight_grad(gpu, tokens, k, experts, n, cols, pad, kind, out):
    torch, moe = gpu
    rng = np.random.default_rng(tokens + n)
    off, token, (q, e) = grad_case(rng, tokens, k, experts, n, cols)
    dy = torch.from_numpy(rng.normal(0, 0.02, (tokens * k, n))).to(types(torch)[kind]).double().numpy()
    dy[off[-1]:] = np.nan           # slots that no expert has
    saved = moe.Saved(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda(), cols)
    got = host(moe.weight_grad(saved, wide(torch, dy, types(torch)[kind], pad), torch.from_numpy(off).int().cuda(),
                               torch.from_numpy(token).int().cuda(), out_dtype=types(torch)[out]))
    x = plain.restore(q, e, cols)
    want = plain.weight_grad(x, dy, off, token)
    size = plain.weight_grad(np.abs(x), np.abs(dy), off, token)
    longest = np.diff(off).max()
    bound = (longest + 8) * U * size + STEP[out] * np.abs(want) + 1e-37
    assert (np.abs(got - want) <= bound).all()


def test_weight_grad_rows_in_order_and_out_of_range(gpu):
    """Without a map slot s reads row s; rows out of range count as zeros;
    values that are not finite stay with their own rows' experts."""
    torch, moe = gpu
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.normal(0, 1, (50, 70))).float().cuda()
    dy = torch.from_numpy(rng.normal(0, 1, (50, 40))).float().cuda()
    dy[20, 3] = float("nan")
    saved = moe.save(x)
    off = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device="cuda")
    back = host(moe.restore(saved))
    ids = np.arange(50)
    got = host(moe.weight_grad(saved, dy, off))
    want = plain.weight_grad(back, host(dy), off.cpu().numpy(), ids)
    assert np.isnan(got[2, 3]).all() and not np.isnan(np.delete(got[2], 3, 0)).any()
    size = plain.weight_grad(np.abs(back), np.abs(host(dy)), off.cpu().numpy(), ids)
    ok = ~np.isnan(want)
    assert (np.abs(got - want)[ok] <= 60 * U * size[ok]).all()
    assert (got[1] == 0).all()
    rows = ids.copy()
    rows[[0, 7, 30]] = [-1, 50, -2**31]
    got = host(moe.weight_grad(saved, dy, off, torch.from_numpy(rows).int().cuda()))
    want = plain.weight_grad(back, host(dy), off.cpu().numpy(), rows)
    ok = ~np.isnan(want)
    assert (np.abs(got - want)[ok] <= 60 * U * size[ok] + 1e-37).all()


def test_weight_grad_keeps_every_bit_of_dy(gpu):
    """One slot, x = 1: the gradient is dy itself."""
    torch, moe = gpu
    rng = np.random.default_rng(4)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        dy = torch.from_numpy(rng.normal(0, 1, (1, 300)) * np.exp(rng.normal(0, 4, (1, 300)))).to(dtype).cuda()
        if dtype == torch.float32:
            dy[0, 0] = torch.finfo(dtype).max
        saved = moe.save(torch.ones((1, 3), device="cuda"))
        off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        got = moe.weight_grad(saved, dy, off)[0, :, 0]
        assert torch.equal(got, dy[0].float())


def test_weight_grad_without_slots(gpu):
    torch, moe = gpu
    saved = moe.save(torch.ones((4, 40), device="cuda"))
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got = moe.weight_grad(saved, torch.empty((0, 24), device="cuda"), off, out_dtype=dtype)
        assert got.shape == (3, 24, 40) and (got == 0).all() and got.dtype == dtype


# ------------------------------------------------------- streams and graphs
def test_calls_on_another_stream_and_in_a_graph(gpu):
    """The chain of a layer on a side stream, then captured and replayed with
    other inputs and eager work in between: the same bits as eager calls."""
    torch, moe = gpu
    r = moe.Router(32, 4, "sigmoid", groups=4, groups_kept=2, group_best=2)
    g = torch.Generator(device="cuda").manual_seed(1)

    def inputs():
        return (torch.randn((600, 32), generator=g, device="cuda").to(torch.bfloat16),
                torch.randn((600, 200), generator=g, device="cuda"),
                torch.randn((2400, 72), generator=g, device="cuda").to(torch.bfloat16),
                torch.randn((600, 4), generator=g, device="cuda"))

    def layer(logits, x, dy, dw):
        e, w = moe.route(r, logits)
        d = moe.dispatch(e, 32, ranks=8, row_bytes=10.0, once_per_rank=True)
        s = moe.save(x)
        return (e, w, *d, moe.restore(s), moe.weight_grad(s, dy, d.offsets, d.token_of_slot),
                moe.route_backward(r, logits, e, dw))

    first = inputs()
    want = layer(*first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = layer(*first)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    static = [t.clone() for t in first]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer(*static)
    for _ in range(4):
        new = inputs()
        want = layer(*new)
        for a, b in zip(static, new):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held))
