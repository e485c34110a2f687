"""The operators at sizes that take their other shapes: many rows (few lanes
per row in routing), wide tiles, sums in parts and more experts than slots
(weight gradients).  The same bounds as tests/test_gpu_operators.py."""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import SMALL, STEP, U, draw_logits, grad_case, gpu, near, types, wide  # noqa: F401
from tests.test_gpu_operators import host

pytestmark = pytest.mark.gpu

# 128 experts or fewer take eight lanes per row from 32,768 rows on, 256 or
# fewer sixteen from 16,384
ROUTERS = [
    (dict(experts=5, top_k=3), 33000),
    (dict(experts=30, top_k=4, scores="sigmoid", groups=6, groups_kept=2, group_best=2), 33001),
    (dict(experts=60, top_k=12, renormalise=False), 33007),
    (dict(experts=64, top_k=8, groups=8, groups_kept=4, group_best=2, scale=2.5), 33000),
    (dict(experts=128, top_k=8, scores="sigmoid", renormalise=False), 32769),
    (dict(experts=120, top_k=32, groups=24, groups_kept=12), 33000),
    (dict(experts=129, top_k=8, renormalise=False), 16500),
    (dict(experts=256, top_k=8, scores="sigmoid", groups=8, groups_kept=4, group_best=2, scale=2.5), 16385),
    (dict(experts=250, top_k=20, groups=25, groups_kept=10, group_best=2), 16500),
    (dict(experts=256, top_k=1), 16390),
    (dict(experts=1024, top_k=8), 3001),
    (dict(experts=1000, top_k=16, scores="sigmoid", scale=0.5), 2501),
    (dict(experts=513, top_k=3, scores="sigmoid", renormalise=False), 2500),
]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("cfg,rows", ROUTERS, ids=lambda c: "-".join(str(v) for v in c.values()) if isinstance(c, dict) else str(c))
def test_route_many_rows(gpu, cfg, rows, with_bias, kind):  # noqa: F811
    """A few rows over and over: every repeat has the first one's choices and
    weights, whichever lanes it falls to."""
    torch, moe = gpu
    r = moe.Router(**cfg)
    bias = None
    if with_bias:
        bias = (np.random.default_rng(6).permutation(r.experts) * 0.0137 - 0.2).astype(np.float32).astype(np.float64)
    x = draw_logits(torch, r, 41, kind, bias, 13)
    at = np.arange(rows) % len(x)
    pad = 3 if rows % 2 else 0      # rows that vectors can and cannot read
    few = torch.from_numpy(x).to(types(torch)[kind]).cuda()
    big = torch.full((rows, r.experts + pad), float("nan"), dtype=few.dtype, device="cuda")
    logits = big[:, :r.experts]
    logits.copy_(few[torch.from_numpy(at).cuda()])
    e, w = moe.route(r, logits, None if bias is None else torch.from_numpy(bias).float().cuda())
    want_e, want_w = plain.route(r, x, bias)
    keep = ~near(r, x, bias)[at]
    np.testing.assert_array_equal(e.cpu().numpy()[keep], want_e[at][keep])
    far = np.where(np.isfinite(x), x, 0)
    far = far.max(1) - far.min(1)
    far[far > 1000] = 0
    bound = (2 * far[:, None] + 40) * U * want_w + 1e-37
    assert (np.abs(host(w) - want_w[at])[keep] <= bound[at][keep]).all()

    dw = np.random.default_rng(9).normal(0, 1, want_e.shape).astype(np.float32)
    got = moe.route_backward(r, logits, torch.from_numpy(want_e[at]).int().cuda(), torch.from_numpy(dw[at]).cuda())
    want = plain.route_backward(r, x, want_e, dw)
    s = plain.scores(r.scores, x)
    total = (np.abs(dw) * (want_e >= 0)).sum(1, keepdims=True) * r.scale
    size = np.ones_like(s) if r.renormalise else s
    bound = (4 * far[:, None] + 100) * U * total * size + (STEP[kind] * np.abs(want) + SMALL[kind])
    assert (np.abs(host(got) - want[at]) <= bound[at]).all()


@pytest.mark.parametrize("kind,out,tokens,k,experts,n,cols,pad", [
    ("bf16", "bf16", 26000, 2, 3, 1001, 1016, 0),      # wide tiles, rows of odd length
    ("bf16", "f32", 13000, 4, 9, 1024, 1100, 8),
    ("f16", "f32", 13000, 2, 4, 1025, 1024, 0),
    ("f32", "bf16", 9000, 2, 2, 1030, 1000, 2),
    ("f32", "f16", 300, 2, 1000, 24, 40, 0),           # more experts than slots
    ("bf16", "f32", 20000, 1, 1, 40, 50, 0),           # one sum in many parts
    ("bf16", "bf16", 3000, 4, 2, 40, 1000, 0),
    ("f16", "bf16", 5000, 2, 8, 300, 260, 1),
    ("f32", "f32", 2100, 1, 1, 7, 33, 0),
])
def test_weight_grad(gpu, kind, out, tokens, k, experts, n, cols, pad):  # noqa: F811
    torch, moe = gpu
    rng = np.random.default_rng(tokens + n)
    off, token, (q, e) = grad_case(rng, tokens, k, experts, n, cols)
    dy = torch.from_numpy(rng.normal(0, 0.02, (tokens * k, n))).to(types(torch)[kind]).double().numpy()
    dy[off[-1]:] = np.nan
    saved = moe.Saved(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda(), cols)
    got = moe.weight_grad(saved, wide(torch, dy, types(torch)[kind], pad), torch.from_numpy(off).int().cuda(),
                          torch.from_numpy(token).int().cuda(), out_dtype=types(torch)[out])
    # the 64-bit sums on the GPU: products of torch, in segments
    x = torch.from_numpy(plain.restore(q, e, cols)).cuda()
    d = torch.from_numpy(dy).cuda()
    rows = torch.from_numpy(token).cuda()
    for i in range(experts):
        a, b = int(off[i]), int(off[i + 1])
        left, right = d[a:b].t().contiguous(), x[rows[a:b]]
        want, size = left @ right, left.abs() @ right.abs()
        bound = (b - a + 8) * U * size + STEP[out] * want.abs() + (2.0 ** -24 if out == "f16" else 1e-37)
        assert ((got[i].double() - want).abs() <= bound).all(), i


def test_weight_grad_twice_the_same_bits(gpu):  # noqa: F811
    """Sums in parts are joined in one order."""
    torch, moe = gpu
    rng = np.random.default_rng(3)
    off, token, (q, e) = grad_case(rng, 6000, 2, 3, 128, 200)
    saved = moe.Saved(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda(), 200)
    dy = torch.from_numpy(rng.normal(0, 1, (12000, 128))).float().cuda()
    args = (saved, dy, torch.from_numpy(off).int().cuda(), torch.from_numpy(token).int().cuda())
    first = moe.weight_grad(*args)
    for _ in range(3):
        assert torch.equal(first, moe.weight_grad(*args))


@pytest.mark.parametrize("tokens,k,experts,ranks,per", [(40000, 8, 256, 64, None), (70001, 3, 1000, 250, None),
                                                        (4097, 1, 512, 512, 9), (33000, 32, 32, 2, 20000)])
@pytest.mark.parametrize("once", [False, True])
def test_dispatch(gpu, tokens, k, experts, ranks, per, once):  # noqa: F811
    torch, moe = gpu
    rng = np.random.default_rng(tokens)
    e = np.minimum((rng.random((tokens, k)) ** 4 * experts).astype(np.int32), experts - 1)
    e[rng.random((tokens, k)) < 0.02] = -1
    got = moe.dispatch(torch.from_numpy(e).cuda(), experts, ranks=ranks, tokens_per_rank=per, row_bytes=3.0,
                       once_per_rank=once)
    want = plain.dispatch(e, experts, ranks, per or -(-tokens // ranks), 3.0, once)
    for name, g, w in zip(got._fields, got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)


def test_weight_grad_against_differences(gpu):  # noqa: F811
    """L(W) = sum over slots of dy_s . (W_e x_row(s)) is linear in W, so its
    central differences are its gradient whatever the step (64-bit sums)."""
    torch, moe = gpu
    rng = np.random.default_rng(11)
    off, token, (q, e) = grad_case(rng, 60, 2, 3, 20, 45)
    dy = rng.normal(0, 1, (120, 20)).astype(np.float32)
    saved = moe.Saved(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda(), 45)
    got = host(moe.weight_grad(saved, torch.from_numpy(dy).cuda(), torch.from_numpy(off).int().cuda(),
                               torch.from_numpy(token).int().cuda()))
    x = plain.restore(q, e, 45)
    expert = np.repeat(np.arange(3), np.diff(off))
    slots = np.arange(off[-1])

    def loss(w):
        return np.einsum("si,sic,sc->", dy[slots].astype(np.float64), w[expert], x[token[slots]])

    w = rng.normal(0, 1, (3, 20, 45))
    size = plain.weight_grad(np.abs(x), np.abs(dy), off, token)
    for _ in range(40):
        at = (rng.integers(3), rng.integers(20), rng.integers(45))
        up, down = w.copy(), w.copy()
        up[at] += 0.5
        down[at] -= 0.5
        # the difference of two 64-bit sums of about 10^5 terms
        assert abs(got[at] - (loss(up) - loss(down))) <= 130 * U * size[at] + 1e-8


def test_operators_of_nothing(gpu):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(8, 2)
    none = torch.empty((0, 8), device="cuda")
    e, w = moe.route(r, none)
    assert e.shape == w.shape == (0, 2)
    assert moe.route_backward(r, none, e, w).shape == (0, 8)
    saved = moe.save(none)
    assert moe.restore(saved).shape == (0, 8)
    # slots whose rows do not exist count as zeros
    off = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    got = moe.weight_grad(saved, torch.ones((3, 4), device="cuda"), off)
    assert got.shape == (1, 4, 8) and (got == 0).all()


def test_rows_past_32_bit_offsets(gpu):  # noqa: F811
    """More than 2^31 saved values, and gradients in rows 60,000 apart."""
    torch, moe = gpu
    rows, cols = 60000, 40000
    try:
        x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
        dy = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")[:, :16]
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no memory for it")
    g = torch.Generator(device="cuda").manual_seed(2)
    x[-1] = torch.randn(cols, generator=g, device="cuda").to(torch.bfloat16)
    dy[-1] = torch.randn(16, generator=g, device="cuda").to(torch.bfloat16)
    dy[0] = dy[-1]
    saved = moe.save(x)
    last = plain.restore(*plain.save(host(x[-1:])), cols)
    assert (saved.q[:-1].max() == 0) and np.array_equal(host(moe.restore(saved)[-1:]), last)
    # slot rows - 1 reads its own row, the last; slot 0 row 0 (zeros), then the last as well
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    once = host(moe.weight_grad(saved, dy, off))[0]
    want = host(dy[-1])[:, None] * last
    assert np.array_equal(once, want)       # one product each, of 15 bits
    row = torch.arange(rows, dtype=torch.int32, device="cuda")
    row[0] = rows - 1
    twice = host(moe.weight_grad(saved, dy, off, row))[0]
    assert np.array_equal(twice, 2 * want)
