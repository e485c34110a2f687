"""Operators at the limits of their sizes: more rows than one grid has threads
for, rows past 32-bit offsets, workgroups that fill their shared memory."""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import STEP, U, gpu, host  # noqa: F401

pytestmark = pytest.mark.gpu


def allocate(torch, make):
    try:
        return make()
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no memory for it")


def marked(torch, tokens, experts):
    """Logits that choose expert 3, but in a few rows (where launches could be
    cut, and the last) another one: (logits, {row: expert})."""
    x = torch.zeros((tokens, experts), dtype=torch.bfloat16, device="cuda")
    x[:, 3] = 1.0
    rows = {i: 4 + n % 4 for n, i in enumerate(sorted({0, 2 ** 25 - 1, 2 ** 25, 2 ** 26 - 1, 2 ** 26, tokens // 2,
                                                       tokens - 1}))}
    for i, e in rows.items():
        x[i, e] = 2.0
    return x, rows


# 8, 16 and 64 lanes a row: 2^32 threads and a few rows more
@pytest.mark.parametrize("tokens,experts", [(2 ** 29 + 77, 8), (2 ** 28 + 3, 129), (2 ** 26 + 5, 257)])
def test_route_of_more_rows_than_a_grid(gpu, tokens, experts):  # noqa: F811
    torch, moe = gpu
    x, rows = allocate(torch, lambda: marked(torch, tokens, experts))
    e, w = allocate(torch, lambda: moe.route(moe.Router(experts, 1), x))
    assert {i: int(e[i, 0]) for i in rows} == rows
    assert int((e == 3).sum()) == tokens - len(rows)
    assert bool((w == 1).all())


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_route_backward_of_more_rows_than_a_grid(gpu, scores):  # noqa: F811
    """A sigmoid's gradient is at the chosen logit, a softmax's in the whole
    row: a kernel for each."""
    torch, moe = gpu
    tokens = 2 ** 29 + 77
    x, rows = allocate(torch, lambda: marked(torch, tokens, 8))
    r = moe.Router(8, 1, scores, False)
    e = allocate(torch, lambda: torch.full((tokens, 1), 3, dtype=torch.int32, device="cuda"))
    for i, expert in rows.items():
        e[i, 0] = expert
    dw = allocate(torch, lambda: torch.ones((tokens, 1), device="cuda"))
    got = allocate(torch, lambda: moe.route_backward(r, x, e, dw))
    at = sorted(rows) + [1, tokens - 2]
    want = plain.route_backward(r, host(x[at]), e[at].cpu().numpy(), np.ones((len(at), 1)))
    assert (np.abs(host(got[at]) - want) <= STEP["bf16"] * np.abs(want) + 200 * U).all()
    ordinary = got[1]
    same = torch.ones(tokens, dtype=torch.bool, device="cuda")
    for c in range(8):
        same &= got[:, c] == ordinary[c]
    assert int((~same).sum()) == len(rows)


def test_save_of_more_blocks_than_a_grid(gpu):  # noqa: F811
    """2^31 blocks and a few more: rows of one column."""
    torch, moe = gpu
    rows = 2 ** 31 + 5
    x = allocate(torch, lambda: torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda"))
    x += 1.0
    at = [0, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 1, 2 ** 31, rows - 1]
    for n, i in enumerate(at):
        x[i, 0] = 3.0 + n
    saved = allocate(torch, lambda: moe.save(x))
    q, e = plain.save(host(x[at]))
    np.testing.assert_array_equal(saved.q[at].cpu().numpy(), q)
    np.testing.assert_array_equal(saved.exponents[at].cpu().numpy(), e)
    back = allocate(torch, lambda: moe.restore(saved, torch.bfloat16))
    assert bool((back == x).all())


@pytest.mark.parametrize("scores,renorm", [("softmax", True), ("sigmoid", False), ("softmax", False)])
def test_route_backward_past_32_bit_offsets(gpu, scores, renorm):  # noqa: F811
    """Rows 40,000 apart, the last ones beyond 2^31 elements: every row has
    logits and weights' gradients of its own."""
    torch, moe = gpu
    rows, ld = 60000, 40000
    big = allocate(torch, lambda: torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(5)
    x = big[:, :16]
    x.copy_(torch.randn((rows, 16), generator=g, device="cuda"))
    dw = torch.randn((rows, 3), generator=g, device="cuda")
    r = moe.Router(16, 3, scores, renorm, scale=1.5)
    e, w = moe.route(r, x)
    at = [0, 1, 26843, 53687, 53688, rows - 2, rows - 1]      # 2^31 / 40,000 = 53,687
    want_e, want_w = plain.route(r, host(x[at]))
    np.testing.assert_array_equal(e[at].cpu().numpy(), want_e)
    assert (np.abs(host(w[at]) - want_w) <= 100 * U * want_w).all()
    got = host(moe.route_backward(r, x, e, dw)[at])
    want = plain.route_backward(r, host(x[at]), want_e, host(dw[at]))
    total = np.abs(host(dw[at])).sum(1, keepdims=True) * r.scale
    assert (np.abs(got - want) <= STEP["bf16"] * np.abs(want) + 200 * U * total).all()
    assert (np.abs(want).max(1) > 1e-3).all()


def test_route_backward_in_all_of_shared_memory(gpu):  # noqa: F811
    """512 experts and 8 choices, 1,024 and 16: a workgroup's rows fill 64 KB."""
    torch, moe = gpu
    for experts, k in ((512, 8), (1024, 16), (1024, 32)):
        r = moe.Router(experts, k, "sigmoid", scale=2.5)
        g = torch.Generator(device="cuda").manual_seed(experts + k)
        x = torch.randn((77, experts), generator=g, device="cuda")
        dw = torch.randn((77, k), generator=g, device="cuda")
        e, _ = moe.route(r, x)
        want = plain.route_backward(r, host(x), e.cpu().numpy(), host(dw))
        total = np.abs(host(dw)).sum(1, keepdims=True) * r.scale
        assert (np.abs(host(moe.route_backward(r, x, e, dw)) - want) <= 200 * U * total).all()


def test_calls_from_two_threads(gpu):  # noqa: F811
    """Two threads with a stream each get the bits of calls from one."""
    import threading

    torch, moe = gpu
    r = moe.Router(32, 4, "sigmoid", groups=4, groups_kept=2, group_best=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    sets = [(torch.randn((700 + 11 * i, 32), generator=g, device="cuda").to(torch.bfloat16),
             torch.randn((700 + 11 * i, 200), generator=g, device="cuda"),
             torch.randn((4 * (700 + 11 * i), 72), generator=g, device="cuda")) for i in range(2)]

    def layer(logits, x, dy):
        e, w = moe.route(r, logits)
        d = moe.dispatch(e, 32, ranks=8, row_bytes=10.0, once_per_rank=True)
        return (e, w, *d, moe.weight_grad(moe.save(x), dy, d.offsets, d.token_of_slot))

    want = [layer(*s) for s in sets]
    torch.cuda.synchronize()
    right = [0, 0]

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = layer(*sets[i])
                stream.synchronize()
                right[i] += all(torch.equal(a, b) for a, b in zip(want[i], got))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert right == [20, 20]


def test_save_over_all_magnitudes(gpu):  # noqa: F811
    """The stated error: 1/64 of the block's largest magnitude, where that is
    at least 2^-120, and 2^-127 below."""
    torch, moe = gpu
    rng = np.random.default_rng(12)
    top = np.exp2(np.arange(-149, 128))
    x = top[:, None] * rng.uniform(-1.999, 1.999, (len(top), 32))
    x[:, 0] = top
    x = torch.from_numpy(x).float().cuda()
    back = host(moe.restore(moe.save(x)))
    most = np.abs(host(x)).max(1)
    bound = np.where(most >= 2.0 ** -120, most / 64, 2.0 ** -127)
    assert np.isfinite(back).all() and (np.abs(back - host(x)) <= bound[:, None]).all()
