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
