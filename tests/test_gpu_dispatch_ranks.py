"""Dispatch where few of the ranks hold tokens, and what its results keep."""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,k,experts,ranks,per", [
    (20000, 8, 256, 64, 20000), (20000, 8, 256, 64, 2 ** 40), (20000, 8, 256, 64, 7000), (9000, 3, 1000, 500, 4500),
    (5000, 4, 1024, 1024, 5000), (30, 2, 64, 64, 30), (30, 2, 64, 64, 29), (1, 8, 64, 64, 2 ** 62), (1025, 8, 8, 8, 1024),
])
@pytest.mark.parametrize("once", [False, True])
def test_ranks_without_tokens(gpu, tokens, k, experts, ranks, per, once):  # noqa: F811
    torch, moe = gpu
    rng = np.random.default_rng(tokens + k)
    e = np.minimum((rng.random((tokens, k)) ** 3 * experts).astype(np.int32), experts - 1)
    e[rng.random((tokens, k)) < 0.05] = -1
    got = moe.dispatch(torch.from_numpy(e).cuda(), experts, ranks=ranks, tokens_per_rank=per, row_bytes=1056.0,
                       once_per_rank=once)
    want = plain.dispatch(e, experts, ranks, per, 1056.0, once)
    for name, g, w in zip(got._fields, got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)


@pytest.mark.parametrize("tokens,k,experts,ranks", [(48, 2, 8, 8), (1000, 8, 256, 64), (20000, 8, 256, 64), (3000, 4, 1024, 1024)])
def test_results_keep_no_workspace(gpu, tokens, k, experts, ranks):  # noqa: F811
    """What a result keeps alive are the results (and one word at most)."""
    torch, moe = gpu
    e = torch.randint(0, experts, (tokens, k), dtype=torch.int32, device="cuda")
    d = moe.dispatch(e, experts, ranks=ranks, row_bytes=8.0)
    whole = sum(t.numel() * 4 for t in (d.offsets, d.token_of_slot, d.slot_of_choice))
    for t in (d.offsets, d.token_of_slot, d.slot_of_choice):
        assert t.untyped_storage().nbytes() <= whole + 4
