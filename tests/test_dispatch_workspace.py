"""The workspace of a dispatch, from the sizes alone (no call here reaches a
device)."""

import pytest

from paper_2505_01616_amd import netsim as ns


@pytest.mark.parametrize("experts,top_k,tokens,ranks", [(256, 8, 131072, 64), (1024, 8, 131072, 1024), (512, 1, 2 ** 20, 512),
                                                        (64, 2, 5000, 64)])
def test_workspace_follows_the_tokens(experts, top_k, tokens, ranks):
    """Ranks without tokens take no room: a chunk is 1,024 choices of whole
    tokens of one rank, with a counter per expert and rank, and a rank's last
    chunk may be short."""
    chunk = 1024 // top_k
    for per in (-(-tokens // ranks), tokens, tokens // 2 + 1, 3 * tokens // ranks, 2 ** 62):
        sources = -(-tokens // per)
        size = ns.netsim_dispatch_work_bytes(experts, top_k, tokens, ranks, per)
        assert 0 < size <= 4 * ((tokens // chunk + sources) * (experts + ranks) + experts)
