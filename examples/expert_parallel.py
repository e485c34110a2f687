"""One expert-parallel layer on 64 simulated GPUs, driven by what its tokens
choose.

The layer's operators run on the one real GPU: the tokens of all ranks are
routed to their experts, the choices dispatched, the rows saved in 8 bits,
and every rank's share of the experts' weight gradients computed.  That gives
the simulation its values: the bytes of the all-to-alls (with rows sent in 8
bits, and for comparison in 16) and the time of every rank's computations,
which differ as the experts' loads do.  The step

    route and save -> all-to-all -> weight gradients -> all-to-all back

is then simulated on a leaf-spine fabric, one stream per rank.

    python examples/expert_parallel.py
"""

from __future__ import annotations

import os
import sys
from typing import NamedTuple

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2505_01616_amd import moe  # noqa: E402
from paper_2505_01616_amd.trace import run_trace  # noqa: E402
from workloads.program import Topology, gbit  # noqa: E402
from workloads.trace import Collective, Compute, Trace  # noqa: E402


class Layer(NamedTuple):
    experts: torch.Tensor        # [tokens, top_k], every rank's tokens in turn
    weights: torch.Tensor
    plan: moe.Dispatch           # slots, and the bytes of rows in 8 bits
    dlogits: torch.Tensor
    grads: torch.Tensor          # [experts, n, cols]
    before: np.ndarray           # seconds of every rank before the first all-to-all
    between: np.ndarray          # and between the two


def seconds(work, repeats: int = 3) -> float:
    """Device time of work(), the shortest of a few runs after one more."""
    work()
    times = []
    for _ in range(repeats):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        work()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e-3)
    return min(times)


def run_layer(router: moe.Router, ranks: int, logits: torch.Tensor, x: torch.Tensor, dy: torch.Tensor,
              dweights: torch.Tensor) -> Layer:
    """The layer's operators on all ranks' tokens, and every rank's times."""
    per = logits.shape[0] // ranks
    saved = moe.save(x)
    experts, weights = moe.route(router, logits)
    plan = moe.dispatch(experts, router.experts, ranks=ranks, tokens_per_rank=per, row_bytes=float(saved.row_bytes))
    grads = moe.weight_grad(saved, dy, plan.offsets, plan.token_of_slot, out_dtype=torch.bfloat16)
    dlogits = moe.route_backward(router, logits, experts, dweights)

    bounds = plan.offsets.tolist()
    own = router.experts // ranks
    before, between = np.zeros(ranks), np.zeros(ranks)
    for r in range(ranks):
        mine = slice(r * per, (r + 1) * per)
        before[r] = seconds(lambda: (moe.route(router, logits[mine]), moe.save(x[mine])))
        first, last = bounds[r * own], bounds[(r + 1) * own]
        offsets = plan.offsets[r * own: (r + 1) * own + 1] - first
        token = plan.token_of_slot[first:last]
        between[r] = seconds(lambda: moe.weight_grad(saved, dy[first:last], offsets, token, out_dtype=torch.bfloat16))
    return Layer(experts, weights, plan, dlogits, grads, before, between)


def layer_trace(ranks: int, traffic: np.ndarray, before: np.ndarray, between: np.ndarray) -> Trace:
    """The step as a trace: one stream per rank."""
    topo = Topology(kind="leaf_spine", servers=max(1, ranks // 8), gpus_per_server=min(8, ranks), servers_per_leaf=1,
                    spines=4, nvlink_Bps=900e9, nic_Bps=gbit(400), fabric_Bps=gbit(800), ecmp_seed=1)
    trace = Trace("expert-parallel layer", topo)
    ids, streams = np.arange(ranks, dtype=np.int32), np.arange(ranks)
    for r in range(ranks):
        trace.add(Compute(r, float(before[r])))
    trace.add(Collective("all_to_all", ids, streams, traffic))
    for r in range(ranks):
        trace.add(Compute(r, float(between[r])))
    trace.add(Collective("all_to_all", ids, streams, traffic.T.copy()))
    return trace


def inputs(router: moe.Router, tokens: int, cols: int, n: int, seed: int = 1):
    """Logits whose first choices follow a power law (the experts' popularity
    falls with their rank to the power 1.2), rows and gradients."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    popularity = -1.2 * torch.log(torch.randperm(router.experts, generator=g, device="cuda").float() + 1)
    noise = -torch.log(-torch.log(torch.rand((tokens, router.experts), generator=g, device="cuda").clamp_(1e-7, 1 - 1e-6)))
    return ((popularity + noise).to(torch.bfloat16),
            torch.randn((tokens, cols), generator=g, device="cuda").to(torch.bfloat16),
            (torch.randn((tokens * router.top_k, n), generator=g, device="cuda") * 0.02).to(torch.bfloat16),
            torch.randn((tokens, router.top_k), generator=g, device="cuda"))


def main():
    ranks, per, cols, n = 64, 512, 2048, 512
    router = moe.Router(experts=256, top_k=8)
    layer = run_layer(router, ranks, *inputs(router, ranks * per, cols, n))
    narrow = layer.plan.traffic.cpu().numpy()
    row = cols + cols // moe.BLOCK
    load = narrow.sum(0) / row
    print(f"rows per rank: mean {load.mean():.0f}, largest {load.max():.0f}; weight gradients "
          f"{layer.between.min() * 1e6:.0f} .. {layer.between.max() * 1e6:.0f} us")
    for name, traffic in (("8", narrow), ("16", narrow / row * 2 * cols)):
        _, _, sync, stats = run_trace(layer_trace(ranks, traffic, layer.before, layer.between))
        print(f"rows in {name} bits: the step takes {max(sync.values()) * 1e3:.3f} ms ({stats['events']} events)")
    even = np.full((ranks, ranks), narrow.sum() / ranks ** 2)
    _, _, sync, _ = run_trace(layer_trace(ranks, even, layer.before, np.full(ranks, layer.between.mean())))
    print(f"rows in 8 bits, all experts equally loaded: {max(sync.values()) * 1e3:.3f} ms")


if __name__ == "__main__":
    main()
