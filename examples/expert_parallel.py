"""One expert-parallel layer on 64 simulated GPUs, driven by what its tokens
choose.

The layer's operators run on the one real GPU: the tokens of all ranks are
routed to their experts, the choices dispatched, the rows saved in 8 bits, and
every rank's share of the experts' products and weight gradients computed (the
products y = W x and dx = dy W are torch's).  That gives the simulation its
values: the bytes of the all-to-alls (with the tokens' rows sent in 8 bits,
and for comparison in 16) and the time of every rank's computations, which
differ as the experts' loads do.  The layer's two passes

    route and save -> all-to-all of x -> y = W x -> all-to-all of y back
    route's gradient -> all-to-all of dy -> dx and dW -> all-to-all of dx back

are then simulated on a leaf-spine fabric, one stream per rank, the second
after the end of the first.

    python examples/expert_parallel.py
"""

from __future__ import annotations

import os
import sys
from typing import NamedTuple, Optional

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
    y: torch.Tensor              # [slots, n]
    dx: torch.Tensor             # [slots, cols]
    # seconds of every rank before the first all-to-all and between the two,
    before: np.ndarray           # in the forward pass
    between: np.ndarray
    back_before: np.ndarray      # and in the backward pass
    back_between: np.ndarray


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


def forward_products(w, saved: moe.Saved, bounds, token, y):
    """y of the slots of len(w) experts: their rows, which arrived in 8 bits,
    by the expert's matrix."""
    x = moe.restore(moe.Saved(saved.q[token], saved.exponents[token], saved.cols), w.dtype)
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        torch.mm(x[a:b], w[e].t(), out=y[a:b])


def backward_products(w, bounds, dy, dx):
    """dx of the same slots."""
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        torch.mm(dy[a:b], w[e], out=dx[a:b])


def run_layer(router: moe.Router, ranks: int, logits: torch.Tensor, x: torch.Tensor, dy: torch.Tensor,
              dweights: torch.Tensor, w: Optional[torch.Tensor] = None) -> Layer:
    """The layer's operators on all ranks' tokens, and every rank's times.
    w: the experts' matrices [experts, n, cols] (drawn where there are none)."""
    per = logits.shape[0] // ranks
    if w is None:
        g = torch.Generator(device="cuda").manual_seed(2)
        w = torch.randn((router.experts, dy.shape[1], x.shape[1]), generator=g, device="cuda", dtype=dy.dtype)
        w *= x.shape[1] ** -0.5
    saved = moe.save(x)
    experts, weights = moe.route(router, logits)
    plan = moe.dispatch(experts, router.experts, ranks=ranks, tokens_per_rank=per, row_bytes=float(saved.row_bytes))
    grads = moe.weight_grad(saved, dy, plan.offsets, plan.token_of_slot, out_dtype=torch.bfloat16)
    dlogits = moe.route_backward(router, logits, experts, dweights)

    bounds = plan.offsets.tolist()
    own = router.experts // ranks
    y = torch.zeros_like(dy)
    dx = torch.zeros((dy.shape[0], x.shape[1]), dtype=dy.dtype, device=dy.device)
    times = np.zeros((4, ranks))
    for r in range(ranks):
        mine, theirs = slice(r * per, (r + 1) * per), slice(r * own, (r + 1) * own)
        first, last = bounds[r * own], bounds[(r + 1) * own]
        here = [b - first for b in bounds[r * own: (r + 1) * own + 1]]
        offsets = plan.offsets[r * own: (r + 1) * own + 1] - first
        token = plan.token_of_slot[first:last]

        def backward():
            backward_products(w[theirs], here, dy[first:last], dx[first:last])
            moe.weight_grad(saved, dy[first:last], offsets, token, out_dtype=torch.bfloat16)

        times[:, r] = (seconds(lambda: (moe.route(router, logits[mine]), moe.save(x[mine]))),
                       seconds(lambda: forward_products(w[theirs], saved, here, token, y[first:last])),
                       seconds(lambda: moe.route_backward(router, logits[mine], experts[mine], dweights[mine])),
                       seconds(backward))
    return Layer(experts, weights, plan, dlogits, grads, y, dx, *times)


def layer_trace(ranks: int, traffic: np.ndarray, before: np.ndarray, between: np.ndarray,
                back: Optional[np.ndarray] = None) -> Trace:
    """One pass of the layer as a trace, one stream per rank.  back: bytes of
    the second all-to-all (the first one's, turned round)."""
    topo = Topology(kind="leaf_spine", servers=max(1, ranks // 8), gpus_per_server=min(8, ranks), servers_per_leaf=1,
                    spines=4, nvlink_Bps=900e9, nic_Bps=gbit(400), fabric_Bps=gbit(800), ecmp_seed=1)
    trace = Trace("expert-parallel layer", topo)
    ids, streams = np.arange(ranks, dtype=np.int32), np.arange(ranks)
    for r in range(ranks):
        trace.add(Compute(r, float(before[r])))
    trace.add(Collective("all_to_all", ids, streams, traffic))
    for r in range(ranks):
        trace.add(Compute(r, float(between[r])))
    trace.add(Collective("all_to_all", ids, streams, traffic.T.copy() if back is None else back))
    return trace


def simulated_step(layer: Layer, rows: np.ndarray, row_bytes: float, even: bool = False):
    """(seconds, events) of both passes.  rows[i, j]: rows from rank i's
    tokens to rank j's experts; x travels in row_bytes a row, y, dy and dx in
    16 bits a value.  even: every computation takes the mean time."""
    ranks, y_bytes, dx_bytes = len(rows), 2.0 * layer.y.shape[1], 2.0 * layer.dx.shape[1]
    times = (layer.before, layer.between, layer.back_before, layer.back_between)
    if even:
        times = tuple(np.full(ranks, t.mean()) for t in times)
    total, events = 0.0, 0
    for trace in (layer_trace(ranks, rows * row_bytes, *times[:2], back=rows.T * y_bytes),
                  layer_trace(ranks, rows * y_bytes, *times[2:], back=rows.T * dx_bytes)):
        _, _, sync, stats = run_trace(trace)
        total, events = total + max(sync.values()), events + stats["events"]
    return total, events


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
    row = cols + cols // moe.BLOCK
    rows = layer.plan.traffic.cpu().numpy() / row
    load = rows.sum(0)
    print(f"rows per rank: mean {load.mean():.0f}, largest {load.max():.0f}; y {layer.between.min() * 1e6:.0f} .. "
          f"{layer.between.max() * 1e6:.0f} us, dx and weight gradients {layer.back_between.min() * 1e6:.0f} .. "
          f"{layer.back_between.max() * 1e6:.0f} us")
    for name, size in (("8", row), ("16", 2 * cols)):
        total, events = simulated_step(layer, rows, size)
        print(f"rows in {name} bits: the step takes {total * 1e3:.3f} ms ({events} events)")
    total, _ = simulated_step(layer, np.full((ranks, ranks), rows.sum() / ranks ** 2), row, even=True)
    print(f"rows in 8 bits, all experts equally loaded: {total * 1e3:.3f} ms")


if __name__ == "__main__":
    main()
