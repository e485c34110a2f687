"""Operators of an expert-parallel layer on torch tensors (the
``netsim_route``, ``netsim_dispatch`` and ``netsim_act_*`` calls of
include/netsim.h, which holds their definitions).

What they compute is what a simulation of such a layer is given: the experts
that the tokens choose, the bytes every rank then sends to every other one
(the matrix of ``netsim_add_all_to_all``), and, timed on one GPU, the
durations of the layer's computations.

Argument checks and marshalling only; every step runs in the library's HIP
kernels, on torch's current stream of the tensors' device, and returns
without waiting.  Tensors of another stream have to be ready on it, as for
any torch operation.  Rows may be parts of wider tensors; the last dimension
is contiguous.  Failures raise ``NetsimError``, wrong tensors ``ValueError``.

The weights of ``route`` carry their gradient to the logits (once; the bias
has none).  The results of the other calls carry none: they are whole numbers,
made from whole numbers, or gradients themselves.
"""

from __future__ import annotations

from dataclasses import dataclass
from typing import NamedTuple, Optional

import torch

from . import netsim as ns

# the current stream's handle without a Stream object around it (1.9 us of a
# call that otherwise takes 8)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_TYPES = {torch.float32: ns.F32, torch.bfloat16: ns.BF16, torch.float16: ns.F16}
_SCORES = {"softmax": ns.SCORES_SOFTMAX, "sigmoid": ns.SCORES_SIGMOID}
BLOCK = 32      # columns of a saved row that share an exponent


@dataclass(frozen=True)
class Router:
    """How tokens choose experts (netsim_router)."""

    experts: int
    top_k: int
    scores: str = "softmax"
    renormalise: bool = True
    groups: int = 1
    groups_kept: int = 1
    group_best: int = 1
    scale: float = 1.0

    def __post_init__(self):
        if self.scores not in _SCORES:
            raise ValueError("scores: 'softmax' or 'sigmoid'")
        object.__setattr__(self, "struct", ns.netsim_router(
            self.experts, self.top_k, _SCORES[self.scores], int(self.renormalise), self.groups, self.groups_kept,
            self.group_best, self.scale))


class Dispatch(NamedTuple):
    offsets: torch.Tensor           # int32 [experts + 1]
    token_of_slot: torch.Tensor     # int32 [tokens * top_k]
    slot_of_choice: torch.Tensor    # int32 [tokens, top_k]
    traffic: torch.Tensor           # float64 [ranks, ranks], bytes


class Saved(NamedTuple):
    """Rows saved in 8 bits."""

    q: torch.Tensor                 # int8 [rows, 32 * blocks]
    exponents: torch.Tensor         # int8 [rows, blocks]
    cols: int

    @property
    def row_bytes(self) -> int:
        """Bytes of a row as it is kept and as it travels."""
        return self.q.shape[1] + self.exponents.shape[1]


def _rows(name: str, t: torch.Tensor, types) -> int:
    """Checks a two-dimensional tensor of rows; its row pitch in elements."""
    if t.dim() != 2 or t.dtype not in types or not t.is_cuda:
        raise ValueError(f"{name}: rows of {', '.join(str(d) for d in types)} on a GPU are wanted")
    rows, cols = t.shape
    if rows > 1 and t.stride(0) < cols or cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap")
    return t.stride(0) if rows > 1 else cols


def _flat(name: str, t: torch.Tensor, dtype, shape, device):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} on {device} is wanted")


def _at(device):
    """(ordinal, current stream) of a tensor's device."""
    return device.index, _raw_stream(device.index)


def _route(router: Router, logits: torch.Tensor, bias: Optional[torch.Tensor]):
    ld = _rows("logits", logits, _TYPES)
    tokens, n = logits.shape
    if n != router.experts:
        raise ValueError("logits: one column per expert is wanted")
    device = logits.device
    if bias is not None:
        _flat("bias", bias, torch.float32, (n,), device)
    index, stream = _at(device)
    experts = torch.empty((tokens, router.top_k), dtype=torch.int32, device=device)
    weights = torch.empty((tokens, router.top_k), dtype=torch.float32, device=device)
    ns.netsim_route(index, router.struct, tokens, _TYPES[logits.dtype], logits.data_ptr(), ld,
                    None if bias is None else bias.data_ptr(), experts.data_ptr(), weights.data_ptr(), stream)
    return experts, weights


class _Routed(torch.autograd.Function):
    """route's weights as a function of its logits, the choice held."""

    @staticmethod
    def forward(ctx, logits, router, bias):
        experts, weights = _route(router, logits, bias)
        ctx.router = router
        ctx.save_for_backward(logits, experts)
        ctx.mark_non_differentiable(experts)
        return experts, weights

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, dweights):
        logits, experts = ctx.saved_tensors
        return route_backward(ctx.router, logits, experts, dweights.contiguous()), None, None


def route(router: Router, logits: torch.Tensor, bias: Optional[torch.Tensor] = None):
    """logits [tokens, experts] -> (experts int32, weights float32), both
    [tokens, top_k]; -1 and 0 where a row has no further expert."""
    if logits.requires_grad and torch.is_grad_enabled():
        return _Routed.apply(logits, router, bias)
    return _route(router, logits, bias)


def route_backward(router: Router, logits: torch.Tensor, experts: torch.Tensor, dweights: torch.Tensor) -> torch.Tensor:
    """The logits' gradient [tokens, experts] from that of the weights."""
    ld = _rows("logits", logits, _TYPES)
    tokens, n = logits.shape
    if n != router.experts:
        raise ValueError("logits: one column per expert is wanted")
    device = logits.device
    _flat("experts", experts, torch.int32, (tokens, router.top_k), device)
    _flat("dweights", dweights, torch.float32, (tokens, router.top_k), device)
    index, stream = _at(device)
    out = torch.empty((tokens, n), dtype=logits.dtype, device=device)
    ns.netsim_route_backward(index, router.struct, tokens, _TYPES[logits.dtype], logits.data_ptr(), ld,
                             experts.data_ptr(), dweights.data_ptr(), out.data_ptr(), n, stream)
    return out


def dispatch(experts: torch.Tensor, num_experts: int, ranks: int = 1, tokens_per_rank: Optional[int] = None,
             row_bytes: float = 0.0, once_per_rank: bool = False) -> Dispatch:
    """Slots of the choices `experts` [tokens, top_k] by expert, and the bytes
    every rank sends to every other one (tokens_per_rank: ceil(tokens/ranks))."""
    if experts.dim() != 2 or not experts.is_cuda:
        raise ValueError("experts: [tokens, top_k] on a GPU is wanted")
    device = experts.device
    tokens, top_k = experts.shape
    _flat("experts", experts, torch.int32, (tokens, top_k), device)
    per = tokens_per_rank if tokens_per_rank is not None else max(1, -(-tokens // max(1, ranks)))
    work = max(0, ns.netsim_dispatch_work_bytes(num_experts, top_k, tokens, ranks, per))
    index, stream = _at(device)
    # the whole numbers are one allocation: each more would cost a tenth of a
    # small call.  So is a small call's workspace, which is a word; a larger
    # one is free again after the call, whatever the caller keeps.
    inside = work // 4 if work <= 4 else 0
    whole = torch.empty(max(0, num_experts) + 1 + 2 * tokens * top_k + inside, dtype=torch.int32, device=device)
    offsets, token_of_slot, slot_of_choice, space = whole.split_with_sizes(
        (max(0, num_experts) + 1, tokens * top_k, tokens * top_k, inside))
    if work > 4:
        space = torch.empty(work // 4, dtype=torch.int32, device=device)
    out = Dispatch(offsets, token_of_slot, slot_of_choice.view(tokens, top_k),
                   torch.empty((max(0, ranks), max(0, ranks)), dtype=torch.float64, device=device))
    ns.netsim_dispatch(index, num_experts, top_k, tokens, experts.data_ptr(), ranks, per, row_bytes,
                       int(once_per_rank), out.offsets.data_ptr(), out.token_of_slot.data_ptr(),
                       out.slot_of_choice.data_ptr(), out.traffic.data_ptr(), space.data_ptr(), work, stream)
    return out


def save(x: torch.Tensor) -> Saved:
    """Rows x [rows, cols] in 8 bits with an exponent per 32 columns."""
    ld = _rows("x", x, _TYPES)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    index, stream = _at(x.device)
    q = torch.empty((rows, blocks * BLOCK), dtype=torch.int8, device=x.device)
    exponents = torch.empty((rows, blocks), dtype=torch.int8, device=x.device)
    ns.netsim_act_save(index, rows, cols, _TYPES[x.dtype], x.data_ptr(), ld, q.data_ptr(), exponents.data_ptr(), stream)
    return Saved(q, exponents, cols)


def _saved(s: Saved):
    rows, blocks = s.q.shape[0], -(-s.cols // BLOCK)
    if not s.q.is_cuda:
        raise ValueError("saved rows: on a GPU are wanted")
    _flat("q", s.q, torch.int8, (rows, blocks * BLOCK), s.q.device)
    _flat("exponents", s.exponents, torch.int8, (rows, blocks), s.q.device)
    return rows


def restore(saved: Saved, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The rows that were saved, to the precision they were saved with."""
    rows = _saved(saved)
    if dtype not in _TYPES:
        raise ValueError("dtype: float32, bfloat16 or float16")
    index, stream = _at(saved.q.device)
    x = torch.empty((rows, saved.cols), dtype=dtype, device=saved.q.device)
    ns.netsim_act_restore(index, rows, saved.cols, saved.q.data_ptr(), saved.exponents.data_ptr(), _TYPES[dtype],
                          x.data_ptr(), saved.cols, stream)
    return x


def weight_grad(saved: Saved, dy: torch.Tensor, offsets: torch.Tensor, row_of_slot: Optional[torch.Tensor] = None,
                out_dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """dW [experts, n, cols]: for every expert the sum over its slots of
    dy[slot] (n values) times the saved row of the slot."""
    rows = _saved(saved)
    ld = _rows("dy", dy, _TYPES)
    slots, n = dy.shape
    device = dy.device
    experts = max(0, offsets.numel() - 1)
    _flat("offsets", offsets, torch.int32, (experts + 1,), device)
    if row_of_slot is not None:
        _flat("row_of_slot", row_of_slot, torch.int32, (slots,), device)
    if saved.q.device != device or out_dtype not in _TYPES:
        raise ValueError("saved rows on dy's device and a float32, bfloat16 or float16 result are wanted")
    kind = _TYPES[dy.dtype]
    work = max(0, ns.netsim_act_weight_grad_work_bytes(experts, slots, n, saved.cols, kind))
    index, stream = _at(device)
    out = torch.empty((experts, n, saved.cols), dtype=out_dtype, device=device)
    space = torch.empty(work, dtype=torch.uint8, device=device) if work else None
    ns.netsim_act_weight_grad(index, experts, slots, n, saved.cols, kind, dy.data_ptr(), ld, rows, saved.q.data_ptr(),
                              saved.exponents.data_ptr(), None if row_of_slot is None else row_of_slot.data_ptr(),
                              offsets.data_ptr(), _TYPES[out_dtype], out.data_ptr(),
                              None if space is None else space.data_ptr(), work, stream)
    return out
