"""The operators of an expert-parallel layer that decide what the simulator
is given, as cases to time and compare.

Routing of tokens to experts (and its gradient), the dispatch of the routed
tokens (slots by expert and the bytes every rank sends to every other one,
the matrix of an all-to-all), activations saved in 8 bits, and the experts'
weight gradients from the saved rows.  With ``own`` set ``run`` makes the
calls a user makes (``paper_2505_01616_amd.moe``); otherwise it computes the
same in elementary torch operations.  ``exact`` computes it in 64 bits.

Tokens choose experts as in the all-to-all workloads of this repository: an
expert's popularity falls with its rank to the power 1.2 (a seeded order of
the experts), and Gumbel noise on the logarithm of the popularity makes the
largest logit a draw from that distribution.
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ZIPF_S = 1.2
BLOCK = 32          # columns of a saved row that share an exponent
ROW_BYTES = 4224.0  # a row of 4096 columns saved in 8 bits, as it travels


def listed():
    return [
        # one token of a generating request: nothing but latency
        _route("route_token", 1, 64, 2, "bf16", "softmax", 1),
        # the tokens of one rank's step: scores of their own per expert, a
        # balancing bias, experts in groups of which a token uses half
        _route("route_step", 16384, 256, 8, "f32", "sigmoid", 1, bias=1, groups=8, kept=4, best=2, scale=2.5),
        # a whole step's tokens at once, rows inside a wider array, some of
        # them padding without any expert; the scores themselves as weights
        _route("route_sweep", 262144, 128, 6, "bf16", "softmax", 0, pad=8, empty=0.02),
        # gradients of a short batch of odd sizes, scores not renormalised:
        # every logit of a row has a gradient
        dict(_route("back_odd", 4099, 60, 4, "f16", "softmax", 0, empty=0.05), op="back"),
        # gradients of a long step
        dict(_route("back_step", 131072, 256, 8, "f32", "sigmoid", 1, scale=2.5), op="back"),
        # the tokens of a small generating batch, an expert per rank
        dict(name="dispatch_small", op="dispatch", tokens=48, experts=8, top_k=2, ranks=8, once=0, empty=0.1),
        # a step of 64 ranks (a group of the 4096-GPU workload), four experts
        # each; a token crosses once to a rank, however many of its experts
        # live there
        dict(name="dispatch_step", op="dispatch", tokens=131072, experts=256, top_k=8, ranks=64, once=1, empty=0.01),
        # odd sizes: rows that are no multiple of a block
        dict(name="save_odd", op="save", rows=77, cols=1000, type="f32", pad=3),
        # the rows of a layer's input, saved and read back
        dict(name="save_step", op="save", rows=32768, cols=4096, type="bf16", pad=0),
        # a few tokens on small experts
        dict(name="grad_small", op="grad", tokens=256, experts=8, top_k=2, n=512, cols=512, type="bf16", out="f32", empty=0.0),
        # odd sizes throughout, gradients with more bits than bfloat16 has
        dict(name="grad_odd", op="grad", tokens=3001, experts=16, top_k=3, n=705, cols=1000, type="f16", out="f32", empty=0.02),
        # a step's experts: a few hot ones hold most of the rows
        dict(name="grad_step", op="grad", tokens=32768, experts=64, top_k=4, n=2048, cols=2048, type="bf16", out="bf16", empty=0.0),
    ]


def _route(name, tokens, experts, top_k, type, scores, renorm, bias=0, groups=1, kept=1, best=1, scale=1.0, pad=0, empty=0.0):
    return dict(name=name, op="route", tokens=tokens, experts=experts, top_k=top_k, type=type, scores=scores, renorm=renorm, bias=bias,
                groups=groups, kept=kept, best=best, scale=scale, pad=pad, empty=empty)


def _log(rng, low, high):
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["route", "back", "dispatch", "save", "grad", "grad"])
    empty = rng.choice([0.0, 0.0, 0.03])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("route", "back"):
        groups = rng.choice([1, 1, 2, 4, 8]) if op == "route" else 1
        experts = groups * _log(rng, 2, 512 // groups)
        kept = rng.randint(1, groups)
        best = rng.choice([1, 2]) if groups > 1 else 1
        top_k = rng.randint(1, min(16, kept * (experts // groups)))
        tokens = _log(rng, 1, min(262144, 33554432 // experts))
        case = _route("", tokens, experts, top_k, kind, rng.choice(["softmax", "sigmoid"]), rng.randint(0, 1), rng.randint(0, 1) if op == "route" else 0,
                      groups, kept, best, rng.choice([1.0, 2.5]), rng.choice([0, 0, 5]), empty)
        case["op"] = op
        del case["name"]
        return case
    if op == "dispatch":
        ranks = _log(rng, 1, 64)
        experts = ranks * _log(rng, 1, max(1, 512 // ranks))
        return dict(op="dispatch", tokens=_log(rng, 1, 131072), experts=experts, top_k=rng.randint(1, min(8, experts)), ranks=ranks,
                    once=rng.randint(0, 1), empty=empty)
    if op == "save":
        return dict(op="save", rows=_log(rng, 1, 32768), cols=_log(rng, 1, 4096), type=kind, pad=rng.choice([0, 0, 7]))
    experts = _log(rng, 1, 64)
    return dict(op="grad", tokens=_log(rng, 1, 32768), experts=experts, top_k=rng.randint(1, min(4, experts)), n=_log(rng, 16, 2048), cols=_log(rng, 16, 2048),
                type=kind, out=rng.choice(["f32", "bf16"]), empty=empty)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _choices(logits, g, popularity):
    """Logits of `logits.shape`: Gumbel noise on the experts' log popularity."""
    u = torch.rand(logits, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-6)
    return popularity - torch.log(-torch.log(u))


def _popularity(experts, g):
    order = torch.randperm(experts, generator=g, device="cuda")
    p = -ZIPF_S * torch.log(order.float() + 1)
    return p - p.mean()


def _close(case, logits, bias):
    """Rows in which two scores that decide a choice are nearer to each other
    than the rounding of a 32-bit score: what is chosen there is the last bit
    of an exponential function's."""
    l = logits.double()
    s = torch.sigmoid(l) if case["scores"] == "sigmoid" else torch.softmax(l, 1)
    c = s + (0 if bias is None else bias.double())
    tol = 2e-6 * c.abs().amax(1, keepdim=True)
    c = c.masked_fill(l == -math.inf, -math.inf)
    bad = torch.zeros(len(l), dtype=torch.bool, device=l.device)
    groups, kept = case["groups"], case["kept"]
    if groups > 1:
        of = c.view(len(c), groups, -1)
        of = of.topk(min(case["best"], of.shape[2]), 2).values
        of = of[:, :, 0] + of[:, :, 1:].masked_fill(of[:, :, 1:] == -math.inf, 0).sum(2)
        of, at = of.sort(1, descending=True)
        if kept < groups:
            bad |= of[:, kept - 1] - of[:, kept] < tol[:, 0]
        use = torch.zeros_like(of, dtype=torch.bool).scatter_(1, at[:, :kept], True)
        c = c.masked_fill(~use.repeat_interleave(case["experts"] // groups, 1), -math.inf)
    top = c.topk(min(case["top_k"] + 1, c.shape[1]), 1).values
    gap = top[:, :-1] - top[:, 1:]
    return bad | ((gap > 0) & (gap < tol)).any(1)


def _logits(case, g):
    """(logits in a row of experts + pad values, bias or None)."""
    T, E, kind = case["tokens"], case["experts"], TYPES[case["type"]]
    pop = _popularity(E, g)
    # a balancing bias is moved by steps of 0.001
    bias = torch.randint(-40, 41, (E,), generator=g, device="cuda").float() * 0.001 if case["bias"] else None
    wide = torch.full((T, E + case["pad"]), 7.0, dtype=kind, device="cuda")
    # padding rows without any expert, and rows that may not use the lower half
    empty = torch.rand((T, 2), generator=g, device="cuda") < case["empty"]
    off = empty[:, :1] | (empty[:, 1:] & (torch.arange(E, device="cuda") < E // 2))
    x = wide[:, :E]
    x.copy_(_choices((T, E), g, pop).masked_fill_(off, -math.inf))
    if bias is not None or case["groups"] > 1:
        for _ in range(8):  # such rows are drawn again
            bad = _close(case, x, bias).nonzero()[:, 0]
            if not len(bad):
                break
            x[bad] = _choices((len(bad), E), g, pop).masked_fill_(off[bad], -math.inf).to(kind)
    return x, bias


def _experts(case, g):
    """Experts [tokens, top_k] as routing leaves them, -1 where there is none."""
    pop = _popularity(case["experts"], g)
    e = _choices((case["tokens"], case["experts"]), g, pop).topk(case["top_k"], 1).indices.int()
    if case["empty"]:
        e[torch.rand(case["tokens"], generator=g, device="cuda") < case["empty"]] = -1
        e[torch.rand(case["tokens"], generator=g, device="cuda") < case["empty"], -1] = -1
    return e


def _rows(shape, g):
    """Activations: normal, with columns that stand out."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x * torch.exp(0.7 * torch.randn(shape[1], generator=g, device="cuda"))


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = {"case": case}
    if op in ("route", "back"):
        s["logits"], s["bias"] = _logits(case, g)
        if op == "back":
            s["experts"] = _top(case, s["logits"].float(), s["logits"].float())
            s["dweights"] = torch.randn((case["tokens"], case["top_k"]), generator=g, device="cuda")
    elif op == "dispatch":
        s["experts"] = _experts(case, g)
    elif op == "save":
        wide = torch.zeros((case["rows"], case["cols"] + case["pad"]), dtype=TYPES[case["type"]], device="cuda")
        s["x"] = wide[:, : case["cols"]]
        s["x"].copy_(_rows((case["rows"], case["cols"]), g))
    else:
        e = _experts(case, g).flatten().long()
        e = torch.where(e < 0, case["experts"], e)
        order = torch.sort(e, stable=True).indices
        count = torch.bincount(e, minlength=case["experts"] + 1)[: case["experts"]]
        s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).int()
        s["token_of_slot"] = (order // case["top_k"]).int()
        s["token_of_slot"][int(count.sum()):] = -1
        # the segments' bounds are on the host as well: an all-to-all was
        # issued with them
        s["bounds"] = s["offsets"].tolist()
        s["dy"] = (torch.randn((len(e), case["n"]), generator=g, device="cuda") * 0.02).to(TYPES[case["type"]])
        s["q"], s["exponents"] = _save(_rows((case["tokens"], case["cols"]), g))
    if own:
        _own(s)
    return s


def _own(s):
    """The plan and the handles a user of the framework keeps."""
    from paper_2505_01616_amd import moe

    case = s["case"]
    s["moe"] = moe
    if case["op"] in ("route", "back"):
        s["router"] = moe.Router(experts=case["experts"], top_k=case["top_k"], scores=case["scores"], renormalise=bool(case["renorm"]), groups=case["groups"],
                                 groups_kept=case["kept"], group_best=case["best"], scale=case["scale"])
    if case["op"] == "grad":
        s["saved"] = moe.Saved(s["q"], s["exponents"], case["cols"])


# ---------------------------------------------------------------- the pass
def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state["case"], state)


def _run_own(s):
    case, moe = s["case"], s["moe"]
    if case["op"] == "route":
        return moe.route(s["router"], s["logits"], s["bias"])
    if case["op"] == "back":
        return moe.route_backward(s["router"], s["logits"], s["experts"], s["dweights"])
    if case["op"] == "dispatch":
        d = moe.dispatch(s["experts"], case["experts"], ranks=case["ranks"], row_bytes=ROW_BYTES, once_per_rank=bool(case["once"]))
        return d.offsets, d.token_of_slot, d.slot_of_choice, d.traffic
    if case["op"] == "save":
        return moe.restore(moe.save(s["x"]), s["x"].dtype)
    return moe.weight_grad(s["saved"], s["dy"], s["offsets"], s["token_of_slot"], out_dtype=TYPES[case["out"]])


def _top(case, choice, logits):
    """The top_k experts by `choice`, ties to the lowest, -1 where a row has
    no further expert whose logit is above minus infinity."""
    choice = choice.masked_fill(logits == -math.inf, -math.inf)
    best = torch.sort(choice, dim=1, descending=True, stable=True)
    e = best.indices[:, : case["top_k"]].int()
    return e.masked_fill(best.values[:, : case["top_k"]] == -math.inf, -1)


def _scores(case, x):
    """Scores of a row; 0 where the logit is minus infinity."""
    if case["scores"] == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    top = x.amax(1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    z = p.sum(1, keepdim=True)
    return p / torch.where(z == 0, torch.ones_like(z), z)


def _plain_route(case, s):
    x = s["logits"].float()
    score = _scores(case, x)
    # without a bias and sums of scores the logits give the order
    choice = x if s["bias"] is None and case["best"] == 1 else score if s["bias"] is None else score + s["bias"]
    if case["groups"] > 1:
        of = choice.masked_fill(x == -math.inf, -math.inf).view(len(x), case["groups"], -1)
        of = torch.sort(of, dim=2, descending=True).values[:, :, : case["best"]]
        # an expert that cannot be chosen adds nothing to its group's score
        of = torch.where((of == -math.inf) & (torch.arange(of.shape[2], device=of.device) > 0), torch.zeros_like(of), of).sum(2)
        at = torch.sort(of, dim=1, descending=True, stable=True).indices[:, : case["kept"]]
        use = torch.zeros_like(of, dtype=torch.bool).scatter_(1, at, True)
        choice = choice.masked_fill(~use.repeat_interleave(case["experts"] // case["groups"], 1), -math.inf)
    e = _top(case, choice, x)
    w = torch.gather(score, 1, e.clamp(min=0).long()).masked_fill(e < 0, 0)
    if case["renorm"]:
        z = w.sum(1, keepdim=True)
        w = w / torch.where(z == 0, torch.ones_like(z), z)
    return e, w * case["scale"]


def _plain_back(case, s):
    x, e, dw = s["logits"].float(), s["experts"], s["dweights"]
    score = _scores(case, x)
    at, has = e.clamp(min=0).long(), e >= 0
    dw = torch.where(has, dw, torch.zeros_like(dw)) * case["scale"]
    p = torch.gather(score, 1, at).masked_fill(~has, 0)
    if case["renorm"]:
        z = p.sum(1, keepdim=True)
        z = torch.where(z == 0, torch.ones_like(z), z)
        dp = (dw - (dw * p / z).sum(1, keepdim=True)) / z
    else:
        dp = dw
    ds = torch.zeros_like(score).scatter_add_(1, at, dp.masked_fill(~has, 0))
    if case["scores"] == "sigmoid":
        dx = ds * score * (1 - score)
    else:
        dx = score * (ds - (dp * p).sum(1, keepdim=True))
    return dx.to(s["logits"].dtype)


def _plain_dispatch(case, s):
    T, k, E, R = case["tokens"], case["top_k"], case["experts"], case["ranks"]
    e = s["experts"].flatten().long()
    key = torch.where(e < 0, E, e)
    ordered, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(ordered, torch.arange(E + 1, device=e.device))
    used = ordered < E
    token = torch.where(used, order // k, -1)
    slot = torch.empty_like(order).scatter_(0, order, torch.where(used, torch.arange(T * k, device=e.device), -1))
    to = torch.div(s["experts"], E // R, rounding_mode="floor")  # -1 stays below 0
    count = to >= 0
    if case["once"]:
        for j in range(1, k):
            count[:, j] &= ~(to[:, :j] == to[:, j: j + 1]).any(1)
    frm = torch.arange(T, device=e.device) // (-(-T // R))
    pair = torch.where(count, frm[:, None] * R + to, R * R).flatten().long()
    rows = torch.zeros(R * R + 1, dtype=torch.int64, device=e.device).index_add_(0, pair, torch.ones_like(pair))
    return offsets.int(), token.int(), slot.int().view(T, k), rows[: R * R].view(R, R).double() * ROW_BYTES


def _save(x):
    """x [rows, cols] as 8-bit whole numbers and an exponent per BLOCK
    columns, rows filled with zeros to whole blocks: x is about q 2^e with
    e = floor(log2(largest magnitude)) - 6, at least -126."""
    rows, cols = x.shape
    b = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, b * BLOCK - cols)).view(rows, b, BLOCK)
    e = (torch.frexp(x.abs().amax(2)).exponent - 7).clamp(min=-126)
    q = torch.round(torch.ldexp(x, -e[:, :, None])).clamp(-127, 127)
    return q.to(torch.int8).view(rows, b * BLOCK), e.to(torch.int8)


def _restore(q, e, cols):
    x = torch.ldexp(q.float().view(len(q), -1, BLOCK), e.int()[:, :, None])
    return x.view(len(q), -1)[:, :cols]


def _plain_save(case, s):
    return _restore(*_save(s["x"]), case["cols"]).to(s["x"].dtype)


def _plain_grad(case, s):
    x = _restore(s["q"], s["exponents"], case["cols"])
    dw = torch.zeros((case["experts"], case["n"], case["cols"]), dtype=TYPES[case["out"]], device="cuda")
    for i, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if b > a:
            dw[i] = (s["dy"][a:b].float().t().contiguous() @ x[s["token_of_slot"][a:b].long()]).to(dw.dtype)
    return dw


_PLAIN = {"route": _plain_route, "back": _plain_back, "dispatch": _plain_dispatch, "save": _plain_save, "grad": _plain_grad}


# -------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op in ("route", "back"):
        T, E, k, size = case["tokens"], case["experts"], case["top_k"], SIZE[case["type"]]
        if op == "route":
            return {"bytes": T * E * size + T * k * 8 + (E * 4 if case["bias"] else 0), "flops": 5 * T * E}
        # renormalised scores: only the chosen logits carry a gradient, and
        # only they are read; the zeros are written all the same
        read = k if case["renorm"] or case["scores"] == "sigmoid" else E
        return {"bytes": T * (read + E) * size + T * k * 8, "flops": 5 * T * read}
    if op == "dispatch":
        T, k, E, R = case["tokens"], case["top_k"], case["experts"], case["ranks"]
        return {"bytes": T * k * 12 + (E + 1) * 4 + R * R * 8, "flops": T * k * 2}
    if op == "save":
        # read, saved, read back, written
        v = case["rows"] * case["cols"]
        return {"bytes": v * 2 * SIZE[case["type"]] + 2 * (v + case["rows"] * -(-case["cols"] // BLOCK)), "flops": 4 * v}
    S, T, n, c = case["tokens"] * case["top_k"], case["tokens"], case["n"], case["cols"]
    return {"bytes": S * n * SIZE[case["type"]] + T * (c + -(-c // BLOCK)) + S * 4 + case["experts"] * (n * c * SIZE[case["out"]] + 4), "flops": 2 * S * n * c}


# ------------------------------------------------------------------- exact
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "route":
        return _exact_route(case, s)
    if op == "back":
        return _exact_back(case, s)
    if op == "dispatch":
        return _exact_dispatch(case, s)
    if op == "save":
        x = s["x"].double()
        out = torch.empty_like(x)
        for a in range(0, case["cols"], BLOCK):
            part = x[:, a: a + BLOCK]
            top = part.abs().amax(1, keepdim=True)
            # the power of two at or below `top`, found by comparison
            p = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -140))))
            p = torch.where(p > top, p / 2, torch.where(2 * p <= top, 2 * p, p))
            step = (p / 64).clamp(min=2.0 ** -126)
            out[:, a: a + BLOCK] = torch.round(part / step).clamp(-127, 127) * step
        return out
    x = torch.empty((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda")
    for a in range(0, case["cols"], BLOCK):
        b = min(case["cols"], a + BLOCK)
        x[:, a:b] = s["q"][:, a:b].double() * torch.exp2(s["exponents"][:, a // BLOCK, None].double())
    dw = torch.zeros((case["experts"], case["n"], case["cols"]), dtype=torch.float64, device="cuda")
    for i in range(case["experts"]):
        a, b = s["bounds"][i], s["bounds"][i + 1]
        for c in range(a, b, 8192):
            at = s["token_of_slot"][c: min(b, c + 8192)].long()
            dw[i] += s["dy"][c: c + len(at)].double().t().contiguous() @ x[at]
    return dw


def _exact_scores(case, x):
    if case["scores"] == "sigmoid":
        return torch.where(x >= 0, 1 / (1 + torch.exp(-x.abs())), torch.exp(-x.abs()) / (1 + torch.exp(-x.abs())))
    top = x.amax(1, keepdim=True).clamp(min=-1e300)
    p = torch.exp(x - top)
    return p / p.sum(1, keepdim=True).clamp(min=1e-300)


def _pick(c):
    """(largest of each row, the lowest place that holds it)."""
    top = c.amax(1, keepdim=True)
    place = torch.arange(c.shape[1], device=c.device).expand_as(c)
    return top[:, 0], torch.where(c == top, place, c.shape[1]).amin(1)


def _exact_route(case, s):
    x = s["logits"].double()
    T, E = x.shape
    score = _exact_scores(case, x)
    c = (score if s["bias"] is not None or case["best"] > 1 else x).clone()
    if s["bias"] is not None:
        c += s["bias"].double()
    c[x == -math.inf] = -math.inf
    rows = torch.arange(T, device=x.device)
    if case["groups"] > 1:
        size = E // case["groups"]
        of = torch.full((T, case["groups"]), -math.inf, dtype=torch.float64, device=x.device)
        for i in range(case["groups"]):
            part = c[:, i * size: (i + 1) * size].clone()
            top, at = _pick(part)
            of[:, i] = top
            if case["best"] == 2 and size > 1:
                part[rows, at] = -math.inf
                more = part.amax(1)
                of[:, i] += torch.where(more == -math.inf, 0, more)
        use = torch.zeros((T, case["groups"]), dtype=torch.bool, device=x.device)
        for _ in range(case["kept"]):
            at = _pick(torch.where(use, -math.inf, of))[1]
            at = torch.where(use.gather(1, at[:, None])[:, 0], use.int().argmin(1), at)
            use[rows, at] = True
        c[~use.repeat_interleave(size, 1)] = -math.inf
    e, w = [], []
    for _ in range(case["top_k"]):
        top, at = _pick(c)
        has = top > -math.inf
        e.append(torch.where(has, at, -1))
        w.append(torch.where(has, score[rows, at], 0))
        c[rows, at] = -math.inf
    e, w = torch.stack(e, 1).int(), torch.stack(w, 1)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return e, w * case["scale"]


def _exact_back(case, s):
    """The derivative of sum_j dweights_j weights_j, expert by expert: the
    weights' Jacobian times the scores'."""
    score = _exact_scores(case, s["logits"].double())
    T, k = s["experts"].shape
    at, has = s["experts"].clamp(min=0).long(), (s["experts"] >= 0).double()
    p = score.gather(1, at) * has
    d = s["dweights"].double() * has * case["scale"]
    jac = torch.diag_embed(has)
    if case["renorm"]:
        z = p.sum(1).clamp(min=1e-300)[:, None, None]
        jac = (jac * z - p[:, :, None] * has[:, None, :]) / z ** 2     # [row, weight, chosen score]
    dp = (d[:, :, None] * jac).sum(1)
    if case["scores"] == "sigmoid":
        return torch.zeros_like(score).scatter_add_(1, at, dp * p * (1 - p))
    dx = -score * (dp * p).sum(1, keepdim=True)
    return dx.scatter_add_(1, at, dp * p)


def _exact_dispatch(case, s):
    import numpy as np

    T, k, E, R = case["tokens"], case["top_k"], case["experts"], case["ranks"]
    e = s["experts"].cpu().numpy().astype(np.int64)
    row, col = np.nonzero(e >= 0)
    order = np.lexsort((col, row, e[row, col]))
    token, slot = np.full(T * k, -1), np.full((T, k), -1)
    token[: len(order)] = row[order]
    slot[row[order], col[order]] = np.arange(len(order))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(e[row, col], minlength=E))])
    per, to = -(-T // R), e[row, col] // (E // R)
    sent = np.stack([row, to], 1)
    if case["once"]:
        sent = np.unique(sent, axis=0)
    traffic = np.zeros((R, R))
    np.add.at(traffic, (sent[:, 0] // per, sent[:, 1]), ROW_BYTES)
    return offsets.astype(np.int32), token.astype(np.int32), slot.astype(np.int32), traffic
