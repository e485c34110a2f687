"""What an expert-parallel layer computes between its dispatch and its next
step, as cases to time and compare.

The experts' gated products act(x Wg^T) * (x Wu^T) and their second product,
both with their gradients; the same products with rows and weights in 8-bit
whole numbers, as a layer serves them; and the AdamW step over the layer's
tensors with its moments in 32 or in 8 bits.  With ``own`` set ``run`` makes
the calls a user makes (``paper_2505_01616_amd.moe``); otherwise it computes
the same in elementary torch operations.  ``exact`` computes it in 64 bits.

Experts get rows as in the all-to-all workloads of this repository: an
expert's popularity falls with its rank to the power 1.2 (a seeded order of
the experts), so a few hot ones hold most of them.
"""

from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ZIPF_S = 1.2
BLOCK = 256         # elements of a tensor whose 8-bit moments share a scale
TOP = 448.0         # the largest 8-bit float (4 exponent bits, 3 of mantissa)
TINY = 2.0 ** -100  # magnitudes below count as this (rows) or as zero (moments)
ADAM = dict(lr=1e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def listed():
    return [
        # one token of a generating request on four of 64 experts: the
        # experts' weights are read once, nothing else counts
        _rows("gated_token", "gated", 1, 64, 4, 2048, 2048, "bf16"),
        # a generating batch of 48 requests
        _rows("gated_batch", "gated", 48, 8, 2, 4096, 1024, "f16", act="gelu"),
        # odd sizes throughout, forward and backward, some choices dropped
        _rows("gated_odd", "gated", 3001, 16, 3, 1000, 705, "f16", back=1, empty=0.02, pad=3),
        # a step's experts, forward and backward: hot ones hold most rows
        _rows("gated_step", "gated", 32768, 64, 4, 2048, 2048, "bf16", back=1),
        # a plain layer (one matrix for all rows) of odd sizes
        _rows("down_odd", "product", 777, 1, 1, 1030, 517, "bf16", back=1, by="dense", pad=1),
        # the second product of a step's experts, rows in the order of slots
        _rows("down_step", "product", 32768, 64, 4, 2048, 2048, "bf16", back=1, by="slot"),
        # one token on two of eight experts, weights in 8 bits
        _rows("eight_token", "product8", 1, 8, 2, 4096, 4096, "bf16"),
        # a plain layer of odd sizes in 32 bits
        _rows("eight_odd", "product8", 300, 1, 1, 1000, 705, "f32", by="dense", pad=5),
        # the prompts of a batch
        _rows("eight_prompt", "product8", 8192, 64, 4, 2048, 4096, "bf16", empty=0.01),
        # the small tensors of a model: nothing but latency
        dict(name="adam_small", op="adamw", tensors=60, largest=4096, type="f32", grad="f32", bits=32, master=0),
        # matrices in 16 bits with 32-bit copies, as layers are trained
        dict(name="adam_wide", op="adamw", tensors=12, largest=1 << 26, type="bf16", grad="bf16", bits=32, master=1),
        # the same without copies, moments in 8 bits
        dict(name="adam_eight", op="adamw", tensors=12, largest=(1 << 26) + 77, type="bf16", grad="bf16", bits=8, master=0),
    ]


def _rows(name, op, tokens, experts, top_k, cols, n, type, act="silu", back=0, by="token", pad=0, empty=0.0):
    return dict(name=name, op=op, tokens=tokens, experts=experts, top_k=top_k, cols=cols, n=n, type=type, act=act, back=back, by=by, pad=pad, empty=empty)


def _log(rng, low, high):
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["gated", "gated", "product", "product8", "adamw"])
    if op == "adamw":
        kind = rng.choice(["f32", "bf16", "f16"])
        tensors = _log(rng, 1, 200)
        return dict(op=op, tensors=tensors, largest=_log(rng, 1, (1 << 26) // tensors), type=kind, grad=rng.choice([kind, "f32"]), bits=rng.choice([32, 8]),
                    master=rng.randint(0, 1) if kind != "f32" else 0)
    by = rng.choice(["token", "token", "slot", "dense"])
    experts = 1 if by == "dense" else _log(rng, 1, 64)
    top_k = rng.randint(1, min(4, experts))
    kind = rng.choice(["f32", "bf16", "f16"] if op == "product8" else ["bf16", "f16"])
    case = _rows("", op, _log(rng, 1, 32768), experts, top_k, _log(rng, 16, 2048), _log(rng, 16, 2048), kind, rng.choice(["silu", "gelu"]),
                 0 if op == "product8" else rng.randint(0, 1), by, rng.choice([0, 0, 8, 3]), 0.0 if by == "dense" else rng.choice([0.0, 0.0, 0.03]))
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _plan(case, s, g):
    """The experts' slots, as a dispatch of tokens' choices gives them."""
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    popularity = -ZIPF_S * torch.log(torch.randperm(E, generator=g, device="cuda").float() + 1)
    noise = torch.rand((T, E), generator=g, device="cuda").clamp_(1e-7, 1 - 1e-6)
    e = (popularity - torch.log(-torch.log(noise))).topk(k, 1).indices
    if case["empty"]:
        e[torch.rand((T, k), generator=g, device="cuda") < case["empty"]] = E      # choices that were dropped
    key, order = torch.sort(e.flatten(), stable=True)
    count = torch.bincount(key, minlength=E + 1)[:E]
    s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).int()
    used = key < E
    s["token_of_slot"] = torch.where(used, order // k, -1).int()
    place = torch.where(used, torch.arange(T * k, device="cuda"), -1)
    s["slot_of_choice"] = torch.empty_like(order).scatter_(0, order, place).int().view(T, k)
    # the segments' bounds are on the host as well: an all-to-all was issued
    # with them
    bounds = s["offsets"].tolist()
    s["parts"] = [(i, a, b) for i, (a, b) in enumerate(zip(bounds, bounds[1:])) if b > a]


def _activations(rows, case, g, type):
    """Normal values with columns that stand out, in rows inside wider ones."""
    wide = torch.full((rows, case["cols"] + case["pad"]), 7.0, dtype=type, device="cuda")
    x = wide[:, : case["cols"]]
    x.copy_(torch.randn((rows, case["cols"]), generator=g, device="cuda") * torch.exp(0.5 * torch.randn(case["cols"], generator=g, device="cuda")))
    return x


def _weights(case, g, type):
    shape = (case["experts"], case["n"], case["cols"])
    return (torch.randn(shape, generator=g, device="cuda") * case["cols"] ** -0.5).to(type)


def _prepare_rows(case, g):
    s, type = {"case": case}, TYPES[case["type"]]
    if case["by"] == "dense":
        s["slots"] = case["tokens"]
        s["offsets"], s["parts"] = None, [(0, 0, case["tokens"])]
    else:
        s["slots"] = case["tokens"] * case["top_k"]
        _plan(case, s, g)
    s["x"] = _activations(s["slots"] if case["by"] == "slot" else case["tokens"], case, g, type)
    if case["op"] == "product8":
        w = torch.randn((case["experts"], case["n"], case["cols"]), generator=g, device="cuda") * case["cols"] ** -0.5
        s["w8"] = _quantise(w)
        return s
    s["w"] = [_weights(case, g, type) for _ in range(2 if case["op"] == "gated" else 1)]
    if case["back"]:
        s["dy"] = (torch.randn((s["slots"], case["n"]), generator=g, device="cuda") * 0.05).to(type)
    return s


def _sizes(case):
    """Elements of every tensor: the largest, and others down to one."""
    r = random.Random(case["tensors"] * 1000003 + case["largest"])
    return [case["largest"]] + [_log(r, 1, case["largest"]) for _ in range(case["tensors"] - 1)]


def _prepare_adam(case, g):
    """Tensors, gradients and moments as parts of flat arrays, each tensor from
    a multiple of BLOCK on; what lies between them is zero."""
    s, at = {"case": case, "steps": 10, "spans": []}, 0
    for n in _sizes(case):
        s["spans"].append((at, at + n))
        at += -(-n // BLOCK) * BLOCK
    live = torch.zeros(at, dtype=torch.bool, device="cuda")
    for a, b in s["spans"]:
        live[a:b] = True

    def normal(scale):
        return (torch.randn(at, generator=g, device="cuda") * scale).masked_fill_(~live, 0)

    # gradients of a scaled loss, some of them zero
    spread = torch.exp(torch.randn(at, generator=g, device="cuda"))
    s["g"] = (normal(1.0) * spread * (torch.rand(at, generator=g, device="cuda") > 0.05)).to(TYPES[case["grad"]])
    p = normal(0.05)
    s["p"] = p.to(TYPES[case["type"]])
    s["master"] = s["p"].float() + normal(1e-5) if case["master"] else None
    m = normal(1e-3) * spread
    v = (normal(1e-3) * spread).square() + m.square()
    if case["bits"] == 8:
        s["m"], s["m_scales"] = _encode(m, False)
        s["v"], s["v_scales"] = _encode(v.sqrt(), True)
    else:
        s["m"], s["v"] = m, v
    return s


def prepare(case, seed):
    g = _gen(seed)
    s = _prepare_adam(case, g) if case["op"] == "adamw" else _prepare_rows(case, g)
    if own:
        _own(s)
    return s


def _own(s):
    """The leaves, weights and handles a user of the framework keeps."""
    from paper_2505_01616_amd import moe

    case = s["case"]
    s["moe"] = moe
    if case["op"] == "adamw":
        def moments(a, b):
            if case["bits"] == 32:
                return moe.Moments(s["m"][a:b], s["v"][a:b])
            q = slice(a, a + -(-(b - a) // BLOCK) * BLOCK)
            f = slice(q.start // BLOCK, q.stop // BLOCK)
            return moe.Moments(s["m"][q], s["v"][q], s["m_scales"][f], s["v_scales"][f])

        s["grads"] = [s["g"][a:b] for a, b in s["spans"]]
        s["adam"] = moe.AdamW([s["p"][a:b] for a, b in s["spans"]], bits=case["bits"], steps=s["steps"], moments=[moments(a, b) for a, b in s["spans"]],
                              masters=[s["master"][a:b] for a, b in s["spans"]] if case["master"] else None, **ADAM)
    elif case["op"] == "product8":
        s["weights"] = moe.Rows8(*s["w8"], case["cols"])
    elif case["back"]:
        s["x"].requires_grad_()
        for w in s["w"]:
            w.requires_grad_()


# ---------------------------------------------------------------- the pass
def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state["case"], state)


def _run_own(s):
    case, moe = s["case"], s["moe"]
    if case["op"] == "adamw":
        s["adam"].step(s["grads"], grad_scale=2.0 ** -10)
        return _adam_outputs(s)
    plan = dict(offsets=s["offsets"])
    if case["by"] == "token":
        plan["row_of_slot"] = s["token_of_slot"]
    if case["op"] == "product8":
        return moe.product8(moe.quantise(s["x"]), s["weights"], out_dtype=TYPES[case["type"]], **plan)
    if case["by"] == "token":
        plan["slots_of_row"] = s["slot_of_choice"]
    y = moe.gated(s["x"], *s["w"], activation=case["act"], **plan) if case["op"] == "gated" else moe.product(s["x"], *s["w"], **plan)
    if not case["back"]:
        return y
    return y.detach(), torch.autograd.grad(y, [s["x"], *s["w"]], s["dy"])


def _act(name, g):
    """(act(g), its derivative)."""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _by_slot(case, s, a, b):
    """The rows of slots a .. b."""
    return s["x"][s["token_of_slot"][a:b].long()] if case["by"] == "token" else s["x"][a:b]


def _to_rows(case, s, dx):
    """The rows' gradients from their slots'."""
    if case["by"] == "token":
        at = s["slot_of_choice"].long()
        dx = (dx[at.clamp(min=0)] * (at >= 0)[:, :, None]).sum(1)
    return dx.to(s["x"].dtype)


def _plain_rows(case, s):
    gated, kind = case["op"] == "gated", s["x"].dtype
    y = torch.zeros((s["slots"], case["n"]), dtype=kind, device="cuda")
    if case["back"]:
        dx = torch.zeros((s["slots"], case["cols"]), device="cuda")
        dw = [torch.zeros_like(w) for w in s["w"]]
    for e, a, b in s["parts"]:
        x = _by_slot(case, s, a, b).float()
        w = [v[e].float() for v in s["w"]]
        z = [x @ v.t() for v in w]
        if gated:
            act, slope = _act(case["act"], z[0])
        y[a:b] = act * z[1] if gated else z[0]
        if case["back"]:
            d = s["dy"][a:b].float()
            dz = [d * z[1] * slope, d * act] if gated else [d]
            dx[a:b] = sum(d @ v for d, v in zip(dz, w))
            for i, d in enumerate(dz):
                dw[i][e] = d.t() @ x
    return (y, (_to_rows(case, s, dx), *dw)) if case["back"] else y


def _quantise(x):
    """Rows in whole numbers of 8 bits and a scale for each: x ~ q scale."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    top = torch.where(top < TINY, TINY, top)
    q = torch.round(x * (127.0 / top)).to(torch.int8)
    return torch.nn.functional.pad(q, (0, -x.shape[-1] % 16)), (top / 127.0).squeeze(-1)


def _plain_product8(case, s):
    q, scale = _quantise(s["x"])
    wq, w_scale = s["w8"]
    y = torch.zeros((s["slots"], case["n"]), dtype=s["x"].dtype, device="cuda")
    for e, a, b in s["parts"]:
        at = s["token_of_slot"][a:b].long() if case["by"] == "token" else slice(a, b)
        y[a:b] = (q[at].float() @ wq[e].float().t()) * scale[at][:, None] * w_scale[e]
    return y


def _decode(q, scales):
    return (q.float().view(-1, BLOCK) * scales[:, None]).view(-1)


def _encode(x, positive):
    """Blocks of x in 8-bit floats and a scale for each; positive: what is
    above zero stays above zero."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    top = torch.where(top < TINY, 0.0, top)
    q = (x * torch.where(top > 0, TOP / top, 0.0)).to(torch.float8_e4m3fn)
    if positive:
        lost = (q.view(torch.uint8) == 0) & (x > 0) & (top > 0)
        q = torch.where(lost, 1, q.view(torch.uint8)).view(torch.float8_e4m3fn)
    return q.view(-1), (top / TOP).view(-1)


def _adam_outputs(s):
    names = ["p", "m", "v"] + ["master"] * s["case"]["master"] + ["m_scales", "v_scales"] * (s["case"]["bits"] == 8)
    return {n: s[n] for n in names}


def _plain_adam(case, s):
    s["steps"] += 1
    b1, b2 = ADAM["betas"]
    eight = case["bits"] == 8
    p = s["master"] if case["master"] else s["p"].float()
    g = s["g"].float() * 2.0 ** -10
    m = _decode(s["m"], s["m_scales"]) if eight else s["m"]
    v = _decode(s["v"], s["v_scales"]).square() if eight else s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    r = torch.sqrt(v)
    d = m / (r * (1 - b2 ** s["steps"]) ** -0.5 + ADAM["eps"])
    p = p * (1 - ADAM["lr"] * ADAM["weight_decay"]) - d * (ADAM["lr"] / (1 - b1 ** s["steps"]))
    s["p"].copy_(p)
    if case["master"]:
        s["master"].copy_(p)
    if eight:
        new = _encode(m, False) + _encode(r, True)
        for name, t in zip(("m", "m_scales", "v", "v_scales"), new):
            s[name].copy_(t)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adam_outputs(s)


_PLAIN = {"gated": _plain_rows, "product": _plain_rows, "product8": _plain_product8, "adamw": _plain_adam}


# -------------------------------------------------------------------- work
def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        p = SIZE[case["type"]] + 8 if case["master"] else 2 * SIZE[case["type"]]
        return {"bytes": n * (p + SIZE[case["grad"]] + state), "flops": n * 15}
    T, E, n, c = case["tokens"], case["experts"], case["n"], case["cols"]
    S = T if case["by"] == "dense" else T * case["top_k"]
    rows, used, size = (S if case["by"] == "slot" else T), min(E, S), SIZE[case["type"]]
    if case["op"] == "product8":
        return {"bytes": rows * c * size + used * n * (c + 4) + S * n * size, "flops": 2 * S * n * c}
    matrices = 2 if case["op"] == "gated" else 1
    forward = {"bytes": (rows * c + used * matrices * n * c + S * n) * size, "flops": 2 * S * n * c * matrices}
    if not case["back"]:
        return forward
    # dy read, the gradients of rows and weights written; two products more
    return {"bytes": forward["bytes"] + (S * n + rows * c + E * matrices * n * c) * size, "flops": 3 * forward["flops"]}


# ------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adam(case, s)
    rows, n = s["slots"], case["n"]
    y = torch.zeros((rows, n), dtype=torch.float64, device="cuda")
    if case["op"] == "product8":
        # whole numbers and scales are what their 32-bit definition gives
        x = s["x"].float()
        top = x.abs().max(1).values.clamp(min=TINY)
        q = (x * (127.0 / top).unsqueeze(1)).round().double()
        scale = (top / 127.0).double()
        for e, a, b in s["parts"]:
            at = torch.arange(a, b, device="cuda") if case["by"] != "token" else s["token_of_slot"][a:b].long()
            w = s["w8"][0][e, :, : case["cols"]].double() * s["w8"][1][e].double()[:, None]
            y[a:b] = torch.mm(q[at] * scale[at, None], w.t())
        return y
    with torch.enable_grad():
        x = s["x"].detach().double().requires_grad_()
        w = [v.detach().double().requires_grad_() for v in s["w"]]
        dx, dw = torch.zeros_like(x), [torch.zeros_like(v) for v in w]
        for e, a, b in s["parts"]:
            for a in range(a, b, 16384):
                to = min(a + 16384, b)
                at = torch.arange(a, to, device="cuda") if case["by"] != "token" else s["token_of_slot"][a:to].long()
                mine = [v[e].detach().requires_grad_() for v in w]
                rows = x.detach()[at].requires_grad_()
                z = torch.mm(rows, mine[0].t())
                if case["op"] == "gated":
                    half = torch.erfc(-z / math.sqrt(2)) / 2
                    z = z * (torch.sigmoid(z) if case["act"] == "silu" else half) * torch.mm(rows, mine[1].t())
                y[a:to] = z.detach()
                if case["back"]:
                    got = torch.autograd.grad(z, [rows, *mine], s["dy"][a:to].double())
                    dx.index_add_(0, at, got[0])
                    for i, d in enumerate(got[1:]):
                        dw[i][e] += d
    return (y, (dx.detach(), *(d.detach() for d in dw))) if case["back"] else y


def _exact_adam(case, s):
    t = s["steps"] + 1
    b1, b2 = ADAM["betas"]
    eight = case["bits"] == 8

    def state(q, scales):
        return q.float().double() * scales.double().repeat_interleave(BLOCK) if eight else q.double()

    m = state(s["m"], s.get("m_scales"))
    v = state(s["v"], s.get("v_scales"))
    g = s["g"].double() / 1024
    m = m + (1 - b1) * (g - m)
    v = v ** 2 if eight else v
    v = v + (1 - b2) * (g ** 2 - v)
    p = s["master"].double() if case["master"] else s["p"].double()
    hat = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + ADAM["eps"])
    p = p - ADAM["lr"] * (ADAM["weight_decay"] * p + hat)
    out = {"p": p, "m": m, "v": v}
    if case["master"]:
        out["master"] = p
    if eight:
        for name, x in (("m", m), ("v", v.sqrt())):
            top = x.view(-1, BLOCK).abs().max(1).values
            out[name + "_scales"] = top / TOP
            out[name] = (x.view(-1, BLOCK) / torch.where(top > 0, top / TOP, 1.0)[:, None]).view(-1)
    return out
