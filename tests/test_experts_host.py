"""What the products of experts, those in 8 bits and the AdamW step refuse,
checked on the host: no call here reaches a device.  And their 64-bit forms
on values worked out by hand."""

import ctypes

import numpy as np
import pytest

from oracle import experts as plain
from paper_2505_01616_amd import netsim as ns

P = 1 << 20     # an address that is never followed


def refused(fn, *args):
    with pytest.raises(ns.NetsimError) as e:
        fn(*args)
    assert e.value.status == ns.E_INVALID
    assert len(ns.netsim_last_error()) > 0
    return str(e.value)


BASE = dict(device=0, experts=4, slots=8, n=16, cols=16, type=ns.BF16, rows=6, x=P, ld=16, map=P, offsets=P)
BAD = [dict(device=-1), dict(device=64), dict(experts=0), dict(experts=1025), dict(slots=-1), dict(slots=1 << 31), dict(n=0),
       dict(n=(1 << 20) + 1), dict(cols=0), dict(cols=(1 << 20) + 1, ld=1 << 21), dict(type=ns.F32), dict(type=7), dict(rows=-1),
       dict(ld=15), dict(x=None), dict(x=P + 1), dict(map=P + 2), dict(offsets=P + 2), dict(offsets=None), dict(map=None)]


def put(base, after, **kw):
    """base with kw's entries behind its entry `after`."""
    out = {}
    for k, v in base.items():
        out[k] = v
        if k == after:
            out.update(kw)
    return out


def test_products():
    base = {**BASE, "w": P, "y": P, "ld_y": 16}
    for bad in BAD + [dict(w=None), dict(w=P + 1), dict(y=None), dict(y=P + 1), dict(ld_y=15)]:
        refused(ns.netsim_experts_product, *{**base, **bad}.values())
    ns.netsim_experts_product(*{**base, "slots": 0, "rows": 0, "x": None, "map": None, "y": None}.values())
    base = {**put(BASE, "type", act=ns.SILU), "w": P, "w2": P, "y": P, "ld_y": 16, "g": None, "u": None}
    for bad in BAD + [dict(g=P), dict(u=P), dict(g=P + 2, u=P),dict(act=2), dict(act=-1), dict(w=None), dict(w2=None), dict(w2=P + 1), dict(y=None), dict(ld_y=15)]:
        refused(ns.netsim_experts_gated, *{**base, **bad}.values())
    assert "offsets" in refused(ns.netsim_experts_gated, *{**base, "offsets": None}.values())
    assert "list" in refused(ns.netsim_experts_gated, *{**base, "map": None}.values())


def test_products_backward():
    more = dict(dy=P, ld_dy=16, list=P, each=2, dx=P, dw=P, work=P, size=1 << 40)
    bads = BAD + [dict(w=None), dict(dy=None), dict(dy=P + 1), dict(ld_dy=15), dict(list=None), dict(list=P + 2), dict(each=0),
                  dict(dx=P + 1), dict(dw=P + 1), dict(work=P + 8)]
    base = {**BASE, "w": P, **more}
    for bad in bads + [dict(size=-1)]:
        refused(ns.netsim_experts_product_backward, *{**base, **bad}.values())
    assert "workspace" in refused(ns.netsim_experts_product_backward, *{**base, "size": 0}.values())
    base = {**put(BASE, "type", act=ns.GELU), "w": P, "w2": P, "g": P, "u": P, **put(more, "dw", dw2=P)}
    for bad in bads + [dict(g=None), dict(u=None), dict(u=P + 2),dict(act=2), dict(dw2=None), dict(dw=None), dict(dw2=P + 1), dict(size=0), dict(work=None)]:
        refused(ns.netsim_experts_gated_backward, *{**base, **bad}.values())
    size = ns.netsim_experts_backward_work_bytes
    assert size(0, 8, 16, 16, 1, 1) == -1 and size(4, 8, 16, 16, 3, 1) == -1 and size(4, 8, 16, 1 << 21, 1, 1) == -1
    assert size(4, 8, 16, 16, 2, 1) > size(4, 8, 16, 16, 1, 1) > size(4, 8, 16, 16, 1, 0) >= 0 and size(4, 0, 16, 16, 2, 1) >= 0


def test_eight():
    for bad in ((-1, 8, 0, P, 8, P, P), (1, 0, 0, P, 8, P, P), (1, (1 << 17) + 1, 0, P, 1 << 18, P, P), (1, 8, 5, P, 8, P, P),
                (1, 8, 0, P, 7, P, P), (1, 8, 0, None, 8, P, P), (1, 8, 0, P, 8, None, P), (1, 8, 0, P, 8, P, None),
                (1, 8, 0, P + 2, 8, P, P), (1, 8, 0, P, 8, P + 8, P), (1, 8, 0, P, 8, P, P + 2)):
        refused(ns.netsim_rows_quantise, 0, *bad)
    ns.netsim_rows_quantise(0, 0, 8, 0, None, 8, None, None)
    base = dict(device=0, experts=4, slots=8, n=16, cols=16, rows=6, q=P, scales=P, map=P, offsets=P, wq=P, ws=P, out=ns.F32, y=P,
                ld=16)
    for bad in (dict(device=-1), dict(experts=0), dict(experts=1025), dict(slots=-1), dict(slots=1 << 31), dict(n=0), dict(cols=0),
                dict(cols=(1 << 17) + 1), dict(rows=-1), dict(q=None), dict(scales=None), dict(map=None), dict(offsets=None),
                dict(wq=None), dict(ws=None), dict(out=3), dict(y=None), dict(ld=15), dict(q=P + 8), dict(wq=P + 4),
                dict(scales=P + 2), dict(y=P + 2), dict(map=P + 1), dict(offsets=P + 3)):
        refused(ns.netsim_experts_product8, *{**base, **bad}.values())
    ns.netsim_experts_product8(*{**base, "slots": 0, "rows": 0, "map": None, "y": None}.values())


def test_adamw():
    def call(tensor=None, tensors=1, bits=32, step=1, counter=None, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, decay=0.0, scale=1.0, **kw):
        base = dict(p=P, g=P, m=P, v=P, ms=P, vs=P, master=None, size=8, pt=ns.F32, gt=ns.F32)
        t = ns.netsim_adamw_tensor(*{**base, **kw}.values())
        ns.netsim_adamw(0, tensors, ctypes.addressof(t) if tensor is None else tensor, bits, step, counter, lr, b1, b2, eps, decay, scale)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(tensors=-1), dict(tensor=0), dict(bits=16), dict(step=0), dict(counter=P + 4), dict(lr=-1.0), dict(lr=nan),
                dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=0.0), dict(eps=1e-31), dict(eps=inf), dict(eps=nan),
                dict(decay=-1.0), dict(decay=nan), dict(scale=nan), dict(scale=inf), dict(size=-1), dict(pt=3), dict(gt=-1),
                dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p=P + 2), dict(g=P + 2), dict(m=P + 2), dict(master=P),
                dict(pt=ns.BF16, p=P + 1), dict(pt=ns.BF16, master=P + 2), dict(bits=8, ms=None), dict(bits=8, vs=None),
                dict(bits=8, m=P + 4), dict(bits=8, vs=P + 2)):
        refused(lambda: call(**bad))
    call(tensors=0, tensor=0)
    call(size=0, p=None, g=None, m=None, v=None)


def test_tensors():
    torch = pytest.importorskip("torch")
    from paper_2505_01616_amd import moe

    x, w = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((1, 4, 8), dtype=torch.bfloat16)
    for call in (lambda: moe.gated(x, w, w), lambda: moe.product(x, w), lambda: moe.quantise(x),
                 lambda: moe.product8(moe.Rows8(torch.zeros((4, 16), dtype=torch.int8), torch.zeros(4), 8),
                                      moe.Rows8(torch.zeros((4, 16), dtype=torch.int8), torch.zeros(4), 8)),
                 lambda: moe.AdamW([torch.zeros(4)])):
        with pytest.raises(ValueError):      # on the CPU
            call()
    with pytest.raises(ValueError, match="activation"):
        moe.gated(x, w, w, activation="relu")
    with pytest.raises(ValueError):
        moe.AdamW([], bits=16)
    assert moe._TENSOR.itemsize == ctypes.sizeof(ns.netsim_adamw_tensor) == 72


def test_oracle_by_hand():
    x = np.array([[1.0, 2.0], [3.0, -1.0], [9.0, 9.0]])
    w = np.array([[[1.0, 0.0]], [[0.0, 2.0]]])
    offsets, row = [0, 1, 3], [1, 0, 7]      # the last slot has no row
    z, top, y = plain.multiply(x, [w], offsets, row)
    assert y.tolist() == [[3.0], [4.0], [0.0]] and top[0].tolist() == [[3.0], [4.0], [0.0]]
    dx, dw = plain.gradients(x, [w], [np.array([[2.0], [5.0], [100.0]])], offsets, row, [[1, -1], [0, -1], [-1, -1]])
    assert dx.tolist() == [[0.0, 10.0], [2.0, 0.0], [0.0, 0.0]] and dw[0].tolist() == [[[6.0, -2.0]], [[5.0, 10.0]]]
    assert plain.used([1, 2, 2], 2, [0, 3, 0], 3, 3).tolist() == [False, False, False]
    a, s = plain.activation("silu", np.array([0.0, 100.0]))
    assert a.tolist() == [0.0, 100.0] and s.tolist() == [0.5, 1.0]
    a, s = plain.activation("gelu", np.array([0.0]))
    assert a.tolist() == [0.0] and s.tolist() == [0.5]
    q, scale = plain.quantise(np.array([[2.0, -1.0, 0.0]]))
    assert q.tolist() == [[127, -64, 0]] and scale[0] == np.float32(2) / np.float32(127)
    assert plain.FLOAT8[[0, 1, 8, 56, 126, 184]].tolist() == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -1.0]
    p, m, v = plain.adamw(np.array([1.0]), np.array([2.0]), np.zeros(1), np.zeros(1), 1, 0.5, 0.9, 0.99, 1e-12, 0.1)
    assert np.allclose([p[0], m[0], v[0]], [1 - 0.05 - 0.5, 0.2, 0.04])
