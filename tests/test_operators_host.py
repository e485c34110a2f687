"""What the operators refuse, checked on the host: no call here reaches a
device.  (The scalar checks of the C entry points come before any device
work; the tensor checks of moe.py before the C call.)"""

import ctypes

import numpy as np
import pytest

from paper_2505_01616_amd import netsim as ns

P = 1 << 20     # an address that is never followed


def router(**kw):
    base = dict(experts=8, top_k=2, scores=ns.SCORES_SOFTMAX, renormalise=1, groups=1, groups_kept=1, group_best=1,
                scale=1.0)
    base.update(kw)
    return ns.netsim_router(*base.values())


def refused(fn, *args):
    with pytest.raises(ns.NetsimError) as e:
        fn(*args)
    assert e.value.status == ns.E_INVALID
    assert len(ns.netsim_last_error()) > 0
    return str(e.value)


@pytest.mark.parametrize("change", [
    dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=9), dict(experts=64, top_k=33), dict(scores=2),
    dict(renormalise=2), dict(groups=3), dict(groups=0), dict(groups=4, groups_kept=5), dict(groups_kept=0),
    dict(group_best=3), dict(group_best=0), dict(scale=float("nan")), dict(scale=float("inf")),
])
def test_routers(change):
    r = router(**change)
    refused(ns.netsim_route, 0, r, 4, ns.F32, P, 2000, None, P, P)
    refused(ns.netsim_route_backward, 0, r, 4, ns.F32, P, 2000, P, P, P, 2000)


def test_route():
    r = router()
    lib = ns.load_library()
    assert lib.netsim_route(0, None, 4, ns.F32, P, 8, None, P, P, None) == ns.E_INVALID
    refused(ns.netsim_route, -1, r, 4, ns.F32, P, 8, None, P, P)
    refused(ns.netsim_route, 64, r, 4, ns.F32, P, 8, None, P, P)
    refused(ns.netsim_route, 0, r, -1, ns.F32, P, 8, None, P, P)
    refused(ns.netsim_route, 0, r, 1 << 31, ns.F32, P, 8, None, P, P)
    refused(ns.netsim_route, 0, r, 4, 3, P, 8, None, P, P)
    refused(ns.netsim_route, 0, r, 4, ns.F32, P, 7, None, P, P)
    for bad in range(3):
        args = [P, P, P]
        args[bad] = None
        assert "NULL" in refused(ns.netsim_route, 0, r, 4, ns.F32, args[0], 8, None, args[1], args[2])
    assert "aligned" in refused(ns.netsim_route, 0, r, 4, ns.F32, P + 2, 8, None, P, P)
    assert "aligned" in refused(ns.netsim_route, 0, r, 4, ns.BF16, P + 2, 8, P + 2, P, P)
    ns.netsim_route(0, r, 0, ns.F32, None, 8, None, None, None)      # nothing to do is no error


def test_route_backward():
    r = router()
    refused(ns.netsim_route_backward, 0, r, 4, ns.F32, P, 7, P, P, P, 8)
    refused(ns.netsim_route_backward, 0, r, 4, ns.F32, P, 8, P, P, P, 7)
    refused(ns.netsim_route_backward, 0, r, 4, 9, P, 8, P, P, P, 8)
    for bad in range(4):
        args = [P] * 4
        args[bad] = None
        refused(ns.netsim_route_backward, 0, r, 4, ns.F32, args[0], 8, args[1], args[2], args[3], 8)
    ns.netsim_route_backward(0, r, 0, ns.F32, None, 8, None, None, None, 8)


def test_dispatch():
    def call(experts=8, top_k=2, tokens=16, d=P, ranks=4, per=4, row=1.0, once=0, off=P, tok=P, slot=P, traffic=P,
             work=P, size=1 << 40):
        ns.netsim_dispatch(0, experts, top_k, tokens, d, ranks, per, row, once, off, tok, slot, traffic, work, size)

    for bad in (dict(experts=0), dict(experts=1028, ranks=1), dict(top_k=0), dict(top_k=33), dict(tokens=-1),
                dict(tokens=1 << 30, per=1 << 30), dict(ranks=3), dict(ranks=0), dict(per=3), dict(per=0),
                dict(row=-1.0), dict(row=float("inf")), dict(row=float("nan")), dict(once=2), dict(d=None),
                dict(off=None), dict(tok=None), dict(slot=None), dict(work=None), dict(size=0), dict(traffic=P + 4),
                dict(d=P + 1)):
        refused(lambda: call(**bad))
    assert ns.netsim_dispatch_work_bytes(8, 2, 16, 3, 16) == -1
    assert ns.netsim_dispatch_work_bytes(8, 2, 0, 4, 1) == 0
    assert ns.netsim_dispatch_work_bytes(8, 2, 16, 4, 4) > 0


def test_saved_rows():
    for fn in (lambda r, c, t, x, ld, q, e: ns.netsim_act_save(0, r, c, t, x, ld, q, e),
               lambda r, c, t, x, ld, q, e: ns.netsim_act_restore(0, r, c, q, e, t, x, ld)):
        for bad in ((-1, 8, 0, P, 8, P, P), (1, 0, 0, P, 8, P, P), (1, (1 << 20) + 1, 0, P, 1 << 21, P, P),
                    (1, 8, 5, P, 8, P, P), (1, 8, 0, P, 7, P, P), (1, 8, 0, None, 8, P, P), (1, 8, 0, P, 8, None, P),
                    (1, 8, 0, P, 8, P, None), (1, 8, 0, P + 2, 8, P, P), (1, 8, 0, P, 8, P + 8, P)):
            refused(fn, *bad)
        fn(0, 8, 0, None, 8, None, None)


def test_weight_grad():
    base = dict(device=0, experts=4, slots=8, n=16, cols=16, type=ns.BF16, dy=P, ld=16, rows=8, q=P, e=P, row=P, off=P,
                out=ns.F32, dw=P, work=P, size=1 << 40)
    for bad in (dict(device=-1), dict(experts=0), dict(experts=1025), dict(slots=-1), dict(slots=1 << 31), dict(n=0),
                dict(cols=0), dict(n=(1 << 20) + 1, ld=1 << 21), dict(type=4), dict(out=-1), dict(ld=15), dict(rows=-1),
                dict(dy=None), dict(q=None), dict(e=None), dict(off=None), dict(dw=None), dict(dy=P + 1),
                dict(dw=P + 2), dict(q=P + 4), dict(off=P + 2), dict(row=P + 3)):
        refused(ns.netsim_act_weight_grad, *{**base, **bad}.values())
    assert ns.netsim_act_weight_grad_work_bytes(0, 8, 16, 16, ns.BF16) == -1
    assert ns.netsim_act_weight_grad_work_bytes(4, 8, 16, 16, 7) == -1


def test_tensors():
    torch = pytest.importorskip("torch")
    from paper_2505_01616_amd import moe

    with pytest.raises(ValueError):
        moe.Router(8, 2, "relu")
    r = moe.Router(8, 2)
    assert (r.struct.experts, r.struct.top_k, r.struct.renormalise, r.struct.scale) == (8, 2, 1, 1.0)
    with pytest.raises(ValueError):      # on the CPU
        moe.route(r, torch.zeros((4, 8)))
    with pytest.raises(ValueError):
        moe.dispatch(torch.zeros((4, 2), dtype=torch.int32), 8)
    with pytest.raises(ValueError):
        moe.save(torch.zeros((4, 8)))
    with pytest.raises(ValueError):
        moe.restore(moe.Saved(torch.zeros((4, 32), dtype=torch.int8), torch.zeros((4, 1), dtype=torch.int8), 8))


def test_oracle_by_hand():
    """The 64-bit operators on values worked out by hand."""
    from oracle import moe as plain

    class R:
        experts, top_k, scores, renormalise, groups, groups_kept, group_best, scale = 4, 2, "softmax", True, 2, 1, 2, 1.0

    x = np.log(np.array([[1.0, 2.0, 3.0, 2.0]]))
    e, w = plain.route(R, x)                 # groups count 3/8 and 5/8
    assert e.tolist() == [[2, 3]] and np.allclose(w, [[0.6, 0.4]])
    e, w = plain.route(R, x, np.array([1.0, 0, 0, 0]))
    assert e.tolist() == [[0, 1]] and np.allclose(w, [[1 / 3, 2 / 3]])
    q, ex = plain.save(np.array([[127.0, -1.0, 0.5, 128.0]]))
    assert ex.tolist() == [[1]] and q[0, :4].tolist() == [64, 0, 0, 64]
    off, token, slot, bytes_ = plain.dispatch(np.array([[1, 0], [1, -1]]), 2, 2, 1, 3.0, False)
    assert off.tolist() == [0, 1, 3] and token.tolist() == [0, 0, 1, -1]
    assert slot.tolist() == [[1, 0], [2, -1]] and bytes_.tolist() == [[3.0, 3.0], [0.0, 3.0]]


def test_struct_layout():
    assert ctypes.sizeof(ns.netsim_router) == 32
