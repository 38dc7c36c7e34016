"""Refusals of the routing, dense-product and given-route calls: everything is checked on the host before anything is launched."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def ex():
    from paper_2608_24938_b200 import build
    build.build()
    from paper_2608_24938_b200 import binding
    return binding


P, BIG = 0x10000, 1 << 40  # a fake aligned address, never dereferenced


def test_route_refusals(ex):
    layer = ex.make_layer(64, 0, 64, 64, 6, "f32")

    def route(layer=layer, lg=P, T=4, ids=P, w=P, load=P, router=True, score=1, groups=8, top=4, gs=1, scale=1.0, bias=P):
        r = ex.exfold_router(score, groups, top, gs, 1, scale, bias)
        return ex.lib.exfold_route(C.byref(layer), lg, T, C.byref(r) if router else None, ids, w, load, None)

    before = ex.exfold_launch_count()
    for bad in (dict(lg=None), dict(ids=None), dict(w=None), dict(router=False), dict(T=-1), dict(T=(1 << 24) + 1), dict(score=2),
                dict(score=-1), dict(groups=0), dict(groups=7), dict(groups=64, top=40), dict(top=0), dict(top=9), dict(gs=2),
                dict(groups=32, top=2),  # 4 candidates for 6 slots
                dict(scale=float("inf")), dict(scale=float("nan")), dict(lg=P + 2), dict(ids=P + 1), dict(w=P + 2),
                dict(load=P + 2), dict(bias=P + 2), dict(layer=ex.make_layer(300, 0, 64, 64, 6, "f32")),
                dict(layer=ex.make_layer(64, 0, 64, 64, 33, "f32"))):
        assert route(**bad) == ex.EXFOLD_ERR_INVALID_ARG, bad
    assert route(T=0, lg=None, ids=None, w=None, load=None) == ex.EXFOLD_OK  # nothing to route

    def back(lg=P, ids=P, dw=P, T=4, out=P, score=0, scale=1.0):
        r = ex.exfold_router(score, 1, 1, 0, 1, scale, None)
        return ex.lib.exfold_route_backward(C.byref(layer), lg, ids, dw, T, C.byref(r), out, None)

    for bad in (dict(lg=None), dict(ids=None), dict(dw=None), dict(out=None), dict(T=-1), dict(score=3), dict(scale=float("nan")),
                dict(dw=P + 2), dict(out=P + 2)):
        assert back(**bad) == ex.EXFOLD_ERR_INVALID_ARG, bad
    assert back(T=0, lg=None, ids=None, dw=None, out=None) == ex.EXFOLD_OK
    assert ex.exfold_launch_count() == before


def test_routed_refusals(ex):
    layer = ex.make_layer(8, 0, 128, 256, 2, "f32")
    tabs = ex.exfold_tables(P, P, P, P, None)

    def prefill(x=P, ids=P, w=P, T=4, tables=C.byref(tabs), kp=1, y=P, ws=P, wsb=BIG):
        return ex.lib.exfold_moe_prefill_routed(C.byref(layer), x, ids, w, T, P, P, P, tables, kp, None, y, None, ws, wsb, None)

    def decode(ids=P, w=P, B=4, tables=C.byref(tabs), m=2, ws=P, wsb=BIG):
        return ex.lib.exfold_moe_decode_routed(C.byref(layer), P, ids, w, B, P, P, P, tables, m, P, None, ws, wsb, None)

    before = ex.exfold_launch_count()
    for bad in (dict(x=None), dict(ids=None), dict(w=None), dict(y=None), dict(T=0), dict(kp=0), dict(kp=3), dict(ids=P + 2),
                dict(w=P + 2), dict(tables=None), dict(ws=P + 8)):
        assert prefill(**bad) == ex.EXFOLD_ERR_INVALID_ARG, bad
    assert prefill(wsb=1024) == prefill(wsb=1024, tables=None, kp=2) == ex.EXFOLD_ERR_WORKSPACE_TOO_SMALL
    for bad in (dict(ids=None), dict(w=None), dict(B=0), dict(m=0), dict(m=9), dict(tables=None), dict(ids=P + 1)):
        assert decode(**bad) == ex.EXFOLD_ERR_INVALID_ARG, bad
    assert decode(B=257) == ex.EXFOLD_ERR_UNSUPPORTED
    assert decode(wsb=1024) == ex.EXFOLD_ERR_WORKSPACE_TOO_SMALL
    assert ex.exfold_launch_count() == before


def test_linear_refusals(ex):
    def desc(i=128, o=64, dt=1, out=1, act=0, ldx=0, ldw=0, ldy=0, ldr=0):
        return ex.exfold_linear_desc(i, o, dt, out, act, ldx, ldw, ldy, ldr)

    def linear(x=P, w=P, bias=P, r=P, T=4, y=P, ws=P, wsb=BIG, **kw):
        return ex.lib.exfold_linear(C.byref(desc(**kw)), x, w, bias, r, T, y, ws, wsb, None)

    before = ex.exfold_launch_count()
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ws=None), dict(T=-1), dict(T=(1 << 24) + 1), dict(i=0), dict(o=0),
                dict(i=(1 << 24) + 1), dict(dt=2), dict(out=2), dict(dt=0, out=1), dict(act=5), dict(act=-1), dict(ldx=127),
                dict(ldw=127), dict(ldy=63), dict(ldr=-1), dict(ldr=60), dict(x=P + 1), dict(w=P + 1), dict(bias=P + 1),
                dict(y=P + 1), dict(r=P + 1), dict(out=0, y=P + 2), dict(dt=0, out=0, x=P + 2), dict(ws=P + 128),
                dict(r=P, y=P, ldr=72)):  # in place, but other rows
        assert linear(**bad) == ex.EXFOLD_ERR_INVALID_ARG, bad
    assert linear(wsb=255) == ex.EXFOLD_ERR_WORKSPACE_TOO_SMALL
    assert linear(T=0, x=None, y=None) == ex.EXFOLD_OK
    assert ex.exfold_launch_count() == before
    assert ex.lib.exfold_linear_workspace_bytes(C.byref(desc(i=0)), 4) == 0
    assert ex.lib.exfold_linear_workspace_bytes(C.byref(desc()), -1) == 0
    sizes = [ex.lib.exfold_linear_workspace_bytes(C.byref(desc(i=i, o=o, dt=d, out=d)), t)
             for d in (0, 1) for i, o in ((1, 1), (4096, 4096), (6591, 333)) for t in (0, 1, 16, 300, 8192)]
    assert all(s >= 256 and s % 256 == 0 for s in sizes)


def test_binding_refuses_what_the_call_cannot_see(ex):
    a, w, y = torch.zeros(4, 8), torch.zeros(3, 8), torch.zeros(4, 3)
    ws = torch.zeros(256, dtype=torch.uint8)
    for bad in (dict(x=a.t().contiguous().t()), dict(x=a[:1].expand(4, 8)), dict(w=w.double()), dict(w=torch.zeros(3, 7)),
                dict(y=torch.zeros(5, 3)), dict(residual=torch.zeros(4, 4)), dict(residual=y.bfloat16()), dict(bias=torch.zeros(4))):
        args = dict(x=a, w=w, y=y, ws=ws)
        args.update(bad)
        with pytest.raises(AssertionError):
            ex.exfold_linear(**args)
    layer = ex.make_layer(8, 0, 64, 64, 2, "f32")
    with pytest.raises(AssertionError):  # 64-bit ids
        ex.exfold_route(layer, torch.zeros(4, 8), ex.make_router(), torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2))
    with pytest.raises(AssertionError):
        ex.exfold_route(layer, torch.zeros(4, 9), ex.make_router(), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(AssertionError):  # a bias of another layer
        ex.exfold_route(layer, torch.zeros(4, 8), ex.make_router(bias=torch.zeros(7)), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(AssertionError):
        ex.make_router(bias=torch.zeros(8, dtype=torch.float64))
    with pytest.raises(KeyError):
        ex.make_router("tanh")


def test_linear_workspace_sizes(ex):
    """Room for copies is asked for by what lies oddly, never less for more tokens, and a single row's distance counts nowhere."""
    def size(t, i=4096, o=512, dt=1, ldx=0, ldw=0):
        return ex.lib.exfold_linear_workspace_bytes(C.byref(ex.exfold_linear_desc(i, o, dt, dt, 0, ldx, ldw, 0, 0)), t)

    row = 4096 * 2
    assert size(1) == size(300) == size(1, ldx=4099) == 256 + row and size(300, dt=0) == 256
    assert size(300, ldx=4099) == size(300, ldw=4099) == 256 + 812 * row
    assert size(1, ldw=4099) == 256 + 513 * row
    assert size(300, o=1) == size(300, o=1, ldw=4099) == 256 + 2 * row
    for kw in (dict(), dict(ldx=4097), dict(ldw=4097), dict(i=4095), dict(o=1, ldx=4097), dict(dt=0)):
        sizes = [size(t, **kw) for t in (0, 1, 2, 3, 9, 100)]
        assert sizes == sorted(sizes)
