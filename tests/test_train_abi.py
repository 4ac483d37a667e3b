"""Products, gated recurrence and AdamW without a GPU: refusals before any launch, workspace sizes,
and the plain 64-bit definitions that the GPU tests compare with (gradients against differences,
the random rounding's numbers and their mean)."""
import ctypes

import numpy as np
import pytest

import paper_2607_05095_amd as fast
from tests import plain64_train as p64

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x1000000  # aligned stand-in addresses, never dereferenced on these paths
BIG = 1 << 31


def at(k):
    """an array of its own, 16 MB from its neighbours"""
    return FAKE + (k << 24)


def call(name, defaults, kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return getattr(fast.lib(), name)(*a.values())


# ------------------------------------------------------------------ products
FWD = dict(n=5, K=10, M=6, dt=0, x=at(1), ldx=10, w=at(2), bias=at(3), act=1, res=at(4), ldres=6, y=at(5), ldy=6,
           pre=at(6), st=None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(K=0), INVALID), (dict(M=-2), INVALID), (dict(dt=2), INVALID), (dict(act=4), INVALID),
    (dict(act=0x7ffffff0), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID),
    (dict(ldx=9), INVALID), (dict(ldy=5), INVALID), (dict(ldres=5), INVALID), (dict(act=0), INVALID),
    (dict(K=16385, ldx=16385), UNSUPPORTED), (dict(M=16385, ldy=16385, ldres=16385), UNSUPPORTED),
    (dict(n=BIG), UNSUPPORTED), (dict(ldx=1 << 22), UNSUPPORTED), (dict(ldy=1 << 22), UNSUPPORTED),
    (dict(ldres=1 << 22), UNSUPPORTED), (dict(x=at(1) + 2), UNSUPPORTED), (dict(w=at(2) + 1), UNSUPPORTED),
    (dict(bias=at(3) + 2), UNSUPPORTED), (dict(res=at(4) + 3), UNSUPPORTED), (dict(y=at(5) + 2), UNSUPPORTED),
    (dict(pre=at(6) + 2), UNSUPPORTED), (dict(dt=1, x=at(1) + 1), UNSUPPORTED),
    (dict(n=BIG - 1, K=1, ldx=1, M=16384, ldy=16384, ldres=16384, pre=None), UNSUPPORTED),
    # overlaps: outputs on inputs, on each other, in the gaps of strided rows
    (dict(y=at(1)), INVALID), (dict(y=at(1) + 40), INVALID), (dict(y=at(2) + 8), INVALID), (dict(y=at(3) + 4), INVALID),
    (dict(y=at(4) + 4), INVALID), (dict(y=at(4), ldy=7), INVALID), (dict(pre=at(4)), INVALID), (dict(pre=at(5)), INVALID),
    (dict(pre=at(1)), INVALID), (dict(pre=at(2)), INVALID), (dict(pre=at(3)), INVALID),
    (dict(x=at(1), ldx=40, y=at(1) + 60, ldy=40), INVALID),
    (dict(n=0, x=None, w=None, y=None, res=None, pre=None), OK)])
def test_linear_fwd_refusals(kw, status):
    assert call("fast_linear_fwd", FWD, kw) == status
    assert (fast.fast_last_error() == "") == (status == OK)


BWD = dict(n=5, K=10, M=6, dt=0, x=at(1), ldx=10, w=at(2), act=1, pre=at(3), dy=at(4), lddy=6, dx=at(5), lddx=10, dw=at(6),
           db=at(7), ws=at(8), wsb=1 << 22, st=None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(K=0), INVALID), (dict(M=0), INVALID), (dict(dt=7), INVALID), (dict(act=9), INVALID),
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(pre=None), INVALID), (dict(act=0), INVALID),
    (dict(dy=None), INVALID), (dict(ldx=9), INVALID), (dict(lddy=5), INVALID), (dict(lddx=9), INVALID),
    (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE), (dict(ws=at(8) + 128), UNSUPPORTED),
    (dict(n=BIG), UNSUPPORTED), (dict(lddy=1 << 22), UNSUPPORTED), (dict(lddx=1 << 22), UNSUPPORTED),
    (dict(ldx=1 << 22), UNSUPPORTED), (dict(dy=at(4) + 2), UNSUPPORTED), (dict(dx=at(5) + 1), UNSUPPORTED),
    (dict(dw=at(6) + 2), UNSUPPORTED), (dict(db=at(7) + 1), UNSUPPORTED), (dict(pre=at(3) + 2), UNSUPPORTED),
    (dict(dx=at(4)), INVALID), (dict(dx=at(1)), INVALID), (dict(dx=at(2)), INVALID), (dict(dx=at(3)), INVALID),
    (dict(dw=at(1)), INVALID), (dict(dw=at(5)), INVALID), (dict(db=at(6) + 8), INVALID), (dict(db=at(5)), INVALID),
    (dict(dx=None, dw=None, db=None, ws=None), OK),
    (dict(n=0, dx=None, dw=None, db=None, x=None, w=None, pre=None, dy=None), OK)])
def test_linear_bwd_refusals(kw, status):
    assert call("fast_linear_bwd", BWD, kw) == status
    assert (fast.fast_last_error() == "") == (status == OK)


def test_linear_arrays_that_are_not_read_may_be_missing():
    """x only for dw, w only for dx: what is left is refused for its workspace alone."""
    for kw in (dict(x=None, dw=None), dict(w=None, dx=None), dict(x=None, w=None, dx=None, dw=None)):
        assert call("fast_linear_bwd", BWD, dict(kw, ws=None)) == WORKSPACE


def test_linear_workspace():
    f = fast.fast_linear_bwd_workspace
    for bad in ((-1, 8, 8, 0, 0), (8, 0, 8, 0, 0), (8, 8, 16385, 0, 0), (BIG, 8, 8, 0, 0), (8, 8, 8, 3, 0)):
        assert f(*bad) == 0
    for dt in (0, 1):
        for act in (0, 2):
            for K, M in ((1, 1), (272, 256), (2048, 2048), (16384, 7)):
                sizes = [f(n, K, M, dt, act) for n in (0, 1, 63, 64, 600, 5000, 40000, 264000, 3000000, BIG - 1)]
                assert sizes == sorted(sizes) and sizes[0] > 0 and all(s % 256 == 0 for s in sizes)


def difference(f, x, d, eps=1e-6):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_plain_linear_gradients_are_those_of_differences(kind):
    r = np.random.default_rng(1)
    x, w, b, res, dy = (r.normal(size=s) for s in ((7, 5), (4, 5), (4,), (7, 4), (7, 4)))
    _, z = p64.linear(x, w, b, kind, res)
    z += np.where(np.abs(z) < 1e-3, 1, 0)                      # (not next to relu's kink)
    dx, dw, db, _ = p64.linear_bwd(x, w, kind, z, dy)
    f = lambda x, w, b: (p64.linear(x, w, b, kind, res)[0] * dy).sum()
    for grad, k in ((dx, 0), (dw, 1), (db, 2)):
        d = r.normal(size=grad.shape)
        a = [x, w, b]
        got = difference(lambda v: f(*(v if i == k else a[i] for i in range(3))), a[k], d)
        assert abs(got - (grad * d).sum()) <= 1e-6 * (1 + np.abs(grad * d).sum())


# ------------------------------------------------------------------ recurrence
def graph(N=4, E=200, off=at(20)):
    return ctypes.byref(fast.TCSR(N, E, off, None, None, None, None))


SF = dict(g=None, D=10, dt=0, x=at(1), gate=at(2), ldx=10, span=at(3), h0=at(4), longest=0, h=at(5), last=at(6),
          states=at(7), ws=at(8), wsb=1 << 22, st=None)
SB = dict(g=None, D=10, dt=0, x=at(1), gate=at(2), ldx=10, span=at(3), h0=at(4), longest=0, states=at(7), dh=at(9),
          dlast=at(10), dx=at(11), dgate=at(12), lddx=10, dh0=at(13), ws=at(8), wsb=1 << 22, st=None)
BOTH = [(dict(D=0), INVALID), (dict(dt=2), INVALID), (dict(x=None), INVALID), (dict(gate=None), INVALID),
        (dict(ldx=9), INVALID), (dict(longest=-1), INVALID), (dict(D=8193, ldx=8193, lddx=8193), UNSUPPORTED),
        (dict(ldx=1 << 26), UNSUPPORTED), (dict(x=at(1) + 2), UNSUPPORTED), (dict(gate=at(2) + 1), UNSUPPORTED),
        (dict(span=at(3) + 2), UNSUPPORTED), (dict(h0=at(4) + 1), UNSUPPORTED), (dict(states=at(7) + 2), UNSUPPORTED),
        (dict(ws=None), WORKSPACE), (dict(wsb=16), WORKSPACE), (dict(ws=at(8) + 64), UNSUPPORTED)]


def scan_call(name, defaults, kw, **g):
    a = dict(defaults)
    a.update({k: v for k, v in kw.items() if k in a})
    a["g"] = graph(**g)
    return getattr(fast.lib(), name)(*a.values())


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(h=None, last=None), INVALID), (dict(h=at(5) + 2), UNSUPPORTED), (dict(last=at(6) + 2), UNSUPPORTED),
    (dict(h=at(1)), INVALID), (dict(h=at(2) + 4), INVALID), (dict(h=at(20)), INVALID), (dict(last=at(5) + 40), INVALID),
    (dict(last=at(4) + 40), INVALID), (dict(states=at(1)), INVALID), (dict(states=at(5)), INVALID),
    (dict(states=at(4)), INVALID), (dict(h=at(3)), INVALID)])
def test_gated_scan_fwd_refusals(kw, status):
    assert scan_call("fast_gated_scan_fwd", SF, kw) == status
    assert fast.fast_last_error() != ""


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(lddx=9), INVALID), (dict(lddx=1 << 26), UNSUPPORTED), (dict(states=None), INVALID), (dict(dx=None), INVALID),
    (dict(dgate=None), INVALID), (dict(dh=at(9) + 2), UNSUPPORTED), (dict(dlast=at(10) + 2), UNSUPPORTED),
    (dict(dh0=at(13) + 1), UNSUPPORTED), (dict(dx=at(9)), INVALID), (dict(dx=at(1)), INVALID), (dict(dgate=at(2)), INVALID),
    (dict(dgate=at(11)), INVALID), (dict(dgate=at(11) + 4), INVALID), (dict(dx=at(7)), INVALID),
    (dict(dgate=at(11) + 36, lddx=20), INVALID),               # one element into the other's row
    (dict(dh0=at(10) + 4), INVALID), (dict(dh0=at(11)), INVALID), (dict(dh0=at(4)), INVALID)])
def test_gated_scan_bwd_refusals(kw, status):
    assert scan_call("fast_gated_scan_bwd", SB, kw) == status
    assert fast.fast_last_error() != ""


@pytest.mark.parametrize("name,defaults", [("fast_gated_scan_fwd", SF), ("fast_gated_scan_bwd", SB)])
def test_gated_scan_graphs(name, defaults):
    assert scan_call(name, defaults, {}, N=-1) == INVALID
    assert scan_call(name, defaults, {}, E=-1) == INVALID
    assert scan_call(name, defaults, {}, off=None) == INVALID
    assert scan_call(name, defaults, {}, off=at(20) + 2) == UNSUPPORTED
    assert scan_call(name, defaults, {}, N=BIG) == UNSUPPORTED
    assert scan_call(name, defaults, {}, E=BIG) == UNSUPPORTED
    # launches of 2^32 threads or more
    wide = dict(D=8192, ldx=8192, lddx=8192, h0=None, last=None, dlast=None, dh0=None, wsb=1 << 62)
    assert scan_call(name, defaults, wide, N=1 << 23, off=1 << 50) == UNSUPPORTED
    assert scan_call(name, defaults, dict(ws=None), N=0) == OK
    a = dict(defaults)
    a["g"] = None
    assert getattr(fast.lib(), name)(*a.values()) == INVALID


def test_gated_scan_sizes():
    assert [fast.fast_gated_scan_state_rows(e) for e in (-1, 0, 1, 8, 9, 2400000)] == [0, 0, 1, 1, 2, 300000]
    f = fast.fast_gated_scan_workspace
    assert f(-1, 5, 5) == f(5, BIG, 5) == f(5, 5, 0) == f(5, 5, 8193) == 0
    sizes = [f(7, e, 100) for e in (0, 127, 128, 129, 5000, 10 ** 6, BIG - 1)]
    assert sizes == sorted(sizes) and sizes[1] == 0 and sizes[2] > 0
    assert sizes[5] < 10 ** 6 * 100 * 4 // 20                   # a small share of the rows


def test_plain_scan_gradients_are_those_of_differences():
    r = np.random.default_rng(2)
    off = np.array([0, 3, 3, 8, 9])
    x, g, dh = (r.normal(size=(9, 4)) for _ in range(3))
    h0, dl = r.normal(size=(2, 4, 4))
    dt = r.exponential(size=9)
    dt[4] = 0

    def f(x, g, h0):
        h, last = p64.scan(off, x, g, dt, h0)
        return (h * dh).sum() + (last * dl).sum()
    grads = p64.scan_bwd(off, x, g, dt, h0, dh, dl)
    for k in range(3):
        d = r.normal(size=grads[k].shape)
        a = [x, g, h0]
        got = difference(lambda v: f(*(v if i == k else a[i] for i in range(3))), a[k], d)
        assert abs(got - (grads[k] * d).sum()) <= 1e-7 * (1 + np.abs(grads[k] * d).sum())
    # without times: the sigmoid of the gate
    h, _ = p64.scan(off, x, g, None, h0)
    u = 1 / (1 + np.exp(-g[0]))
    np.testing.assert_allclose(h[0], (1 - u) * h0[0] + u * x[0], rtol=1e-14)


# ------------------------------------------------------------------ AdamW
def tensors(*rows, **kw):
    base = dict(w=at(1), grad=at(2), m=at(3), v=at(4), ms=None, vs=None, copy=at(5), n=100, decay=0.0)
    a = (fast.AdamWTensor * max(len(rows), 1))()
    for j, row in enumerate(rows):
        d = dict(base, **row)
        a[j] = fast.AdamWTensor(*d.values())
    return a


STEP = dict(t=None, count=1, gdt=0, fmt=0, lr=1e-3, b1=.9, b2=.999, eps=1e-8, step=1, seed=0, lrd=None, stepd=None, scale=None,
            st=None)


@pytest.mark.parametrize("row,kw,status", [
    ({}, dict(count=-1), INVALID), ({}, dict(count=1025), UNSUPPORTED), ({}, dict(gdt=2), INVALID), ({}, dict(fmt=2), INVALID),
    ({}, dict(b1=1.0), INVALID), ({}, dict(b2=-.1), INVALID), ({}, dict(b2=float("nan")), INVALID), ({}, dict(eps=-1.0), INVALID),
    ({}, dict(eps=float("inf")), INVALID), ({}, dict(lr=float("nan")), INVALID), ({}, dict(step=0), INVALID),
    ({}, dict(lrd=at(9) + 2), UNSUPPORTED), ({}, dict(stepd=at(9) + 4), UNSUPPORTED), ({}, dict(scale=at(9) + 1), UNSUPPORTED),
    (dict(n=-1), {}, INVALID), (dict(n=1 << 40), {}, UNSUPPORTED), (dict(w=None), {}, INVALID), (dict(grad=None), {}, INVALID),
    (dict(m=None), {}, INVALID), (dict(v=None), {}, INVALID), (dict(decay=float("inf")), {}, INVALID),
    (dict(ms=at(6)), {}, INVALID), (dict(ms=at(6)), dict(fmt=1), INVALID), (dict(w=at(1) + 2), {}, UNSUPPORTED),
    (dict(m=at(3) + 2), {}, UNSUPPORTED), (dict(v=at(4) + 1), {}, UNSUPPORTED), (dict(copy=at(5) + 1), {}, UNSUPPORTED),
    (dict(grad=at(2) + 2), {}, UNSUPPORTED), (dict(grad=at(2) + 1), dict(gdt=1), UNSUPPORTED),
    # arrays that overlap: one tensor's, by a byte, a gradient under a state
    (dict(m=at(1)), {}, INVALID), (dict(v=at(3) + 396), {}, INVALID), (dict(copy=at(1) + 200), {}, INVALID),
    (dict(grad=at(3) + 4), {}, INVALID), (dict(ms=at(6), vs=at(6) + 3), dict(fmt=1), INVALID),
    (dict(ms=at(3) + 99, vs=at(6)), dict(fmt=1), INVALID)])
def test_adamw_refusals(row, kw, status):
    a = dict(STEP, t=tensors(row))
    a.update(kw)
    assert fast.lib().fast_adamw(*a.values()) == status
    assert fast.fast_last_error() != ""


def test_adamw_refuses_a_tensor_twice_and_takes_empty_ones():
    other = dict(w=at(11), grad=at(12), m=at(13), v=at(14), copy=None)
    for rows in (({}, {}), ({}, dict(other, m=at(3))), ({}, dict(other, w=at(5) + 196)), (other, {}, other)):
        a = dict(STEP, t=tensors(*rows), count=len(rows))
        assert fast.lib().fast_adamw(*a.values()) == INVALID
        assert "overlaps" in fast.fast_last_error()
    empty = dict(n=0, w=None, grad=None, m=None, v=None, copy=None)
    assert fast.lib().fast_adamw(*dict(STEP, t=tensors(empty, empty), count=2).values()) == OK
    assert fast.lib().fast_adamw(*dict(STEP, t=None, count=0).values()) == OK
    assert fast.lib().fast_adamw(*dict(STEP, t=None, count=1).values()) == INVALID
    big = dict(n=(1 << 40) - 1, w=1 << 50, grad=1 << 53, m=1 << 54, v=1 << 55, copy=None)
    assert fast.lib().fast_adamw(*dict(STEP, t=tensors(*[dict(big, w=(1 << 50) + (k << 43), m=(1 << 54) + (k << 43),
                                                              v=(1 << 55) + (k << 43), grad=(1 << 53) + (k << 43))
                                                         for k in range(8)]), count=8).values()) == UNSUPPORTED


NORM = dict(t=None, count=1, gdt=0, most=1.0, norm=at(7), scale=at(8), ws=at(9), wsb=1 << 20, st=None)


@pytest.mark.parametrize("row,kw,status", [
    ({}, dict(count=-1), INVALID), ({}, dict(count=1025), UNSUPPORTED), ({}, dict(gdt=3), INVALID), ({}, dict(most=0.0), INVALID),
    ({}, dict(most=float("nan")), INVALID), ({}, dict(norm=None), INVALID), ({}, dict(scale=at(7)), INVALID),
    ({}, dict(norm=at(7) + 2), UNSUPPORTED), ({}, dict(scale=at(8) + 1), UNSUPPORTED), ({}, dict(ws=None), WORKSPACE),
    ({}, dict(wsb=8), WORKSPACE), ({}, dict(ws=at(9) + 4), UNSUPPORTED), (dict(grad=None), {}, INVALID),
    (dict(n=-5), {}, INVALID), (dict(grad=at(2) + 2), {}, UNSUPPORTED)])
def test_grad_norm_refusals(row, kw, status):
    a = dict(NORM, t=tensors(row))
    a.update(kw)
    assert fast.lib().fast_grad_norm(*a.values()) == status


@pytest.mark.parametrize("kw", [dict(lrd=at(1) + 8), dict(stepd=at(3) + 392), dict(scale=at(4)), dict(scale=at(5) + 196)])
def test_adamw_refuses_a_step_s_numbers_among_what_it_writes(kw):
    assert fast.lib().fast_adamw(*{**STEP, "t": tensors({}), **kw}.values()) == INVALID
    assert "overlaps" in fast.fast_last_error()


@pytest.mark.parametrize("kw", [dict(norm=at(2) + 396), dict(scale=at(2)), dict(norm=at(9)), dict(scale=at(9) + 8)])
def test_grad_norm_refuses_results_in_grads_and_workspace(kw):
    assert fast.lib().fast_grad_norm(*{**NORM, "t": tensors({}), **kw}.values()) == INVALID
    assert "lies in" in fast.fast_last_error()


def test_grad_norm_workspace():
    f = fast.fast_grad_norm_workspace
    assert f(-1, 1) == f(5, -1) == f(5, 1025) == 0
    sizes = [f(n, 7) for n in (0, 1, 2047, 2048, 10 ** 5, 1 << 22, (1 << 22) + 1, 10 ** 7, 1 << 24, 10 ** 9)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and f(10 ** 6, 8) >= f(10 ** 6, 7)


def test_adamw_descriptor_has_the_header_s_layout():
    assert ctypes.sizeof(fast.AdamWTensor) == 72
    assert fast.AdamWTensor.n.offset == 56 and fast.AdamWTensor.decay.offset == 64


def test_random_numbers_are_uniform_and_differ_by_tensor_and_step():
    """Sixteen equal cells of each half over 2^16 elements: a cell's count is within 6 standard deviations
    (61 each) of 4096; numbers of neighbouring tensors and steps agree as often as chance has it."""
    n = 1 << 16
    a, b, c = (p64.rounding_bits(7, t, j, n) for t, j in ((1, 0), (1, 1), (2, 0)))
    for r in (a, b, c):
        for half in (r & np.uint64(0xFFFF), r >> np.uint64(16)):
            counts = np.bincount((half >> np.uint64(12)).astype(int), minlength=16)
            assert np.abs(counts - 4096).max() <= 6 * 62
    assert (a >> np.uint64(24) == b >> np.uint64(24)).mean() < 0.006 and (a >> np.uint64(24) == c >> np.uint64(24)).mean() < 0.006


def test_rounding_at_random_keeps_the_mean():
    """Over all 65536 random numbers a value's codes average to it, to a 65536th of their distance."""
    r = np.arange(65536)
    for v in (0.3, 0.99, 1e-3, 5e-4):
        x = np.array([448.0, v])
        got = np.mean([p64.from_codes(*p64.to_codes(x, np.array([0, k]), False))[1] for k in r[::97]])
        step = 2.0 ** max(np.floor(np.log2(v)) - 3, -9)
        assert abs(got - v) <= step * 0.01
    c, s = p64.to_codes(np.array([448.0, 1e-30]), np.array([0, 65535]), True)
    assert p64.from_codes(c, s)[1] == 2.0 ** -9 and p64.from_codes(*p64.to_codes(np.array([448.0, 1e-30]),
                                                                                 np.array([0, 65535]), False))[1] == 0
