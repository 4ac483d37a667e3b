"""GPU parity of layer norm and rotary positions against their plain 64-bit
definitions, through the C ABI.  Tolerances are rounding bounds written beside
each comparison (U = 2^-24, half a step of fp32)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64 as p64
from tests.parity import tdtype, to_dev
from tests.plain64 import HALF, U

pytestmark = pytest.mark.gpu

DT = {"f32": fast.F32, "bf16": fast.BF16}


def rand(shape, dt, seed, offset=0.0, scale=1.0):
    """A device tensor of the storage type and the values it holds, in 64 bits."""
    r = np.random.default_rng(seed)
    t = torch.from_numpy((r.normal(size=shape) * scale + offset).astype(np.float32)).to(tdtype(dt))
    return t.cuda(), t.double().numpy()


def host(t):
    return t.detach().double().cpu().numpy()


def within(x, ref, tol, what):
    x = host(x)
    assert x.shape == ref.shape, what
    bad = ~(np.abs(x - ref) <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.size, float(np.abs(x - ref).max()),
                           [(tuple(i), x[tuple(i)], ref[tuple(i)]) for i in np.argwhere(bad)[:3]])


# ------------------------------------------------------------------ layer norm
def norm_bounds(h, mu, r, gamma, beta, y, dt):
    """A sum of D fp32 terms takes at most 32 additions in a lane and 10 across lanes:
    45 U of the terms' mean magnitude, so 45 U M in the mean, M the largest |h| (3 U for
    rounding h itself); the sum of squares twice the relative error of its terms plus 45 U."""
    M = np.abs(h).max(1, keepdims=True)
    xh = np.abs((h - mu[:, None]) * r[:, None])
    c = 50 * U * M * r[:, None]                  # error of xhat from the mean
    tol = np.abs(gamma) * (c + xh * (c * c + 30 * U)) + 4 * U * (np.abs(y) + np.abs(beta))
    return tol + HALF[dt] * np.abs(y)


SHAPES = [(1, 1), (3, 1), (7, 2), (5, 3), (4, 7), (33, 8), (600, 100), (9, 64), (257, 172), (31, 129),
          (5, 500), (3, 1023), (4, 2048), (3, 2049), (2, 4096), (2, 5001), (2, 8192), (1, 8191)]


@pytest.mark.parametrize("n,D", SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("res", [False, True])
def test_layer_norm_fwd(n, D, dt, res):
    print(f"[layer] norm fwd n={n} D={D} {dt} res={res}", flush=True)
    x, x64 = rand((n, D), dt, 1, offset=0.5)
    r, r64 = rand((n, D), dt, 2) if res else (None, 0.0)
    ga, g64 = rand((D,), "f32", 3)
    be, b64 = rand((D,), "f32", 4)
    y = torch.full((n + 1, D), 7.0, dtype=tdtype(dt), device="cuda")
    h = torch.full((n + 1, D), 7.0, dtype=tdtype(dt), device="cuda") if res else None
    mean, rstd = torch.zeros(2, n + 1, device="cuda").unbind(0)
    fast.fast_layer_norm_fwd(n, D, DT[dt], x, r, ga, be, 1e-5, y, h, mean, rstd)
    h64 = torch.from_numpy(x64 + r64).to(tdtype(dt)).double().numpy()
    ref, mu, rs = p64.layer_norm(h64, g64, b64, 1e-5)
    within(y[:n], ref, norm_bounds(h64, mu, rs, g64, b64, ref, dt), "y")
    M = np.abs(h64).max(1)
    within(mean[:n], mu, 50 * U * M, "mean")
    within(rstd[:n], rs, rs * (40 * U + (50 * U * M * rs) ** 2), "rstd")
    if res:
        np.testing.assert_array_equal(host(h[:n]), h64)
        assert (h[n] == 7).all()
        x2, r2 = x.clone(), r.clone()             # the sum in x's place, y in res's
        fast.fast_layer_norm_fwd(n, D, DT[dt], x2, r2, ga, be, 1e-5, r2, x2)
        assert torch.equal(x2, h[:n]) and torch.equal(r2, y[:n])
    assert (y[n] == 7).all() and float(mean[n]) == 0 and float(rstd[n]) == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_layer_norm_far_from_zero_and_without_weights(dt):
    # rows whose mean is 1000 times their spread; ones and zeros for NULL weights; constant rows
    x, x64 = rand((40, 100), dt, 5, offset=1000.0)
    x[3] = 2.5
    x64[3] = 2.5
    y = torch.empty_like(x)
    fast.fast_layer_norm_fwd(40, 100, DT[dt], x, None, None, None, 1e-5, y)
    ref, mu, rs = p64.layer_norm(x64, 1.0, 0.0, 1e-5)
    within(y, ref, norm_bounds(x64, mu, rs, 1.0, 0.0, ref, dt), "y")
    assert (host(y)[3] == 0).all()
    # in place
    z = x.clone()
    fast.fast_layer_norm_fwd(40, 100, DT[dt], z, None, None, None, 1e-5, z)
    assert torch.equal(z, y)


def test_layer_norm_nonfinite_rows_stay_in_their_row():
    x, x64 = rand((64, 36), "f32", 6)
    x[5, 7] = float("inf")
    x[9, 0] = float("nan")
    y = torch.empty_like(x)
    fast.fast_layer_norm_fwd(64, 36, fast.F32, x, None, None, None, 1e-5, y)
    nan = torch.isnan(y).any(1).cpu().numpy()
    assert nan[5] and nan[9] and nan.sum() == 2


@pytest.mark.parametrize("n,D", SHAPES + [(20000, 36), (70001, 4), (9000, 2), (3000, 500)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("dsum", [False, True])
def test_layer_norm_bwd(n, D, dt, dsum):
    print(f"[layer] norm bwd n={n} D={D} {dt} dsum={dsum}", flush=True)
    h, h64 = rand((n, D), dt, 7, offset=0.3)
    dy, dy64 = rand((n, D), dt, 8)
    ds, ds64 = rand((n, D), dt, 9) if dsum else (None, None)
    ga, g64 = rand((D,), "f32", 10)
    _, mu, rs = p64.layer_norm(h64, g64, 0.0, 1e-2)
    mean, rstd = to_dev(mu.astype(np.float32)), to_dev(rs.astype(np.float32))
    mu, rs = host(mean), host(rstd)               # the inputs, as rounded
    dx = torch.full((n + 1, D), 7.0, dtype=tdtype(dt), device="cuda")
    dg, db = torch.full((2, D + 1), 7.0, device="cuda").unbind(0)
    wsb = fast.fast_layer_norm_bwd_workspace(n, D)
    ws = torch.empty(wsb + 64, dtype=torch.uint8, device="cuda").fill_(0xAB)
    fast.fast_layer_norm_bwd(n, D, DT[dt], h, ga, mean, rstd, dy, ds, dx, dg, db, ws, wsb)
    rx, rg, rb = p64.layer_norm_bwd(h64, g64, mu, rs, dy64, ds64)
    xh = np.abs((h64 - mu[:, None]) * rs[:, None])
    Mr = (np.abs(h64).max(1) + np.abs(mu))[:, None] * rs[:, None]
    g = np.abs(dy64 * g64)
    m1, m2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    tol = U * rs[:, None] * 60 * (g + m1 + (xh + Mr) * (m2 + m1 * Mr)) + 2 * U * np.abs(rx)
    tol = tol + (U * np.abs(ds64) if dsum else 0) + HALF[dt] * np.abs(rx)
    within(dx[:n], rx, tol, "dx")
    # a term carries 4 U Mr |dy| from xhat; at most 32 of them are added in fp32
    within(dg[:D], rg, U * (40 * np.abs(dy64 * xh).sum(0) + 4 * (np.abs(dy64) * Mr).sum(0)) + U * np.abs(rg), "dgamma")
    within(db[:D], rb, U * 33 * np.abs(dy64).sum(0) + U * np.abs(rb), "dbeta")
    assert (dx[n] == 7).all() and float(dg[D]) == 7 and float(db[D]) == 7 and (ws[wsb:] == 0xAB).all()
    # one gradient only, none, and dx in dy's place give the same bits
    dg2, dx2 = torch.empty(D, device="cuda"), dy.clone()
    fast.fast_layer_norm_bwd(n, D, DT[dt], h, ga, mean, rstd, dx2, ds, dx2, dg2, None, ws, wsb)
    assert torch.equal(dg2, dg[:D]) and torch.equal(dx2, dx[:n])
    fast.fast_layer_norm_bwd(n, D, DT[dt], h, ga, mean, rstd, dy, ds, dx2, None, None, None, 0)
    assert torch.equal(dx2, dx[:n])
    if dsum:                                      # dx in dsum's place
        dx3 = ds.clone()
        fast.fast_layer_norm_bwd(n, D, DT[dt], h, ga, mean, rstd, dy, dx3, dx3, None, None, None, 0)
        assert torch.equal(dx3, dx[:n])


@pytest.mark.parametrize("n,D", [(1, 1), (2, 54), (32, 54), (33, 54), (2, 944), (1, 8192), (2, 8192), (3, 8192), (70000, 4)])
def test_layer_norm_bwd_of_one_weight_alone(n, D):
    """Whether one workgroup writes the sums or several have theirs added."""
    h, dy = rand((n, D), "f32", 21)[0], rand((n, D), "f32", 22)[0]
    mean, rstd = h.mean(1), 1 / (h.var(1, unbiased=False) + 1e-3).sqrt()
    dx, wsb = torch.empty_like(h), fast.fast_layer_norm_bwd_workspace(n, D)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    both, one = torch.full((2, 2, D + 1), 7.0, device="cuda").unbind(0)
    args = (n, D, fast.F32, h, None, mean, rstd, dy, None, dx)
    fast.fast_layer_norm_bwd(*args, both[0], both[1], ws, wsb)
    fast.fast_layer_norm_bwd(*args, one[0], None, ws, wsb)
    assert (one[1] == 7).all()
    fast.fast_layer_norm_bwd(*args, None, one[1], ws, wsb)
    assert torch.equal(both, one) and (both[:, D] == 7).all()


def test_layer_norm_bwd_without_rows_zeroes_the_weight_gradients():
    dg, db = torch.full((2, 12), 7.0, device="cuda").unbind(0)
    wsb = fast.fast_layer_norm_bwd_workspace(0, 12)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_layer_norm_bwd(0, 12, fast.F32, None, None, None, None, None, None, None, dg, db, ws, wsb)
    assert (dg == 0).all() and (db == 0).all()


# ------------------------------------------------------------------ rotary
ROT = [  # n, H, dh, pairs, axes
    (1, 1, 2, 1, 1), (3, 1, 3, 1, 2), (600, 2, 50, 25, 1), (65, 2, 50, 24, 3), (77, 4, 32, 16, 1),
    (130, 8, 128, 64, 3), (5, 3, 7, 2, 2), (64, 1, 256, 128, 4), (33, 5, 43, 21, 1), (9, 64, 16, 8, 2),
    (257, 2, 20, 0, 1)]


@pytest.mark.parametrize("n,H,dh,pairs,axes", ROT)
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rotary(n, H, dh, pairs, axes, inter, dt):
    print(f"[layer] rotary n={n} H={H} dh={dh} pairs={pairs} axes={axes} inter={inter} {dt}", flush=True)
    r = np.random.default_rng(n + dh)
    x, x64 = rand((n, H, dh), dt, 11)
    pos = (r.uniform(-1, 1, (n, axes)) * 10.0 ** r.uniform(0, 7, (n, axes))).astype(np.float32)
    ax = r.integers(0, axes, max(pairs, 1)).astype(np.int32)[:pairs]
    om = (10.0 ** r.uniform(-6, 0.3, max(pairs, 1))).astype(np.float32)[:pairs]
    F = H * dh
    dpos, dax, dom = to_dev(pos), to_dev(ax), to_dev(om)

    def bound(ref, sign):
        # sine and cosine within 2e-7, two products and a sum in fp32
        turned = np.abs(p64.rotary(np.abs(x64), np.zeros_like(pos, np.float64), ax, om, pairs, inter))
        a = np.arange(pairs) * (2 if inter else 1)
        b = a + (1 if inter else pairs)
        both = turned.copy()
        both[..., a] = both[..., b] = turned[..., a] + turned[..., b]
        t = both * (2e-7 + 3 * U)
        t[..., 2 * pairs:] = 0
        return t + HALF[dt] * np.abs(ref) * (dt == "bf16")

    for sign, f in ((1.0, fast.fast_rotary_fwd), (-1.0, fast.fast_rotary_bwd)):
        ref = p64.rotary(x64, pos.astype(np.float64), ax, om.astype(np.float64), pairs, inter, sign)
        y = torch.full((n + 1, H, dh), 7.0, dtype=tdtype(dt), device="cuda")
        f(n, H, dh, DT[dt], x, F, dpos, axes, dax, dom, pairs, inter, y, F)
        within(y[:n], ref, bound(ref, sign), "y")
        assert (y[n] == 7).all()
        # the K half of packed rows, in place; V stays as it was
        kv = torch.full((n, 2, H, dh), 3.0, dtype=tdtype(dt), device="cuda")
        kv[:, 0] = x
        f(n, H, dh, DT[dt], kv, 2 * F, dpos, axes, dax, dom, pairs, inter, kv, 2 * F)
        assert torch.equal(kv[:, 0], y[:n]) and (kv[:, 1] == 3).all()
        # from the K half into the V half
        kv[:, 0] = x
        f(n, H, dh, DT[dt], kv, 2 * F, dpos, axes, dax, dom, pairs, inter, kv[:, 1], 2 * F)
        assert torch.equal(kv[:, 0], x) and torch.equal(kv[:, 1], y[:n])


def test_rotary_axis_out_of_range_null_axis_and_infinite_position():
    x, x64 = rand((4, 1, 8), "f32", 12)
    pos = to_dev(np.array([[1.0, 2.0], [3.0, 4.0], [np.inf, 1.0], [0.0, 0.0]], np.float32))
    om = to_dev(np.array([1.0, 0.5, 2.0, 0.0], np.float32))
    y, z, w = torch.empty(3, 4, 1, 8, device="cuda").unbind(0)
    fast.fast_rotary_fwd(4, 1, 8, 0, x, 8, pos, 2, to_dev(np.array([-5, 9, 0, 1], np.int32)), om, 4, 0, y, 8)
    fast.fast_rotary_fwd(4, 1, 8, 0, x, 8, pos, 2, to_dev(np.array([0, 1, 0, 1], np.int32)), om, 4, 0, z, 8)
    assert torch.equal(y.nan_to_num(9), z.nan_to_num(9))
    fast.fast_rotary_fwd(4, 1, 8, 0, x, 8, pos[:, :1].contiguous(), 1, None, om, 4, 0, z, 8)
    fast.fast_rotary_fwd(4, 1, 8, 0, x, 8, pos, 2, to_dev(np.zeros(4, np.int32)), om, 4, 0, w, 8)
    assert torch.equal(z.nan_to_num(9), w.nan_to_num(9))
    assert torch.isnan(z[2, 0, 0]) and not torch.isnan(z[[0, 1, 3]]).any() and torch.equal(z[3], x[3])


@pytest.mark.parametrize("inter", [False, True])
def test_rotary_angles_of_any_size(inter):
    """Sine and cosine within 2e-7 at Unix seconds, nanoseconds and the largest fp32 position."""
    r = np.random.default_rng(5)
    mags = np.repeat([1e8, 1.6e9, 1.6e12, 2e13, 1e15, 1.6e18, 1e25, 3e38], 40)
    pos = (r.uniform(0.5, 1, len(mags)) * mags * r.choice([-1, 1], len(mags))).astype(np.float32)
    om = np.array([1.0, 0.37, 1e-3, 3.0], np.float32)
    n, x = len(pos), torch.zeros(len(pos), 1, 8, device="cuda")
    a = np.arange(4) * (2 if inter else 1)
    b = a + (1 if inter else 4)
    x[..., a] = 1.0                              # (1, 0) turns into (cos, sin)
    y = torch.empty_like(x)
    fast.fast_rotary_fwd(n, 1, 8, 0, x, 8, to_dev(pos[:, None]), 1, None, to_dev(om), 4, int(inter), y, 8)
    th = pos.astype(np.float64)[:, None] * om.astype(np.float64)      # exact: 48 bits
    y = y.cpu().numpy().astype(np.float64)[:, 0]
    for got, f in ((y[:, a], math.cos), (y[:, b], math.sin)):
        ref = np.vectorize(f)(th)
        assert np.abs(got - ref).max() <= 2e-7 + U       # and the product with 1


# ------------------------------------------------------------------ arrays past 2^31 elements
def test_norm_and_rotary_past_two_to_the_31_elements():
    """The first rows, the last ones, and those around element 2^31."""
    n, H, dh = 34_000_000, 2, 32
    D = H * dh
    assert n * D > 1 << 31
    print(f"[layer] {n} x {D} bf16", flush=True)
    torch.manual_seed(1)
    x = torch.randn(n, D, dtype=torch.bfloat16, device="cuda")
    mid = (1 << 31) // D
    rows = torch.tensor([0, 1, mid - 1, mid, mid + 1, n - 2, n - 1], device="cuda")
    x64 = host(x[rows])
    y = torch.empty_like(x)
    mean, rstd = torch.empty(2, n, device="cuda").unbind(0)
    fast.fast_layer_norm_fwd(n, D, fast.BF16, x, None, None, None, 1e-5, y, None, mean, rstd)
    ref, mu, rs = p64.layer_norm(x64, 1.0, 0.0, 1e-5)
    within(y[rows], ref, norm_bounds(x64, mu, rs, 1.0, 0.0, ref, "bf16"), "y")
    dx = torch.empty_like(x)
    dg, db = torch.empty(2, D, device="cuda").unbind(0)
    wsb = fast.fast_layer_norm_bwd_workspace(n, D)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_layer_norm_bwd(n, D, fast.BF16, x, None, mean, rstd, y, None, dx, dg, db, ws, wsb)
    # with dy = y, dx = r (y - xhat) up to terms of eps: 2^-8 |y|, |y| < 6, r < 1.5
    assert float(dx[rows].float().abs().max()) <= 2.0 ** -8 * 10
    total = torch.zeros(D, dtype=torch.float64, device="cuda")
    for a in range(0, n, 1 << 22):
        total += y[a:a + (1 << 22)].double().sum(0)
    # 33 U of each of 32 rows' magnitudes, at most 6 on n rows
    assert (db.double() - total).abs().max() <= 33 * U * 6 * n
    del dx
    pos = torch.full((n, 1), 3.0, device="cuda")
    om = torch.ones(dh // 2, device="cuda")
    fast.fast_rotary_fwd(n, H, dh, fast.BF16, x, D, pos, 1, None, om, dh // 2, 0, y, D)
    ref = p64.rotary(x64.reshape(-1, H, dh), np.full((len(rows), 1), 3.0), np.zeros(dh // 2, int), np.ones(dh // 2),
                     dh // 2, False)
    big = np.abs(x64).max()
    within(y[rows].view(-1, H, dh), ref, 2 * big * (2e-7 + 3 * U) + HALF["bf16"] * np.abs(ref), "turned")


# ------------------------------------------------------------------ streams, graphs, several at once
def test_norm_and_rotary_on_another_stream_and_in_a_graph():
    n, D, H, dh = 3000, 100, 2, 50
    x, _ = rand((n, D), "f32", 13)
    dy, _ = rand((n, D), "f32", 14)
    ga, _ = rand((D,), "f32", 15)
    pos = torch.rand(n, 1, device="cuda") * 1000
    om = torch.rand(25, device="cuda")
    wsb = fast.fast_layer_norm_bwd_workspace(n, D)

    def buffers():
        b = dict(y=torch.zeros(n, D, device="cuda"), z=torch.zeros(n, H, dh, device="cuda"),
                 dx=torch.zeros(n, D, device="cuda"), mean=torch.zeros(n, device="cuda"),
                 rstd=torch.zeros(n, device="cuda"), dg=torch.zeros(D, device="cuda"),
                 db=torch.zeros(D, device="cuda"), ws=torch.zeros(wsb, dtype=torch.uint8, device="cuda"))
        return b

    def step(b, stream=None):
        fast.fast_layer_norm_fwd(n, D, 0, x, None, ga, None, 1e-5, b["y"], None, b["mean"], b["rstd"], stream)
        fast.fast_rotary_fwd(n, H, dh, 0, b["y"], D, pos, 1, None, om, 25, 1, b["z"], D, stream)
        fast.fast_layer_norm_bwd(n, D, 0, x, ga, b["mean"], b["rstd"], dy, None, b["dx"], b["dg"], b["db"],
                                 b["ws"], wsb, stream)

    want = buffers()
    step(want)
    torch.cuda.synchronize()
    names = ("y", "z", "dx", "dg", "db")
    got = buffers()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    step(got, st)
    st.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in names)
    cap = buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cap)
    for k in range(3):
        for b in cap.values():
            b.zero_()
        step(got)                                  # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(cap[m], want[m]) for m in names), k
