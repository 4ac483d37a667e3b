"""GPU parity of the ways that a call of the layer operators is carried out at sizes where another
kernel takes over: streamed rows, workgroup-owned segments with pieces behind them, caches past
4 GiB.  The ways' own sizes are checked against the rules that choose them."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64 as p64
from tests.parity import tdtype, to_dev
from tests.plain64 import HALF, U
from tests.test_gpu_cache_rows import Block

pytestmark = pytest.mark.gpu

DT = {"f32": fast.F32, "bf16": fast.BF16}
FMT = {8: fast.MXFP8, 4: fast.MXFP4}
LAST_LEVEL = 256 << 20                          # bytes past which rows are streamed


def host(t):
    return t.detach().double().cpu().numpy()


def some_rows(n, seed):
    r = np.random.default_rng(seed)
    return torch.from_numpy(np.unique(np.concatenate([[0, 1, n - 2, n - 1], r.integers(0, n, 60)]))).cuda()


# ------------------------------------------------------------------ attention
def counts_about(N, E, long, seed):
    """N segments of E edges in all: the lengths `long`, empty ones, the rest about the mean."""
    r = np.random.default_rng(seed)
    c = np.zeros(N, np.int64)
    at = r.choice(N, len(long), replace=False)
    c[at] = long
    rest = np.setdiff1d(np.arange(N), at)[3:]
    left = E - c.sum()
    c[rest] = left // len(rest)
    move = r.integers(-(left // len(rest) // 2), left // len(rest) // 2, len(rest) // 2)
    c[rest[:len(move)]] += move
    c[rest[-len(move):]] -= move
    c[rest[0]] += E - c.sum()
    assert c.sum() == E and (c >= 0).all()
    return c


@pytest.mark.parametrize("N,E,cut,H,dh", [
    (300, 30000, 256, 2, 50), (300, 30000, 256, 8, 128), (300, 30000, 256, 3, 7), (300, 30000, 256, 16, 9),
    (300, 30000, 256, 2, 33), (70, 5000, 64, 20, 50), (100, 9000, 256, 1, 256), (1000, 500000, 1024, 4, 32),
    (300, 570000, 4096, 2, 50)])
@pytest.mark.parametrize("fmt", [8, 4])
def test_a_workgroup_per_segment_with_pieces_behind(N, E, cut, H, dh, fmt):
    """64 to 2048 segments of 64 edges or more: lengths about the cut, whole ones and long ones."""
    print(f"[routes] attention N={N} E={E} H={H} dh={dh} fmt={fmt}", flush=True)
    assert 64 <= N <= 2048 and E // N >= 64
    long = [cut - 1, cut, cut + 1, cut + 2, 2 * cut - 1, 2 * cut, 2 * cut + 1, 5 * cut + 3, 1, 2]
    b = Block(counts_about(N, E, long, N + dh), H, dh, fmt, "f32" if (H + fmt) % 3 else "bf16", seed=E + H)
    b.check(*b.run())


@pytest.mark.parametrize("counts", [
    [3, 0, 70, 9, 1] * 30, [0, 1, 64, 65, 3, 3000], [2] * 4500 + [300, 0, 70], [100] * 90 + [255, 256, 257, 900]],
    ids=["waves", "few", "lanes", "workgroups"])
@pytest.mark.parametrize("H,dh,fmt", [(2, 50, 8), (4, 32, 4), (2, 33, 8), (8, 128, 4), (1, 200, 8), (16, 9, 8)])
def test_cached_attention_past_four_gib(counts, H, dh, fmt):
    """The block on a cache of more than 4 GiB, its rows spread over all of it."""
    print(f"[routes] attention, large cache, N={len(counts)} H={H} dh={dh} fmt={fmt}", flush=True)
    b = Block(counts, H, dh, fmt, "f32", seed=dh)
    stride = b.cache.shape[1]
    rows = (9 << 29) // stride + 1                  # 4.5 GiB
    at = np.linspace(0, rows - 1, b.rows).astype(np.int64)
    assert at[-1] * stride > 1 << 32
    out, lse, ws, wsb, g, ids, _ = b.buffers()
    small, smap = b.cache, np.where((b.smap >= 0) & (b.smap < b.rows), at[np.clip(b.smap, 0, b.rows - 1)], -1)
    cache = torch.empty(rows, stride, dtype=torch.uint8, device="cuda")
    cache[to_dev(at)] = small
    fast.fast_edge_attention_fwd_cached(g, H, dh, DT[b.dt], b.Q, ids, b.bound, to_dev(smap.astype(np.int32)), FMT[fmt],
                                        cache, rows, b.scale, b.slope, out, lse, ws, wsb)
    b.check(out, lse)


def test_slots_named_by_the_ids_themselves():
    """Without a map an id is its record's place."""
    for counts in ([3, 0, 70, 9, 1] * 30, [0, 1, 64, 65, 3, 3000], [2] * 4500 + [300, 0, 70]):
        b = Block(counts, 2, 50, 8, "f32", seed=len(counts))
        b.ids = np.random.default_rng(1).integers(-2, b.rows + 2, b.E)
        b.bound, b.smap = b.rows + 1, np.append(np.arange(b.rows), -1).astype(np.int32)
        out, lse, ws, wsb, g, ids, _ = b.buffers()
        fast.fast_edge_attention_fwd_cached(g, 2, 50, 0, b.Q, ids, b.bound, None, fast.MXFP8, b.cache, b.rows, b.scale,
                                            b.slope, out, lse, ws, wsb)
        b.check(out, lse)


BLOCKS = {"waves": [3, 0, 70, 9, 1] * 30, "few": [0, 1, 64, 65, 3, 3000], "lanes": [2] * 4500 + [300, 0, 70],
          "workgroups": [100] * 90 + [255, 256, 257, 900]}


@pytest.mark.parametrize("H,dh", [(2, 50), (8, 128)])
def test_a_workspace_left_by_other_blocks(H, dh):
    """One workspace for the largest block, never cleared, whatever block used it before."""
    blocks = [Block(c, H, dh, 8, "f32", seed=k) for k, c in enumerate(BLOCKS.values())]
    N, E = max(b.N for b in blocks), max(b.E for b in blocks)
    wsb = fast.fast_edge_attention_cached_workspace(N, E, H, dh)
    ws = torch.zeros(wsb, dtype=torch.uint8, device="cuda")
    for b in blocks + blocks[::-1]:
        out, lse, _, _, g, ids, smap = b.buffers()
        b.check(*b.run(bufs=(out, lse, ws, wsb, g, ids, smap)))


@pytest.mark.parametrize("name", list(BLOCKS))
@pytest.mark.parametrize("H,dh", [(2, 50), (8, 128)])
def test_malformed_offsets_write_nothing_else(name, H, dh):
    """Offsets that decrease, are negative or past the last edge are clamped: the results say nothing, but only
    they and the workspace are written, and the next call finds all it needs."""
    print(f"[routes] malformed offsets {name} H={H} dh={dh}", flush=True)
    b = Block(BLOCKS[name], H, dh, 8, "f32", seed=5)
    guard = 4096
    wsb = fast.fast_edge_attention_cached_workspace(b.N, b.E, H, dh)
    r = np.random.default_rng(H)
    for kind in range(4):
        off = b.off.copy()
        at = r.choice(b.N + 1, max(b.N // 3, 2), replace=False)
        if kind == 0:
            off[at] = r.integers(-2 ** 31, 2 ** 31, len(at))
        elif kind == 1:
            off = off[::-1].copy()
        elif kind == 2:
            off[:] = r.integers(0, b.E + 1, len(off))
        else:
            off[1::2] = 2 ** 31 - 1
        ws = torch.full((wsb + guard,), kind, dtype=torch.uint8, device="cuda")
        ws[wsb:] = 0xA5
        bufs = b.buffers()
        fast.fast_edge_attention_fwd_cached(fast.tcsr(to_dev(off.astype(np.int32)), b.E), H, dh, 0, b.Q, bufs[5], b.bound,
                                            bufs[6], fast.MXFP8, b.cache, b.rows, b.scale, b.slope, bufs[0], bufs[1],
                                            ws, wsb)
        assert (bufs[0][b.N] == 7).all() and (bufs[1][b.N] == 7).all() and (ws[wsb:] == 0xA5).all()
        b.check(*b.run(bufs=(bufs[0], bufs[1], ws, wsb) + bufs[4:]))


# ------------------------------------------------------------------ cached rows
def test_cached_rows_past_two_to_the_31_elements():
    """Rows written from and read to arrays of more than 2^31 elements."""
    n, width, rows = 13_000_000, 172, 3_000_000
    assert n * width > 1 << 31
    print(f"[routes] cache write and gather {n} x {width} bf16", flush=True)
    torch.manual_seed(4)
    src = torch.randn(n, 1, width, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(n, device="cuda") % (rows + 7)            # seven without a row; the last of a slot stays
    stride = fast.fast_cache_row_bytes(1, width, fast.MXFP4)
    cache = torch.zeros(rows, stride, dtype=torch.uint8, device="cuda")
    wsb = fast.fast_cache_write_workspace(n, rows)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_cache_write(ids, n, rows, None, 1, width, fast.BF16, src, fast.MXFP4, cache, rows, False, ws, wsb)
    at = some_rows(rows, 7)
    last = (n - 1 - at) // (rows + 7) * (rows + 7) + at
    assert int(last.max()) * width > 1 << 31
    c, s = p64.quantize(host(src[last]), 4)
    np.testing.assert_array_equal(cache[at].cpu().numpy(), p64.pack(c, s, 4))
    src.fill_(7.0)
    fast.fast_cache_gather(ids, n, rows, None, 1, width, fast.MXFP4, cache, rows, fast.BF16, src)
    np.testing.assert_array_equal(host(src[at]), p64.values(c, s, 4))
    np.testing.assert_array_equal(host(src[last]), p64.values(c, s, 4))
    assert (src[rows:rows + 7] == 7).all()


@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("width", [172, 43])
def test_reads_past_64_mib(width, fmt, dt):
    """Streamed results: those of reads in small portions, and some rows' definition."""
    es = 4 if dt == "f32" else 2
    n = (70 << 20) // (width * es)
    print(f"[routes] gather n={n} width={width} fmt={fmt} {dt}", flush=True)
    rows, bound = 5000, 6000
    r = np.random.default_rng(width)
    smap = np.full(bound, -1, np.int32)
    smap[r.choice(bound, rows, replace=False)] = np.arange(rows)
    c, s = p64.quantize(r.normal(size=(rows, 1, width)) * 2.0 ** r.integers(-9, 9, (rows, 1, 1)), fmt)
    cache, dmap = to_dev(p64.pack(c, s, fmt)), to_dev(smap)
    ids_np = r.integers(-5, bound + 5, n)
    ids = to_dev(ids_np)
    big = torch.full((n, 1, width), 7.0, dtype=tdtype(dt), device="cuda")
    fast.fast_cache_gather(ids, n, bound, dmap, 1, width, FMT[fmt], cache, rows, DT[dt], big)
    part = torch.full_like(big, 7.0)
    for a in range(0, n, n // 3 + 1):
        m = min(n - a, n // 3 + 1)
        fast.fast_cache_gather(ids[a:a + m], m, bound, dmap, 1, width, FMT[fmt], cache, rows, DT[dt], part[a:a + m])
    assert torch.equal(big, part)
    at = some_rows(n, 3)
    slot = p64.slots(ids_np, bound, smap, rows)[at.cpu().numpy()]
    want = torch.from_numpy(p64.values(c, s, fmt)[np.maximum(slot, 0)]).to(tdtype(dt)).double().numpy()
    want[slot < 0] = 7
    np.testing.assert_array_equal(host(big[at]), want)


# ------------------------------------------------------------------ rotary
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("dh,pairs", [(32, 16), (64, 20)])
def test_rotary_of_streamed_rows(dt, dh, pairs):
    """Pairs side by side, rows of whole lines, rows and results past the last-level cache: the
    results of small portions, some rows' definition, and in place (where nothing is copied)."""
    H, es = 4, 4 if dt == "f32" else 2
    F = H * dh
    n = LAST_LEVEL // (2 * F * es) + 300
    print(f"[routes] rotary n={n} {dt} dh={dh}", flush=True)
    torch.manual_seed(3)
    x = torch.randn(n, H, dh, device="cuda").to(tdtype(dt))
    pos = torch.rand(n, 2, device="cuda") * 1e6
    om = torch.pow(10.0, -5 * torch.rand(pairs, device="cuda"))
    ax = (torch.arange(pairs, device="cuda") % 2).int()
    assert F * es % 128 == 0 and 2 * n * F * es > LAST_LEVEL
    for f, sign in ((fast.fast_rotary_fwd, 1.0), (fast.fast_rotary_bwd, -1.0)):
        y, part = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        f(n, H, dh, DT[dt], x, F, pos, 2, ax, om, pairs, 1, y, F)
        for a in range(0, n, n // 3 + 1):
            m = min(n - a, n // 3 + 1)
            f(m, H, dh, DT[dt], x[a:a + m], F, pos[a:a + m], 2, ax, om, pairs, 1, part[a:a + m], F)
        assert torch.equal(y, part)
        at = some_rows(n, 4)
        x64 = host(x[at])
        ref = p64.rotary(x64, host(pos[at]), ax.cpu().numpy(), host(om), pairs, True, sign)
        # sine and cosine within 2e-7, two products and a sum in fp32, of at most twice the largest |x|
        assert (np.abs(host(y[at]) - ref) <= 2 * np.abs(x64).max() * (2e-7 + 3 * U) + HALF[dt] * np.abs(ref)).all()
        part.copy_(x)
        f(n, H, dh, DT[dt], part, F, pos, 2, ax, om, pairs, 1, part, F)
        assert torch.equal(y, part)


# ------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("dt,D", [("f32", 512), ("bf16", 512), ("f32", 64), ("bf16", 2048)])
def test_norm_of_streamed_rows(dt, D):
    """Both directions past the last-level cache: rows as in small portions and, in some, as
    defined; the weights' gradients as defined."""
    es = 4 if dt == "f32" else 2
    n = LAST_LEVEL // (3 * D * es) + 77             # the fewest arrays that a pass here moves: 3
    print(f"[routes] norm n={n} D={D} {dt}", flush=True)
    assert D * es % 128 == 0 and 3 * n * D * es > LAST_LEVEL
    torch.manual_seed(5)
    x, r, dy, ds = (torch.randn(n, D, device="cuda").to(tdtype(dt)) for _ in range(4))
    ga, be = torch.randn(2, D, device="cuda").unbind(0)

    def pieces():
        return ((a, min(n - a, n // 5 + 1)) for a in range(0, n, n // 5 + 1))
    y, h, y2, h2 = (torch.full_like(x, 7.0) for _ in range(4))
    mean, rstd, mean2, rstd2 = torch.zeros(4, n, device="cuda").unbind(0)
    fast.fast_layer_norm_fwd(n, D, DT[dt], x, r, ga, be, 1e-5, y, h, mean, rstd)
    for a, m in pieces():
        k = slice(a, a + m)
        fast.fast_layer_norm_fwd(m, D, DT[dt], x[k], r[k], ga, be, 1e-5, y2[k], h2[k], mean2[k], rstd2[k])
    assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    at = some_rows(n, 6)
    h64, g64, b64 = host((x[at].float() + r[at].float()).to(tdtype(dt))), host(ga), host(be)
    np.testing.assert_array_equal(host(h[at]), h64)
    ref, mu, rs = p64.layer_norm(h64, g64, b64, 1e-5)
    # 50 U of the largest |h| in the mean; the squares' sum twice that in its terms and 45 U (see test_gpu_layer.py)
    M, xh = np.abs(h64).max(1, keepdims=True), np.abs(h64 - mu[:, None]) * rs[:, None]
    c = 50 * U * M * rs[:, None]
    tol = np.abs(g64) * (c + xh * (c * c + 30 * U)) + 4 * U * (np.abs(ref) + np.abs(b64)) + HALF[dt] * np.abs(ref)
    assert (np.abs(host(y[at]) - ref) <= tol).all()
    y.copy_(x)                                      # y in x's place, the sum in res's
    h.copy_(r)
    fast.fast_layer_norm_fwd(n, D, DT[dt], y, h, ga, be, 1e-5, y, h)
    assert torch.equal(y, y2) and torch.equal(h, h2)

    dx, dx2 = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    dg, db = torch.zeros(2, D, device="cuda").unbind(0)
    wsb = fast.fast_layer_norm_bwd_workspace(n, D)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_layer_norm_bwd(n, D, DT[dt], h, ga, mean, rstd, dy, ds, dx, dg, db, ws, wsb)
    for a, m in pieces():
        k = slice(a, a + m)
        fast.fast_layer_norm_bwd(m, D, DT[dt], h[k], ga, mean[k], rstd[k], dy[k], ds[k], dx2[k], None, None, None, 0)
    assert torch.equal(dx, dx2)
    # the definition at the rounded statistics that the call is given
    mu, rs, dy64 = host(mean[at]), host(rstd[at]), host(dy[at])
    rx, _, _ = p64.layer_norm_bwd(h64, g64, mu, rs, dy64, host(ds[at]))
    xh = np.abs((h64 - mu[:, None]) * rs[:, None])
    Mr = (np.abs(h64).max(1) + np.abs(mu))[:, None] * rs[:, None]
    g = np.abs(dy64 * g64)
    m1, m2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    tol = U * rs[:, None] * 60 * (g + m1 + (xh + Mr) * (m2 + m1 * Mr)) + 2 * U * np.abs(rx) + U * np.abs(host(ds[at]))
    assert (np.abs(host(dx[at]) - rx) <= tol + HALF[dt] * np.abs(rx)).all()
    check_weight_gradients(h, dy, mean, rstd, dg, db)


def check_weight_gradients(h, dy, mean, rstd, dg, db):
    """dgamma and dbeta against 64-bit sums of all rows.  A term of dgamma carries 4 U (|h| + |mu|) r |dy| from
    xhat; at most 32 terms are added in fp32, then a workgroup's and the last sum rounded once each."""
    D = h.shape[1]
    g, ga, gt, b, ba = torch.zeros(5, D, dtype=torch.float64, device="cuda").unbind(0)
    for k in torch.arange(h.shape[0], device="cuda").split(1 << 20):
        k = slice(int(k[0]), int(k[-1]) + 1)
        hk, dk, mu, rs = h[k].double(), dy[k].double(), mean[k].double()[:, None], rstd[k].double()[:, None]
        t = dk * (hk - mu) * rs
        g += t.sum(0)
        ga += t.abs().sum(0)
        gt += (dk.abs() * (hk.abs() + mu.abs()) * rs).sum(0)
        b += dk.sum(0)
        ba += dk.abs().sum(0)
    assert ((dg.double() - g).abs() <= U * (40 * ga + 4 * gt + g.abs())).all()
    assert ((db.double() - b).abs() <= U * (33 * ba + b.abs())).all()


def test_norm_backward_past_two_to_the_31_elements():
    """Every sampled row of dx is written with its own gradient, and the weights' gradients hold all rows."""
    n, D = 34_000_000, 64
    assert n * D > 1 << 31
    print(f"[routes] norm backward {n} x {D} bf16", flush=True)
    torch.manual_seed(2)
    h = torch.randn(n, D, dtype=torch.bfloat16, device="cuda")
    dy = torch.randn(n, D, dtype=torch.bfloat16, device="cuda")
    mean = torch.randn(n, device="cuda") * 0.1
    rstd = torch.rand(n, device="cuda") + 0.5
    ga = torch.randn(D, device="cuda")
    dx = torch.full_like(h, 768.0)
    dg, db = torch.empty(2, D, device="cuda").unbind(0)
    wsb = fast.fast_layer_norm_bwd_workspace(n, D)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_layer_norm_bwd(n, D, fast.BF16, h, ga, mean, rstd, dy, None, dx, dg, db, ws, wsb)
    mid = (1 << 31) // D
    at = torch.cat([some_rows(n, 8), torch.tensor([mid - 1, mid, mid + 1], device="cuda")])
    h64, mu, rs, dy64, g64 = (host(t) for t in (h[at], mean[at], rstd[at], dy[at], ga))
    rx, _, _ = p64.layer_norm_bwd(h64, g64, mu, rs, dy64, None)
    xh = np.abs((h64 - mu[:, None]) * rs[:, None])
    Mr = (np.abs(h64).max(1) + np.abs(mu))[:, None] * rs[:, None]
    g = np.abs(dy64 * g64)
    m1, m2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    tol = U * rs[:, None] * 60 * (g + m1 + (xh + Mr) * (m2 + m1 * Mr)) + 2 * U * np.abs(rx)
    assert (np.abs(host(dx[at]) - rx) <= tol + HALF["bf16"] * np.abs(rx)).all()
    for k in range(0, n, 1 << 22):                  # nothing is left as it was
        assert not (dx[k:k + (1 << 22)] == 768).any()
    check_weight_gradients(h, dy, mean, rstd, dg, db)
