"""GPU parity of the cached rows (8 and 4 bits) and of the attention that reads
them, against the plain 64-bit definitions, through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64 as p64
from tests.parity import tdtype, to_dev
from tests.plain64 import HALF, U

pytestmark = pytest.mark.gpu

DT = {"f32": fast.F32, "bf16": fast.BF16}
FMT = {8: fast.MXFP8, 4: fast.MXFP4}


def host(t):
    return t.detach().double().cpu().numpy()


def make_rows(n, parts, width, dt, seed):
    """Rows of mixed magnitudes, with zeros, ties and the formats' own values among them."""
    r = np.random.default_rng(seed)
    x = r.normal(size=(n, parts, width)) * 2.0 ** r.integers(-20, 20, (n, parts, 1))
    kind = r.integers(0, 12, n)
    x[kind == 0] = 0
    x[kind == 1] = r.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, 17.0, 19.0, 448.0, 1.0625],
                            (int((kind == 1).sum()), parts, width))
    x[kind == 2] *= 2.0 ** -120
    x[kind == 3] *= 2.0 ** 100
    t = torch.from_numpy(x.astype(np.float32)).to(tdtype(dt))
    return t.cuda(), t.double().numpy()


def write(ids, bound, smap, src, fmt, cache, rows, distinct, dt):
    n, parts, width = src.shape
    wsb = 0 if distinct else fast.fast_cache_write_workspace(n, rows)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda")
    fast.fast_cache_write(ids, n, bound, smap, parts, width, DT[dt], src, FMT[fmt], cache, rows, distinct, ws, wsb)


def test_every_code_and_scale_reads_back():
    """All 256 codes under all 256 scales of both formats."""
    for fmt in (8, 4):
        print(f"[cache] all codes fmt={fmt}", flush=True)
        codes = np.tile(np.arange(2 ** fmt, dtype=np.uint8), 32 if fmt == 4 else 2)[:512].reshape(1, 512)
        codes = np.repeat(codes[None], 256, 0)
        sc = np.repeat(np.arange(256, dtype=np.uint8)[:, None, None], 16, 2)
        rec = to_dev(p64.pack(codes, sc, fmt))
        ids = torch.arange(256, device="cuda")
        out = torch.empty(256, 1, 512, device="cuda")
        fast.fast_cache_gather(ids, 256, 256, None, 1, 512, FMT[fmt], rec, 256, fast.F32, out)
        with np.errstate(over="ignore"):
            want = p64.values(codes, sc, fmt).astype(np.float32)
        np.testing.assert_array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("parts,width", [(1, 1), (1, 7), (1, 172), (2, 31), (4, 32), (4, 50), (8, 33), (16, 128),
                                         (1, 1000), (128, 64), (6, 8), (2, 256)])
@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_write_and_gather(parts, width, fmt, dt):
    print(f"[cache] parts={parts} width={width} fmt={fmt} {dt}", flush=True)
    n, rows, bound = 150, 400, 1000
    r = np.random.default_rng(width)
    src, s64 = make_rows(n, parts, width, dt, width + fmt)
    smap = np.full(bound, -1, np.int32)
    hot = r.choice(bound, rows, replace=False)
    smap[hot] = np.arange(rows)
    smap[r.choice(np.setdiff1d(np.arange(bound), hot), 5)] = [rows, rows + 7, -9, 2 ** 31 - 1, -2 ** 31]
    ids = r.choice(bound, n, replace=False).astype(np.int64)
    ids[:4] = [-1, bound, 2 ** 62, -2 ** 62]                       # no row
    stride = p64.record(parts, width, fmt)[3]
    before = r.integers(0, 256, (rows, stride), dtype=np.uint8)
    cache = to_dev(before)
    write(to_dev(ids), bound, to_dev(smap), src, fmt, cache, rows, True, dt)
    slot = p64.slots(ids, bound, smap, rows)
    code, groups, content, _ = p64.record(parts, width, fmt)
    want = before.copy()
    c, s = p64.quantize(s64[slot >= 0], fmt)
    want[slot[slot >= 0], :content] = p64.pack(c, s, fmt)[:, :content]
    got = cache.cpu().numpy()
    # codes, scales, the other records and the bytes behind a record's content
    np.testing.assert_array_equal(got, want)
    # read back: written rows, by id, in both types; ids without a row leave theirs
    for od in ("f32", "bf16"):
        out = torch.full((n + 1, parts, width), 7.0, dtype=tdtype(od), device="cuda")
        fast.fast_cache_gather(to_dev(ids), n, bound, to_dev(smap), parts, width, FMT[fmt], cache, rows, DT[od], out)
        with np.errstate(over="ignore"):
            v = torch.from_numpy(p64.values(c, s, fmt)).float().to(tdtype(od)).double().numpy()
        np.testing.assert_array_equal(host(out[:n])[slot >= 0], v)
        assert (out[:n][to_dev(slot < 0)] == 7).all() and (out[n] == 7).all()


@pytest.mark.parametrize("fmt", [8, 4])
def test_groups_that_are_not_numbers(fmt):
    src, s64 = make_rows(6, 2, 70, "f32", 3)
    for i, bad in enumerate([np.inf, -np.inf, np.nan]):
        src[i, 1, 40] = bad
        s64[i, 1, 40] = bad
    cache = torch.zeros(6, p64.record(2, 70, fmt)[3], dtype=torch.uint8, device="cuda")
    ids = torch.arange(6, device="cuda")
    write(ids, 6, None, src, fmt, cache, 6, True, "f32")
    c, s = p64.quantize(s64, fmt)
    np.testing.assert_array_equal(cache.cpu().numpy(), p64.pack(c, s, fmt))
    out = torch.empty(6, 2, 70, device="cuda")
    fast.fast_cache_gather(ids, 6, 6, None, 2, 70, FMT[fmt], cache, 6, fast.F32, out)
    nan = torch.isnan(out).cpu().numpy()
    assert nan[:3, 1, 32:64].all() and nan.sum() == 96


@pytest.mark.parametrize("n,rows", [(1, 1), (2, 1), (300, 7), (5000, 100), (5000, 4000), (70000, 9)])
def test_the_last_row_of_a_slot_stays(n, rows):
    print(f"[cache] repeats n={n} rows={rows}", flush=True)
    r = np.random.default_rng(n)
    src, s64 = make_rows(n, 3, 40, "f32", 8)
    ids = r.integers(-2, rows + 2, n)
    cache = torch.zeros(rows, p64.record(3, 40, 8)[3], dtype=torch.uint8, device="cuda")
    write(to_dev(ids), rows, None, src, 8, cache, rows, False, "f32")
    last = np.full(rows, -1)
    for i, s in enumerate(ids):
        if 0 <= s < rows:
            last[s] = i
    c, s = p64.quantize(s64[last[last >= 0]], 8)
    got = p64.unpack(cache.cpu().numpy()[last >= 0], 3, 40, 8)
    np.testing.assert_array_equal(got, p64.values(c, s, 8))


def test_cache_past_four_gib():
    print("[cache] 6 GB cache", flush=True)
    rows = 24_000_000
    stride = fast.fast_cache_row_bytes(4, 50, fast.MXFP8)
    assert rows * stride > 5 << 30
    cache = torch.zeros(rows, stride, dtype=torch.uint8, device="cuda")
    ids = np.array([0, 1, 8_388_607, 8_388_608, 16_777_215, 16_777_216, rows - 1], np.int64)
    src, s64 = make_rows(len(ids), 4, 50, "f32", 5)
    write(to_dev(ids), rows, None, src, 8, cache, rows, True, "f32")
    c, s = p64.quantize(s64, 8)
    want = p64.values(c, s, 8)
    out = torch.empty(len(ids), 4, 50, device="cuda")
    fast.fast_cache_gather(to_dev(ids), len(ids), rows, None, 4, 50, fast.MXFP8, cache, rows, fast.F32, out)
    np.testing.assert_array_equal(host(out), want)
    Q = torch.zeros(1, 2, 50, device="cuda")
    res = torch.empty(1, 2, 50, device="cuda")
    g = fast.tcsr(to_dev(np.array([0, len(ids)], np.int32)), len(ids))
    wsb = fast.fast_edge_attention_cached_workspace(1, len(ids), 2, 50)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_edge_attention_fwd_cached(g, 2, 50, fast.F32, Q, to_dev(ids), rows, None, fast.MXFP8, cache, rows,
                                        1.0, 0.2, res, None, ws, wsb)
    mean = want[:, 2:].mean(0)                     # a zero query weighs every edge alike
    assert (np.abs(host(res)[0] - mean) <= 20 * U * np.abs(want[:, 2:]).max(0)).all()
    # many segments of one edge each return that edge's value
    N = 5000
    pick = np.arange(N) % len(ids)
    Q = torch.randn(N, 2, 50, device="cuda")
    res = torch.empty(N, 2, 50, device="cuda")
    g = fast.tcsr(torch.arange(N + 1, dtype=torch.int32, device="cuda"), N)
    wsb = fast.fast_edge_attention_cached_workspace(N, N, 2, 50)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_edge_attention_fwd_cached(g, 2, 50, fast.F32, Q, to_dev(ids[pick]), rows, None, fast.MXFP8, cache, rows,
                                        1.0, 0.2, res, None, ws, wsb)
    np.testing.assert_array_equal(host(res), want[pick, 2:])
    del cache


# ------------------------------------------------------------------ attention
class Block:
    def __init__(self, counts, H, dh, fmt, dt, rows=97, bound=200, seed=0, miss=0.2):
        r = np.random.default_rng(seed)
        self.H, self.dh, self.fmt, self.dt, self.rows, self.bound = H, dh, fmt, dt, rows, bound
        self.off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.N, self.E = len(counts), int(self.off[-1])
        kv = r.normal(size=(rows, 2 * H, dh)).astype(np.float32)
        c, s = p64.quantize(kv, fmt)
        self.kv = p64.values(c, s, fmt)
        self.cache = to_dev(p64.pack(c, s, fmt, fill=0xFF))
        self.smap = np.full(bound, -1, np.int32)
        hot = r.choice(bound, rows, replace=False)
        self.smap[hot] = np.arange(rows)
        self.ids = np.where(r.random(self.E) < miss, r.integers(-3, bound + 3, self.E),
                            hot[r.integers(0, rows, self.E)]).astype(np.int64)
        q = torch.from_numpy(r.normal(size=(self.N, H, dh)).astype(np.float32)).to(tdtype(dt))
        self.Q, self.q64 = q.cuda(), q.double().numpy()
        self.scale, self.slope = 1 / np.sqrt(dh), 0.2

    def run(self, want_lse=True, stream=None, bufs=None):
        N, H, dh = self.N, self.H, self.dh
        if bufs is None:
            bufs = self.buffers()
        out, lse, ws, wsb, g, ids, smap = bufs
        fast.fast_edge_attention_fwd_cached(g, H, dh, DT[self.dt], self.Q, ids, self.bound, smap, FMT[self.fmt],
                                            self.cache, self.rows, self.scale, self.slope, out,
                                            lse if want_lse else None, ws, wsb, stream)
        return out, lse

    def buffers(self):
        wsb = fast.fast_edge_attention_cached_workspace(self.N, self.E, self.H, self.dh)
        return (torch.full((self.N + 1, self.H, self.dh), 7.0, dtype=tdtype(self.dt), device="cuda"),
                torch.full((self.N + 1, self.H), 7.0, device="cuda"),
                torch.empty(wsb, dtype=torch.uint8, device="cuda").fill_(0xFF), wsb,
                fast.tcsr(to_dev(self.off), self.E), to_dev(self.ids), to_dev(self.smap))

    def check(self, out, lse):
        slot = p64.slots(self.ids, self.bound, self.smap, self.rows)
        ro, rl, vmax, qk = p64.attention(self.off, self.q64, slot, self.kv, self.scale, self.slope)
        # a logit: dh products in fp32, at most 8 in a lane and 5 across lanes, q scaled twice:
        # 16 U of sum |q k|, and 2 U of the shifted logit (at most 2 qk) in the exponential's
        # argument plus its own 2 U; a weight twice that.  Then sums of at most 256 / 2 + 40
        # weighted rows in a lane chain, joined; E / 512 partial results in a row at most.
        delta = U * (20 * qk + 8)
        chain = U * (180 + self.E / 512)
        n, H = self.N, self.H
        tol = (vmax * (2 * delta + chain))[..., None] + HALF[self.dt] * np.abs(ro)
        o = host(out[:n])
        bad = ~(np.abs(o - ro) <= tol)
        assert not bad.any(), (int(bad.sum()), float(np.abs(o - ro).max()), np.argwhere(bad)[:4].tolist())
        l = host(lse[:n])
        empty = np.isinf(rl)
        assert (l[empty] == -np.inf).all() and (o[empty] == 0).all()
        assert (np.abs(l - rl)[~empty] <= (delta + chain + 4 * U * np.abs(rl))[~empty]).all()
        assert (out[n] == 7).all() and (lse[n] == 7).all()


@pytest.mark.parametrize("H,dh", [(2, 50), (4, 32), (1, 1), (3, 7), (1, 8), (8, 128), (2, 256), (64, 16), (5, 43),
                                  (16, 9), (20, 50), (1, 100), (7, 64)])
@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_cached_attention_shapes(H, dh, fmt, dt):
    print(f"[cache] attention H={H} dh={dh} fmt={fmt} {dt}", flush=True)
    b = Block([0, 1, 10, 3, 0, 64, 65, 17, 200, 0, 16, 15, 2, 0], H, dh, fmt, dt, seed=H * 1000 + dh)
    b.check(*b.run())


@pytest.mark.parametrize("counts", [
    [1], [0], [0, 0, 0], [64], [65], [1000], [5000], [1, 5000, 0, 0, 70, 64, 0, 4097, 3], [63, 1, 129, 1, 127],
    [10] * 500 + [3000] + [0] * 300 + [9] * 400 + [130], [64] * 40, [128, 128, 192, 256], [0] * 5000 + [300],
    [300] + [0] * 5000, [2] * 9000], ids=lambda c: f"N{len(c)}E{sum(c)}m{max(c)}")
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_cached_attention_lengths(counts, dt):
    print(f"[cache] attention lengths N={len(counts)} E={sum(counts)} {dt}", flush=True)
    b = Block(counts, 2, 50, 8, dt, seed=len(counts))
    b.check(*b.run())


@pytest.mark.parametrize("H,dh", [(1, 1), (1, 8), (3, 7), (2, 50), (8, 128), (2, 256), (64, 16), (20, 50), (1, 100),
                                  (5, 43), (4, 40)])
@pytest.mark.parametrize("fmt", [8, 4])
def test_cached_attention_many_segments(H, dh, fmt):
    """More segments than a wave each is chosen for: a few lanes per segment, empty and long ones among them."""
    print(f"[cache] attention many segments H={H} dh={dh} fmt={fmt}", flush=True)
    r = np.random.default_rng(dh)
    counts = r.integers(0, 6, 4500)
    counts[[7, 900, 901, 4499]] = [300, 70, 257, 1100]
    b = Block(counts, H, dh, fmt, "f32" if H % 2 else "bf16", seed=dh + H)
    b.check(*b.run())


@pytest.mark.parametrize("H,dh", [(2, 33), (4, 40), (3, 65), (2, 100), (1, 136), (3, 161), (1, 232)])
@pytest.mark.parametrize("fmt", [8, 4])
def test_cached_attention_heads_just_past_a_group(H, dh, fmt):
    """The last piece of a head starts in the group before its own codes, whose scale may be any
    other: here so large that the codes before would overflow under it."""
    print(f"[cache] attention H={H} dh={dh} fmt={fmt}, scales far apart", flush=True)
    counts = [3, 0, 70, 9, 1] * 30
    b = Block(counts, H, dh, fmt, "bf16", seed=dh)
    b.check(*b.run())
    b = Block(counts, H, dh, fmt, "f32", seed=dh)
    r = np.random.default_rng(dh)
    last = dh // 32 * 32
    kv = r.normal(size=(b.rows, 2 * H, dh)).astype(np.float32)
    kv[:, :, last - 32:last] = np.clip(kv[:, :, last - 32:last], -1, 1)
    kv[:, :, last - 8:last] = 1.0                       # 256 or 4 times its group's scale
    # the largest magnitude, 2^120 (2^126) times a code, is finite; 256 (4) times that scale is not
    top = np.float32(3.0e38 if fmt == 8 else 2.6e38)
    kv[:, :H, last:] = np.clip(kv[:, :H, last:], -1, 1) * top
    kv[:, :H, last] = top
    c, s = p64.quantize(kv, fmt)
    b.kv = p64.values(c, s, fmt)
    assert np.abs(b.kv).max() < 3.4e38
    b.cache = to_dev(p64.pack(c, s, fmt, fill=0xFF))
    b.q64[..., last:] *= 1e-37
    b.q64 = b.q64.astype(np.float32).astype(np.float64)
    b.Q = to_dev(b.q64.astype(np.float32))
    b.check(*b.run())


@pytest.mark.parametrize("most", [1, 20, 40])
def test_cached_attention_long_among_very_many_short(most):
    """Lengths about every cut of a block whose segments belong to a few lanes each."""
    r = np.random.default_rng(most)
    counts = r.integers(0, most, 6000)
    long = [63, 64, 65, 66, 127, 128, 129, 130, 255, 256, 257, 600]
    counts[100:100 + len(long)] = long
    counts[r.choice(np.arange(1000, 6000), len(long), replace=False)] = long
    counts[5999] = 65
    print(f"[cache] attention long among short N=6000 E={counts.sum()}", flush=True)
    b = Block(counts, 2, 50, 8, "f32", seed=most)
    b.check(*b.run())


@pytest.mark.parametrize("E,N", [(400000, 3), (600000, 20000)])
def test_cached_attention_long_histories(E, N):
    """Piece lengths above the shortest, a hub across very many pieces."""
    print(f"[cache] attention hub E={E} N={N}", flush=True)
    r = np.random.default_rng(E)
    counts = r.integers(0, 20, N)
    counts[N // 2] += E - counts.sum()
    b = Block(counts, 4, 32, 4, "bf16", rows=3000, bound=5000, seed=9)
    b.check(*b.run())


def test_cached_attention_queries_past_two_to_the_31_elements():
    """Segments of no edges but at the first, the last and those around element 2^31 of Q."""
    H, dh, N = 4, 32, 17_000_000
    mid = (1 << 31) // (H * dh)
    assert N > mid + 1
    print(f"[cache] attention N={N}", flush=True)
    at = np.array([0, mid - 1, mid, mid + 1, N - 1])
    b = Block([3, 1, 7, 2, 300], H, dh, 8, "bf16", rows=50, bound=60)
    off = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    for v, c in zip(at, np.diff(b.off)):
        off[v + 1:] += int(c)
    Q = torch.zeros(N, H, dh, dtype=torch.bfloat16, device="cuda")
    Q[to_dev(at)] = b.Q
    out = torch.full((N, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(N, H, device="cuda")
    wsb = fast.fast_edge_attention_cached_workspace(N, b.E, H, dh)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_edge_attention_fwd_cached(fast.tcsr(off, b.E), H, dh, fast.BF16, Q, to_dev(b.ids), b.bound,
                                        to_dev(b.smap), fast.MXFP8, b.cache, b.rows, b.scale, b.slope, out, lse, ws, wsb)
    pad = torch.full((1, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    b.check(torch.cat([out[to_dev(at)], pad]), torch.cat([lse[to_dev(at)], pad[:, :, 0].float()]))
    out[to_dev(at)] = 0
    assert not out.any()


def test_cached_attention_no_edge_is_cached():
    b = Block([3, 100, 0, 700], 2, 50, 8, "f32")
    b.smap[:] = -1
    out, lse = b.run()
    b.check(out, lse)
    assert (out[:4] == 0).all() and (lse[:4] == float("-inf")).all()
    b.rows, b.cache = 0, None
    out, lse = b.run()
    assert (out[:4] == 0).all() and (lse[:4] == float("-inf")).all()


def test_cached_attention_masked_edges_read_nothing_of_their_record():
    # every record that no edge may read holds NaN scales, and the query's own infinity in a
    # segment without edges stays there
    b = Block([5, 0, 300, 12], 2, 50, 8, "f32", miss=0.5)
    slot = p64.slots(b.ids, b.bound, b.smap, b.rows)
    unused = np.setdiff1d(np.arange(b.rows), slot)
    b.cache[to_dev(unused)] = 0xFF
    b.Q[1] = float("inf")
    b.q64[1] = np.inf
    b.check(*b.run())


def test_cached_attention_nan_rows_stay_in_their_head_and_segment():
    b = Block([4, 6, 200], 2, 50, 8, "f32", miss=0.0, rows=300, bound=400)
    b.ids[:] = np.flatnonzero(b.smap >= 0)[np.arange(b.E) % 300]
    slot = b.smap[b.ids[5]]                       # an edge of segment 1
    code, groups, content, _ = p64.record(4, 50, 8)
    b.cache[int(slot), 4 * code + 0] = 255        # K, head 0, first group
    out, lse = b.run()
    nan = torch.isnan(out[:3]).cpu().numpy()
    assert nan[1, 0].all() and nan.sum() == 50 and torch.isnan(lse[1, 0]) and int(torch.isnan(lse).sum()) == 1


def test_cached_attention_is_repeatable_on_streams_and_in_graphs():
    b = Block([10] * 700 + [2000, 0, 900] + [7] * 300, 2, 50, 8, "f32")
    want = [t.clone() for t in b.run()]
    torch.cuda.synchronize()
    one, two = b.buffers(), b.buffers()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s1, bufs=one)                     # two calls at once, a workspace each
    b.run(stream=s2, bufs=two)
    torch.cuda.synchronize()
    for bufs in (one, two):
        assert torch.equal(bufs[0], want[0]) and torch.equal(bufs[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(bufs=one)
    for _ in range(3):
        one[0].fill_(7.0)
        one[1].fill_(7.0)
        b.run(bufs=two)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one[0], want[0]) and torch.equal(one[1], want[1])


def test_cache_write_in_a_graph_with_repeats():
    n, rows = 900, 200
    src, s64 = make_rows(n, 4, 50, "f32", 21)
    ids = torch.randint(0, rows, (n,), device="cuda")
    stride = fast.fast_cache_row_bytes(4, 50, fast.MXFP4)
    cache = torch.zeros(rows, stride, dtype=torch.uint8, device="cuda")
    want = torch.zeros_like(cache)
    wsb = fast.fast_cache_write_workspace(n, rows)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.zeros(n, 4, 50, device="cuda")

    def step(c):
        fast.fast_cache_write(ids, n, rows, None, 4, 50, fast.F32, src, fast.MXFP4, c, rows, False, ws, wsb)
        fast.fast_cache_gather(ids, n, rows, None, 4, 50, fast.MXFP4, c, rows, fast.F32, out)
    step(want)
    first = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache)
    for _ in range(3):
        cache.zero_()
        ws.fill_(0xCD)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cache, want) and torch.equal(out, first)
        step(want)
