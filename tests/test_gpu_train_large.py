"""Products, recurrence and AdamW on arrays of more than 2^31 elements (2^32 for the states in 8 bits, whose random
numbers go by the element's whole number): the rows on both sides of the border and the last ones."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64_train as p64
from tests.plain64 import HALF, U
from tests.test_gpu_layer import host, within

pytestmark = pytest.mark.gpu

BIG = 1 << 31


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("less than 100 GB of memory free")
    yield
    torch.cuda.empty_cache()


def fill(shape, dtype, seed, whole=False):
    """normal numbers, or whole ones of -3 .. 3, made in pieces (of 2^28 elements)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    for k in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - k)
        flat[k:k + n] = torch.randint(-3, 4, (n,), generator=g, device="cuda") if whole else torch.randn(n, generator=g, device="cuda")
    return t


@pytest.mark.parametrize("K,M,dt", [(272, 8, "bf16"), (8, 272, "bf16"), (520, 130, "f32"), (65, 1030, "bf16")])
def test_linear_past_2_31_elements(K, M, dt):
    n = BIG // max(K, M) + 3000
    print(f"[large] linear n={n} K={K} M={M} {dt}", flush=True)
    T, t = (0, torch.float32) if dt == "f32" else (1, torch.bfloat16)
    x, dy = fill((n, K), t, 1, True), fill((n, M), t, 2, True)
    w = (fill((M, K), torch.float32, 3) / K ** 0.5).to(t)
    y, dx = torch.empty(n, M, dtype=t, device="cuda"), torch.empty(n, K, dtype=t, device="cuda")
    fast.fast_linear_fwd(n, K, M, T, x, K, w, None, 0, None, M, y, M)
    wsb = fast.fast_linear_bwd_workspace(n, K, M, T, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    dw, db = torch.empty(M, K, device="cuda"), torch.empty(M, device="cuda")
    fast.fast_linear_bwd(n, K, M, T, x, K, w, 0, None, dy, M, dx, K, dw, db, ws, wsb)
    w64 = host(w)
    for r in (0, BIG // max(K, M) - 500, n - 1000):
        x64, d64 = host(x[r:r + 1000]), host(dy[r:r + 1000])
        ref = x64 @ w64.T
        within(y[r:r + 1000], ref, 2 * (K + 3) * U * (np.abs(x64) @ np.abs(w64).T) * 1.01 + HALF[dt] * np.abs(ref), "y")
        ref = d64 @ w64
        within(dx[r:r + 1000], ref, 2 * (M + 3) * U * (np.abs(d64) @ np.abs(w64)) * 1.01 + HALF[dt] * np.abs(ref), "dx")
    # whole numbers: a split's sums are at most 9 * 16384 < 2^24, exact in fp32, and joined in fp64
    rw, rb = torch.zeros(M, K, dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda")
    for r in range(0, n, 1 << 20):
        d = dy[r:r + (1 << 20)].double()
        rw += d.t().contiguous() @ x[r:r + (1 << 20)].double()
        rb += d.sum(0)
    assert torch.equal(dw, rw.float()) and torch.equal(db, rb.float())


def test_linear_activation_past_2_31_elements():
    n, K, M = BIG // 260 + 3000, 16, 260
    print(f"[large] linear n={n} K={K} M={M} silu", flush=True)
    pre, dy, x = fill((n, M), torch.bfloat16, 1), fill((n, M), torch.bfloat16, 2), fill((n, K), torch.bfloat16, 4)
    w = fill((M, K), torch.bfloat16, 3)
    dx = torch.empty(n, K, dtype=torch.bfloat16, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 1, fast.ACT_SILU)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    dw = torch.empty(M, K, device="cuda")
    fast.fast_linear_bwd(n, K, M, 1, x, K, w, fast.ACT_SILU, pre, dy, M, dx, K, dw, None, ws, wsb)
    w64 = host(w)
    for r in (0, BIG // M - 500, BIG // (2 * M) - 500, n - 1000):
        dz = host(dy[r:r + 1000]) * p64.slope("silu", host(pre[r:r + 1000]))
        a = np.abs(host(dy[r:r + 1000])) @ np.abs(w64)
        ref = dz @ w64
        # (slope_error of the products' tests is at most 24 U (1 + |z|), |z| < 8)
        within(dx[r:r + 1000], ref, (216 * U + 2.0 ** -16 + 2 * (2 * M + 3) * U) * a * 1.2 + HALF["bf16"] * np.abs(ref), "dx")
    assert torch.isfinite(dw).all()


def test_gated_scan_past_2_31_elements():
    """Short segments are walked alone: the same bits as a call of their own."""
    D, E = 1024, BIG // 1024 + 9000
    print(f"[large] scan E={E} D={D}", flush=True)
    r = np.random.default_rng(1)
    lengths = r.integers(0, 60, E // 25)
    off = np.minimum(np.concatenate([[0], np.cumsum(lengths)]), E).astype(np.int32)
    off[-1] = E
    off = off[:np.searchsorted(off, E) + 1]
    N, longest = len(off) - 1, int(np.diff(off).max())
    xg = fill((E, 2, D), torch.bfloat16, 1)
    dh = fill((E, D), torch.bfloat16, 2)
    dt = fill((E,), torch.float32, 3).abs()
    OFF = torch.from_numpy(off).cuda()

    def both(a, b):
        """segments a .. b"""
        lo, hi = int(off[a]), int(off[b])
        n, e = b - a, hi - lo
        blk = fast.tcsr((OFF[a:b + 1] - lo).contiguous(), e)
        v, t, d = xg[lo:hi], dt[lo:hi], dh[lo:hi]
        h, last = torch.empty(e, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, D, device="cuda")
        keep = torch.empty(fast.fast_gated_scan_state_rows(e), D, device="cuda")
        dxg = torch.empty(e, 2, D, dtype=torch.bfloat16, device="cuda")
        wsb = fast.fast_gated_scan_workspace(n, e, D)
        ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda")
        fast.fast_gated_scan_fwd(blk, D, 1, v[:, 0], v[:, 1], 2 * D, t, None, longest, h, last, keep, ws, wsb)
        fast.fast_gated_scan_bwd(blk, D, 1, v[:, 0], v[:, 1], 2 * D, t, None, longest, keep, d, None, dxg[:, 0], dxg[:, 1],
                                 2 * D, None, ws, wsb)
        return h, last, dxg
    h, last, dxg = both(0, N)
    for a in (0, int(np.searchsorted(off, BIG // D)) - 100, int(np.searchsorted(off, BIG // (2 * D))) - 100, N - 200):
        b = a + 200
        lo, hi = int(off[a]), int(off[b])
        want = both(a, b)
        assert torch.equal(h[lo:hi], want[0]) and torch.equal(last[a:b], want[1]) and torch.equal(dxg[lo:hi], want[2])


@pytest.mark.parametrize("low", [False, True], ids=["32", "8"])
def test_adamw_past_2_31_and_2_32_elements(low):
    n = (1 << 32) + 12325 if low else BIG + 12325
    print(f"[large] adamw n={n} low={low}", flush=True)
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    places = [0, BIG - 2048, n - 4133] + ([(1 << 32) - 2048] if low else [])
    places = [p - p % 32 for p in places]
    for k, p in enumerate(places):
        w[p:p + 4096], g[p:p + 4096] = fill((4096,), torch.float32, k), fill((4096,), torch.bfloat16, 10 + k)
    state = torch.uint8 if low else torch.float32
    m, v = torch.zeros(n, dtype=state, device="cuda"), torch.zeros(n, dtype=state, device="cuda")
    s = [torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda") for _ in range(2)] if low else [None, None]
    old = [w[p:p + 4096].clone() for p in places]
    ts = fast.adamw_tensors([w], [g], [m], [v], [s[0]] if low else None, [s[1]] if low else None)
    norm, scale = torch.zeros(2, 1, device="cuda").unbind(0)
    wsb = fast.fast_grad_norm_workspace(n, 1)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_grad_norm(ts, 1, 1e30, norm, scale, ws, wsb)
    want = np.sqrt(sum((host(g[p:p + 4096]) ** 2).sum() for p in places))
    assert abs(float(norm) - want) <= 2 * U * want and float(scale) == 1
    fast.fast_adamw(ts, 1, fast.STATE_MXFP8 if low else fast.STATE_F32, 1e-3, .9, .999, 1e-8, 3, 77, scale=scale)
    c = np.uint64(0xFFFFFFFF)
    for p, w0 in zip(places, old):
        at = slice(p, p + 4096)
        g64 = host(g[at])
        rw, rm, rv = p64.adamw(host(w0), g64, 0 * g64, 0 * g64, 3, 1e-3, .9, .999, 1e-8, 0.0)
        within(w[at], rw, 1e-3 * 40 * U * np.abs((rw - host(w0)) / 1e-3) + 2 * U * np.abs(rw) + 1e-12, "w")
        if not low:
            within(m[at], rm, 4 * U * np.abs(rm), "m")
            within(v[at], rv, 5 * U * rv, "v")
            continue
        i = np.arange(p, p + 4096, dtype=np.uint64)
        key = p64.mix(p64.mix(np.array(77 ^ (3 * 0x9E3779B9 & 0xFFFFFFFF), np.uint64)))
        hi = ((i >> np.uint64(32)) * np.uint64(0x9E3779B9)) & c
        bits = p64.mix(p64.mix((key + hi) & c) ^ (i & c)).astype(np.int64)
        for got, sc, val, r, root in ((m, s[0], rm, bits & 0xFFFF, False), (v, s[1], np.sqrt(rv), bits >> 16, True)):
            code, scales = p64.to_codes(val.astype(np.float32).astype(np.float64), r, root)
            np.testing.assert_array_equal(got[at].cpu().numpy(), code)
            np.testing.assert_array_equal(sc[p // 32:p // 32 + 128].cpu().numpy(), scales)
    far = slice(BIG + 4096, BIG + 5000) if low else slice(BIG // 2, BIG // 2 + 5000)
    assert (w[far] == 0).all() and (m[far] == 0).all()
