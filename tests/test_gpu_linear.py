"""GPU parity of the products with an epilogue and their backward against the plain 64-bit
definitions, through the C ABI.  U = 2^-24 is half a step of fp32; a sum of k products in fp32 is
within 2 (k + 3) U of the sum of their magnitudes, however its terms are grouped and whichever
way the matrix unit rounds (a step each)."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64_train as p64
from tests.parity import tdtype
from tests.plain64 import HALF, U
from tests.test_gpu_layer import DT, host, rand, within

pytestmark = pytest.mark.gpu

ACT = {"none": fast.ACT_NONE, "relu": fast.ACT_RELU, "gelu": fast.ACT_GELU, "silu": fast.ACT_SILU}
# one row, one column, odd sizes, both sides of every tile's edge, many rows, long products
SHAPES = [(1, 1, 1), (1, 272, 100), (3, 7, 5), (31, 33, 65), (33, 64, 32), (130, 129, 131), (600, 372, 200),
          (257, 100, 257), (1000, 1030, 64), (2, 2048, 500), (33001, 20, 50), (8300, 75, 520), (16390, 130, 258),
          (520, 1, 300), (700, 300, 1)]
KINDS = ["none", "relu", "gelu", "silu"]


def act_error(kind, z, dz):
    """of act(z) where z is off by dz: slopes are at most 1.13, evaluation a few roundings; the
    argument of the complementary error function carries 2 U, which its logarithm's slope
    (at most |z| + 1) multiplies by its size"""
    return 1.13 * dz + U * np.abs(p64.act(kind, z)) * (16 + 3 * z * z) + 1e-37


def slope_error(kind, z):
    if kind in ("none", "relu"):
        return np.zeros_like(z)
    s = np.abs(p64.slope(kind, z))
    if kind == "gelu":
        bell = np.exp(-z * z / 2) * 0.4
        return U * (4 * s + (16 + 3 * z * z) * np.minimum(1, np.exp(-z * z / 2) + (z > 0)) + np.abs(z) * bell * (8 + z * z))
    return 24 * U * (1 + np.abs(z)) / (1 + np.exp(-z))


def strided(n, F, ld, dt, seed, scale=1.0):
    """rows of F elements, ld apart, the gaps not a number; one element off the 16-byte grid where
    ld says so (ld odd)"""
    t, v = rand((n, F), dt, seed, scale=scale)
    if ld == F:
        return t, v
    base = torch.full((n * ld + 1,), float("nan"), dtype=tdtype(dt), device="cuda")
    view = base[1:].view(n, ld)[:, :F]
    view.copy_(t)
    return view, v


def check_fwd(n, K, M, dt, kind, res, wide, seed=1):
    print(f"[linear] fwd n={n} K={K} M={M} {dt} {kind} res={res} wide={wide}", flush=True)
    ldx, ldy = (K + 3, M + 5) if wide else (K, M)
    x, x64 = strided(n, K, ldx, dt, seed)
    w, w64 = rand((M, K), dt, seed + 1, scale=1 / np.sqrt(K))
    b, b64 = rand((M,), "f32", seed + 2)
    r, r64 = strided(n, M, ldy, dt, seed + 3) if res else (None, None)
    y = torch.full((n + 1, ldy), 7.0, dtype=tdtype(dt), device="cuda")
    pre = torch.full((n + 1, M), 7.0, dtype=tdtype(dt), device="cuda") if kind != "none" else None
    fast.fast_linear_fwd(n, K, M, DT[dt], x, ldx, w, b, ACT[kind], r, ldy, y[:, :M], ldy, pre)
    ref, z = p64.linear(x64, w64, b64, kind, r64)
    tz = 2 * (K + 3) * U * (np.abs(x64) @ np.abs(w64).T + np.abs(b64))
    ty = act_error(kind, z, tz) + U * (np.abs(p64.act(kind, z)) + (0 if r64 is None else np.abs(r64)))
    within(y[:n, :M], ref, ty * (1 + HALF[dt]) + HALF[dt] * np.abs(ref), "y")
    if pre is not None:
        within(pre[:n], z, tz * (1 + HALF[dt]) + HALF[dt] * np.abs(z), "pre")
        assert (pre[n] == 7).all()
    assert (y[n] == 7).all() and (y[:, M:] == 7).all()
    # without pre: the same y; y in res's place: the same y
    if res:
        z2 = torch.full((n * ldy + 1,), 7.0, dtype=tdtype(dt), device="cuda")[1 if wide else 0:][:n * ldy].view(n, ldy)[:, :M]
        z2.copy_(r)
        fast.fast_linear_fwd(n, K, M, DT[dt], x, ldx, w, b, ACT[kind], z2, ldy, z2, ldy)
        assert torch.equal(z2, y[:n, :M])


@pytest.mark.parametrize("n,K,M", SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_fwd(n, K, M, dt, wide):
    k = KINDS[(n + K + M) % 4]
    check_fwd(n, K, M, dt, k, (n + M) % 2 == 0, wide)


@pytest.mark.parametrize("K,M", [(8, 1), (9, 33), (15, 7), (31, 32), (63, 64), (65, 31), (100, 172), (129, 40), (187, 100),
                                 (200, 200), (224, 9), (225, 250), (256, 288), (272, 256), (287, 225), (288, 3), (64, 960)])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_narrow_long(K, M, wide):
    """Many rows, a few columns: weights that a compute unit's memory just holds and just does not,
    lengths on both sides of the matrix unit's steps, a last group of rows that is not whole."""
    check_fwd(16384 + K, K, M, "bf16", "none", False, wide, seed=30)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 9, 32, 33])
@pytest.mark.parametrize("K,M", [(256, 5), (257, 300), (512, 1), (515, 130), (1025, 64), (2049, 7), (4100, 33)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_handful(n, K, M, dt):
    """A request's rows: long products of few results, forward and as the rows' gradient."""
    check_fwd(n, K, M, dt, KINDS[(n + K) % 4], M % 2 == 1, n % 2 == 0, seed=35)
    check_bwd(n, M, K, dt, KINDS[(n + M) % 4], n % 2 == 1, seed=36)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,M", [(70, 50, 90), (16500, 33, 300)])
def test_linear_fwd_activations(kind, dt, n, K, M):
    for res in (False, True):
        check_fwd(n, K, M, dt, kind, res, True, seed=20)


def test_linear_activation_values():
    """A product with the identity: activations far from and next to 0 and their slopes."""
    z = np.concatenate([np.linspace(-30, 30, 4001), [0.0, -0.0, 1e-30, -1e-30, 88.0, -88.0, 100.0, -100.0, 3e38, -3e38]])
    z = z.astype(np.float32)
    n = len(z)
    x = torch.from_numpy(z).cuda().view(n, 1)
    one = torch.ones(1, 1, device="cuda")
    for kind in KINDS[1:]:
        y, pre, dx = torch.empty(n, 1, device="cuda"), torch.empty(n, 1, device="cuda"), torch.empty(n, 1, device="cuda")
        fast.fast_linear_fwd(n, 1, 1, 0, x, 1, one, None, ACT[kind], None, 1, y, 1, pre)
        assert torch.equal(pre, x)
        z64 = z.astype(np.float64)
        with np.errstate(over="ignore"):
            ref, sl = p64.act(kind, z64), p64.slope(kind, z64)
            within(y[:, 0], ref, np.where(np.abs(z64) < 1e30, act_error(kind, z64, 0), U * np.abs(ref) * 16), kind)
            wsb = fast.fast_linear_bwd_workspace(n, 1, 1, 0, ACT[kind])
            ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
            dy = torch.ones(n, 1, device="cuda")
            fast.fast_linear_bwd(n, 1, 1, 0, x, 1, one, ACT[kind], pre, dy, 1, dx, 1, None, None, ws, wsb)
            ok = np.abs(z64) < 1e18
            within(dx[:, 0][torch.from_numpy(ok).cuda()], sl[ok], slope_error(kind, z64[ok]) + 4 * U, kind + " slope")


def check_bwd(n, K, M, dt, kind, wide, seed=40):
    print(f"[linear] bwd n={n} K={K} M={M} {dt} {kind} wide={wide}", flush=True)
    ldx, ldy = (K + 3, M + 5) if wide else (K, M)
    x, x64 = strided(n, K, ldx, dt, seed)
    w, w64 = rand((M, K), dt, seed + 1, scale=1 / np.sqrt(M))
    dy, dy64 = strided(n, M, ldy, dt, seed + 2)
    pre, pre64 = rand((n, M), dt, seed + 3) if kind != "none" else (None, None)
    dx = torch.full((n + 1, ldx), 7.0, dtype=tdtype(dt), device="cuda")
    dw, db = torch.full((M + 1, K), 7.0, device="cuda"), torch.full((M + 1,), 7.0, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, DT[dt], ACT[kind])
    ws = torch.full((wsb + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(n, K, M, DT[dt], x, ldx, w, ACT[kind], pre, dy, ldy, dx[:, :K], ldx, dw, db, ws, wsb)
    rx, rw, rb, dz = p64.linear_bwd(x64, w64, kind, pre64, dy64)
    low = dt == "bf16" and kind != "none"
    tdz = (np.abs(dy64) * slope_error(kind, pre64) + 2 * U * np.abs(dz)) if kind != "none" else 0 * dz
    a = np.abs(dz)
    # dx: bf16 products read dz rounded; dw: in three parts, which hold all of it
    tx = (tdz + (HALF[dt] * a if low else 0)) @ np.abs(w64) * 1.01 + 2 * (M + 3) * U * (a @ np.abs(w64))
    within(dx[:n, :K], rx, tx * (1 + HALF[dt]) + HALF[dt] * np.abs(rx), "dx")
    tw = tdz.T @ np.abs(x64) * 1.01
    tw = tw + 2 * (min(n, 16384) + 3) * U * (a.T @ np.abs(x64)) + U * np.abs(rw)
    within(dw[:M], rw, tw, "dw")
    within(db[:M], rb, tdz.sum(0) * 1.01 + 70 * U * a.sum(0) + U * np.abs(rb), "dbias")
    assert (dx[n] == 7).all() and (dx[:, K:] == 7).all() and (dw[M] == 7).all() and float(db[M]) == 7
    assert (ws[wsb:] == 0xAB).all()
    # each alone: the same bits
    dx2, dw2, db2 = torch.empty(n, K, dtype=tdtype(dt), device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(M, device="cuda")
    call = lambda *o: fast.fast_linear_bwd(n, K, M, DT[dt], x, ldx, w, ACT[kind], pre, dy, ldy, o[0], K, o[1], o[2], ws, wsb)
    call(dx2, None, None)
    call(None, dw2, None)
    call(None, None, db2)
    assert torch.equal(dx2, dx[:n, :K]) and torch.equal(dw2, dw[:M]) and torch.equal(db2, db[:M])


@pytest.mark.parametrize("n,K,M", SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_bwd(n, K, M, dt, wide):
    check_bwd(n, K, M, dt, KINDS[(n + K + M + wide) % 4], wide)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_bwd_activations(kind, dt):
    check_bwd(300, 70, 140, dt, kind, True, seed=60)
    check_bwd(40000, 36, 20, dt, kind, False, seed=70)


def test_linear_no_rows():
    w = torch.randn(5, 7, device="cuda")
    dw, db = torch.full((5, 7), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda")
    e = torch.empty(0, 7, device="cuda")
    f = torch.empty(0, 5, device="cuda")
    fast.fast_linear_fwd(0, 7, 5, 0, e, 7, w, None, 0, None, 5, f, 5)
    wsb = fast.fast_linear_bwd_workspace(0, 7, 5, 0, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(0, 7, 5, 0, e, 7, w, 0, None, f, 5, e, 7, dw, db, ws, wsb)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [40, 33000])
def test_linear_nonfinite_values_stay_in_their_row_or_column(dt, n):
    K, M = 50, 60
    x, _ = rand((n, K), dt, 1)
    w, _ = rand((M, K), dt, 2)
    x[3, 5], x[7, 49], x[9, 0] = float("inf"), float("nan"), float("-inf")
    y = torch.empty(n, M, dtype=tdtype(dt), device="cuda")
    fast.fast_linear_fwd(n, K, M, DT[dt], x, K, w, None, 0, None, M, y, M)
    bad = ~torch.isfinite(y)
    assert bad.any(1).nonzero().view(-1).tolist() == [3, 7, 9] and bad[[3, 7, 9]].all()
    assert torch.equal(torch.sign(y[3].float()), torch.sign(w[:, 5].float())) and torch.isinf(y[3]).all()
    assert torch.equal(torch.sign(y[9].float()), -torch.sign(w[:, 0].float()))
    # backward: a gradient that is not finite reaches its row of dx, its column of dw and dbias
    dy, _ = rand((n, M), dt, 3)
    x, _ = rand((n, K), dt, 4)
    dy[5, 11] = float("inf")
    dx, dw, db = torch.empty(n, K, dtype=tdtype(dt), device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(M, device="cuda")
    pre = torch.ones(n, M, dtype=tdtype(dt), device="cuda")
    for kind, p in (("none", None), ("relu", pre)):
        wsb = fast.fast_linear_bwd_workspace(n, K, M, DT[dt], ACT[kind])
        ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
        fast.fast_linear_bwd(n, K, M, DT[dt], x, K, w, ACT[kind], p, dy, M, dx, K, dw, db, ws, wsb)
        assert (~torch.isfinite(dx)).any(1).nonzero().view(-1).tolist() == [5]
        assert (~torch.isfinite(dw)).any(1).nonzero().view(-1).tolist() == [11] and torch.isinf(dw[11]).all()
        assert (~torch.isfinite(db)).nonzero().view(-1).tolist() == [11] and torch.isinf(db[11])


def test_linear_captured_and_on_another_stream():
    n, K, M, dt = 5000, 100, 200, "bf16"
    x, _ = rand((n, K), dt, 1)
    w, _ = rand((M, K), dt, 2)
    b, _ = rand((M,), "f32", 3)
    dy, _ = rand((n, M), dt, 4)
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 1, ACT["gelu"])

    def buffers():
        return [torch.empty(n, M, dtype=torch.bfloat16, device="cuda"), torch.empty(n, M, dtype=torch.bfloat16, device="cuda"),
                torch.empty(n, K, dtype=torch.bfloat16, device="cuda"), torch.empty(M, K, device="cuda"),
                torch.empty(M, device="cuda"), torch.empty(wsb, dtype=torch.uint8, device="cuda")]

    def step(o, stream=None):
        fast.fast_linear_fwd(n, K, M, 1, x, K, w, b, ACT["gelu"], None, M, o[0], M, o[1], stream=stream)
        fast.fast_linear_bwd(n, K, M, 1, x, K, w, ACT["gelu"], o[1], dy, M, o[2], K, o[3], o[4], o[5], wsb, stream=stream)

    o = buffers()
    step(o)
    want = [t.clone() for t in o[:5]]
    other = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(other, side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(other, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o)
    for _ in range(3):
        for t in o[:5]:
            t.fill_(-1)
        graph.replay()
        step(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(o, want))
