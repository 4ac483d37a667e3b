"""fp32 products of many rows, formed from three bf16 parts of each value: how far a product may be off, and
values that are not finite.  U = 2^-24 is half a step of fp32."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests.plain64 import U
from tests.test_gpu_layer import host, rand, within
from tests.test_gpu_linear import strided

pytestmark = pytest.mark.gpu

# every bit below the first part set, and below the second; halves of their steps and just not
HARD = [0x3f80ffff, 0x3f807fff, 0x3f807fbf, 0x3f80ff7f, 0x3fff7fff, 0x3f808080, 0x3f817f7f, 0x3fffffff, 0x3f800001]


def hard(n, seed):
    """fp32 numbers of all mantissas and signs, within 2^20 of 1"""
    r = np.random.default_rng(seed)
    b = r.integers(0, 1 << 23, n).astype(np.uint32) | np.uint32(0x3f800000)
    k = r.random(n) < 0.7
    b[k] = r.choice(np.array(HARD, np.uint32), k.sum())
    return (b.view(np.float32) * np.exp2(r.integers(-20, 21, n)) * r.choice([-1, 1], n)).astype(np.float32)


def alone(got, a, b, what):
    """One product a b that nothing else is added to: the three left-out products of parts are within
    2 (2^-8 2^-16) + 2^-32 of it, so 2^-22 with a margin of two; adding the parts' products and
    rounding the result take a step of fp32 of it."""
    ref = a.astype(np.float64) * b.astype(np.float64)
    within(got, ref, (2.0 ** -22 + 2 * U) * np.abs(ref), what)


@pytest.mark.parametrize("n,K,M", [(16500, 75, 141), (16384, 64, 128), (33001, 100, 66)])
def test_linear_parts_hold_a_product(n, K, M):
    """Rows with one value each: y and dx are single products; columns of dw likewise."""
    print(f"[parts] one product n={n} K={K} M={M}", flush=True)
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 0, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    rows = np.arange(n)
    xv, wv = hard(n, 1), hard(M * K, 2).reshape(M, K)
    x = np.zeros((n, K), np.float32)
    x[rows, rows % K] = xv
    X, W = torch.from_numpy(x).cuda(), torch.from_numpy(wv).cuda()
    y = torch.empty(n, M, device="cuda")
    fast.fast_linear_fwd(n, K, M, 0, X, K, W, None, 0, None, M, y, M)
    alone(y, xv[:, None], wv.T[rows % K], "y")
    dy = np.zeros((n, M), np.float32)
    dy[rows, rows % M] = xv
    dx = torch.empty(n, K, device="cuda")
    fast.fast_linear_bwd(n, K, M, 0, None, K, W, 0, None, torch.from_numpy(dy).cuda(), M, dx, K, None, None, ws, wsb)
    alone(dx, xv[:, None], wv[rows % M], "dx")
    # dw[m, k] = dy[r, m] x[r, k] of the one row r that holds m
    dy[M:] = 0
    x = np.zeros((n, K), np.float32)
    x[:M] = wv
    dw = torch.empty(M, K, device="cuda")
    fast.fast_linear_bwd(n, K, M, 0, torch.from_numpy(x).cuda(), K, None, 0, None, torch.from_numpy(dy).cuda(), M, None, K,
                         dw, None, ws, wsb)
    alone(dw, xv[:M, None], wv, "dw")


def test_linear_parts_next_to_the_largest_number():
    """Two values whose first parts, rounded up, have a product past the largest number: their own is 3.39e38."""
    n, K, M = 16500, 64, 128
    v = np.array([0x3fff7fff], np.uint32).view(np.float32)[0] * np.float32(2.0 ** 63)
    big = np.full(n, v, np.float32)
    x = np.zeros((n, K), np.float32)
    x[np.arange(n), np.arange(n) % K] = v
    X = torch.from_numpy(x).cuda()
    w = torch.full((M, K), float(v), device="cuda")
    w[1::2] = 2.0 ** -40
    y = torch.empty(n, M, device="cuda")
    fast.fast_linear_fwd(n, K, M, 0, X, K, w, None, 0, None, M, y, M)
    alone(y[:, ::2], big[:, None], np.full((1, M // 2), v), "y")
    alone(y[:, 1::2], big[:, None], np.full((1, M // 2), 2.0 ** -40, np.float32), "y beside it")
    dw = torch.empty(M, K, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 0, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    dy = torch.zeros(n, M, device="cuda")
    dy[torch.arange(K), torch.arange(K)] = float(v)
    fast.fast_linear_bwd(n, K, M, 0, X, K, None, 0, None, dy, M, None, K, dw, None, ws, wsb)
    assert (dw[:K] == torch.diag(torch.diagonal(dw))).all()
    alone(torch.diagonal(dw), big[:K], big[:K], "dw")


def test_linear_weight_gradients_always_in_parts():
    """One row: fp32 weight gradients are formed from parts at any n, and held to the same."""
    K, M = 37, 53
    a, b = hard(M, 3), hard(K, 4)
    dw = torch.empty(M, K, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(1, K, M, 0, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(1, K, M, 0, torch.from_numpy(b).cuda().view(1, K), K, None, 0, None,
                         torch.from_numpy(a).cuda().view(1, M), M, None, K, dw, None, ws, wsb)
    alone(dw, a[:, None], b[None], "dw")


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_linear_weight_gradients_of_bf16_rows_hold_dz(kind):
    """With an activation dz is no bf16 number; dw reads all of it."""
    from tests import plain64_train as p64
    from tests.test_gpu_linear import ACT, slope_error
    n, K, M = 300, 40, 60
    x, x64 = rand((n, K), "bf16", 1)
    dy, dy64 = rand((n, M), "bf16", 2)
    pre, pre64 = rand((n, M), "bf16", 3)
    keep = torch.arange(n, device="cuda")[:, None] == torch.arange(M, device="cuda")
    dy = dy * keep
    dy64 = dy64 * keep.cpu().numpy()
    dw = torch.empty(M, K, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 1, ACT[kind])
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(n, K, M, 1, x, K, None, ACT[kind], pre, dy, M, None, K, dw, None, ws, wsb)
    dz = dy64 * p64.slope(kind, pre64)
    off = np.abs(dy64) * slope_error(kind, pre64) + 2 * U * np.abs(dz)
    ref = dz.T @ x64
    within(dw, ref, off.T @ np.abs(x64) * 1.01 + 4 * U * np.abs(ref) + 1e-37, "dw")


@pytest.mark.parametrize("n,K,M", [(16500, 75, 141), (16385, 66, 130)])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_parts_and_values_that_are_not_finite(n, K, M, wide):
    """A tile that meets such a value is formed again with fp32 instructions: it reaches its own row (a
    weight's: its own column), with the sign that it has; all else is as close as always."""
    print(f"[parts] not finite n={n} K={K} M={M} wide={wide}", flush=True)
    ldx, ldy = (K + 3, M + 5) if wide else (K, M)
    x, x64 = strided(n, K, ldx, "f32", 1)
    w, w64 = rand((M, K), "f32", 2)
    dy, dy64 = strided(n, M, ldy, "f32", 3)
    inf, nan = float("inf"), float("nan")
    # a first row, the last one, a row inside; the first element, the last one (the tail of k), one inside
    spots = [(0, 0, inf), (n - 1, K - 1, -inf), (8000, K - 2, nan), (129, 40, -inf)]
    for r, c, v in spots:
        x[r, c] = v
    y = torch.full((n + 1, ldy), 7.0, device="cuda")
    fast.fast_linear_fwd(n, K, M, 0, x, ldx, w, None, 0, None, ldy, y[:, :M], ldy)
    assert (y[n] == 7).all() and (y[:, M:] == 7).all()
    got, ok = host(y[:n, :M]), np.ones(n, bool)
    for r, c, v in spots:
        ok[r] = False
        np.testing.assert_array_equal(got[r], v * np.sign(w64[:, c]))
    tol = 2 * (K + 3) * U * (np.abs(x64) @ np.abs(w64).T)
    within(y[:n, :M][torch.from_numpy(ok).cuda()], (x64 @ w64.T)[ok], tol[ok], "y")
    # weights: their columns of y, and of dx
    x, x64 = strided(n, K, ldx, "f32", 1)
    w[M - 1, K - 1], w[3, 5], w[70, 0] = inf, -inf, nan
    fast.fast_linear_fwd(n, K, M, 0, x, ldx, w, None, 0, None, ldy, y[:, :M], ldy)
    got, ok = host(y[:n, :M]), np.ones(M, bool)
    for m, c, v in ((M - 1, K - 1, inf), (3, 5, -inf), (70, 0, nan)):
        ok[m] = False
        np.testing.assert_array_equal(got[:, m], v * np.sign(x64[:, c]))
    within(y[:n, :M][:, torch.from_numpy(ok).cuda()], (x64 @ w64.T)[:, ok], tol[:, ok], "y of weights")
    dx = torch.full((n + 1, ldx), 7.0, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 0, 0)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")

    def back(dw=None):
        fast.fast_linear_bwd(n, K, M, 0, x, ldx, w, 0, None, dy, ldy, dx[:, :K], ldx, dw, None, ws, wsb)
        assert (dx[n] == 7).all() and (dx[:, K:] == 7).all()
        return host(dx[:n, :K])
    got, ok = back(), np.ones(K, bool)
    for m, c, v in ((M - 1, K - 1, inf), (3, 5, -inf), (70, 0, nan)):
        ok[c] = False
        np.testing.assert_array_equal(got[:, c], v * np.sign(dy64[:, m]))
    tol = 2 * (M + 3) * U * (np.abs(dy64) @ np.abs(w64))
    within(dx[:n, :K][:, torch.from_numpy(ok).cuda()], (dy64 @ w64)[:, ok], tol[:, ok], "dx of weights")
    # gradients: their rows of dx, their columns of dw
    w, w64 = rand((M, K), "f32", 2)
    spots = [(0, M - 1, inf), (n - 1, 0, -inf), (9001, 65, nan)]
    for r, c, v in spots:
        dy[r, c] = v
    dw = torch.empty(M, K, device="cuda")
    got, ok, okw = back(dw), np.ones(n, bool), np.ones(M, bool)
    for r, c, v in spots:
        ok[r], okw[c] = False, False
        np.testing.assert_array_equal(got[r], v * np.sign(w64[c]))
        np.testing.assert_array_equal(host(dw)[c], v * np.sign(x64[r]))
    within(dx[:n, :K][torch.from_numpy(ok).cuda()], (dy64 @ w64)[ok], tol[ok], "dx of gradients")
    # (sums of at most 16384 rows in fp32)
    tol = 2 * 16387 * U * (np.abs(dy64).T @ np.abs(x64))
    within(dw[torch.from_numpy(okw).cuda()], (dy64.T @ x64)[okw], tol[okw], "dw")
