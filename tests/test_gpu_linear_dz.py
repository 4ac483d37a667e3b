"""GPU parity of the rows' gradient of bf16 products with an activation, held to how far dz may be off there:
two bf16 parts hold dz within 2^-16 of it (each is rounded to nearest, half a step of bf16 of what is left), 256
times finer than the rounding of dx itself.  U = 2^-24 is half a step of fp32."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64_train as p64
from tests.plain64 import HALF, U
from tests.test_gpu_layer import host, rand, within
from tests.test_gpu_linear import ACT, KINDS, slope_error, strided

pytestmark = pytest.mark.gpu


def gradient(n, K, M, kind, pre, dy, lddy, w, lddx=None):
    lddx = lddx or K
    dx = torch.full((n + 1, lddx), 7.0, dtype=torch.bfloat16, device="cuda")
    wsb = fast.fast_linear_bwd_workspace(n, K, M, 1, ACT[kind])
    ws = torch.full((wsb + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(n, K, M, 1, None, K, w, ACT[kind], pre, dy, lddy, dx[:, :K], lddx, None, None, ws, wsb)
    assert (ws[wsb:] == 0xAB).all() and (dx[n] == 7).all() and (dx[:, K:] == 7).all()
    return dx[:n, :K]


# one column, less than a chunk of them, few and many rows; parts side by side that reach just past and just not
# past what a streamed row may hold; both sides of a step of the matrix unit; a handful of long rows; wide ones
@pytest.mark.parametrize("n,K,M", [(1, 256, 1), (64, 64, 1), (700, 40, 3), (40001, 33, 1), (33001, 40, 3), (33001, 20, 8),
                                   (20001, 65, 100), (20000, 130, 144), (17003, 65, 145), (4000, 300, 70), (9000, 200, 129),
                                   (3, 700, 500), (1, 40, 2049), (515, 129, 1030), (16501, 1030, 515)])
@pytest.mark.parametrize("kind", KINDS[1:])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_dx_reads_dz_in_two_parts(n, K, M, kind, wide):
    print(f"[linear] dx n={n} K={K} M={M} {kind} wide={wide}", flush=True)
    ldx, ldy = (K + 3, M + 5) if wide else (K, M)
    w, w64 = rand((M, K), "bf16", 1, scale=1 / np.sqrt(M))
    dy, dy64 = strided(n, M, ldy, "bf16", 2)
    pre, pre64 = rand((n, M), "bf16", 3)
    dx = gradient(n, K, M, kind, pre, dy, ldy, w, ldx)
    dz = dy64 * p64.slope(kind, pre64)
    a = np.abs(dz) @ np.abs(w64)
    off = (np.abs(dy64) * slope_error(kind, pre64) + 2 * U * np.abs(dz)) @ np.abs(w64) * 1.01
    tol = off + 2.0 ** -16 * a + 2 * (2 * M + 3) * U * a
    ref = dz @ w64
    within(dx, ref, tol * (1 + HALF["bf16"]) + HALF["bf16"] * np.abs(ref) + 1e-37, "dx")


def test_linear_dx_of_weights_and_gradients_that_are_not_finite():
    """An infinite weight reaches its column of dx with the sign of dz, whatever dz's second part is; a
    NaN likewise; a gradient that is not finite reaches its row."""
    n, K, M = 300, 40, 33
    w, _ = rand((M, K), "bf16", 1)
    dy, dy64 = rand((n, M), "bf16", 2)
    pre, pre64 = rand((n, M), "bf16", 3)
    w[5, 7], w[32, 0], w[0, 39] = float("inf"), float("-inf"), float("nan")
    dx = host(gradient(n, K, M, "gelu", pre, dy, M, w))
    dz = dy64 * p64.slope("gelu", pre64)
    assert (dz[:, [5, 32]] != 0).all()
    assert sorted(set(np.argwhere(~np.isfinite(dx))[:, 1])) == [0, 7, 39] and np.isnan(dx[:, 39]).all()
    np.testing.assert_array_equal(dx[:, 7], np.inf * np.sign(dz[:, 5]))
    np.testing.assert_array_equal(dx[:, 0], -np.inf * np.sign(dz[:, 32]))
    w, w64 = rand((M, K), "bf16", 1)
    dy[11, 3], dy[200, 32] = float("-inf"), float("nan")
    dx = host(gradient(n, K, M, "silu", pre, dy, M, w))
    assert sorted(set(np.argwhere(~np.isfinite(dx))[:, 0])) == [11, 200] and np.isnan(dx[200]).all()
    np.testing.assert_array_equal(dx[11], -np.inf * np.sign(w64[3] * p64.slope("silu", pre64[11, 3])))


def test_linear_dx_next_to_the_largest_number():
    """dz between the largest bf16 number and the largest fp32 number: finite, as its product with a small weight."""
    pre = torch.linspace(0.7, 0.9, 256, device="cuda").bfloat16().view(-1, 1)
    n = pre.shape[0]
    dy = torch.full((n, 1), 3.3895313892515355e38, dtype=torch.bfloat16, device="cuda")
    w = torch.full((1, 8), 2.0 ** -30, dtype=torch.bfloat16, device="cuda")
    dz = host(dy) * p64.slope("gelu", host(pre))
    ok = (dz < 3.4028e38)[:, 0]
    assert ((dz > 3.3962e38)[:, 0] & ok).any()
    dx = host(gradient(n, 8, 1, "gelu", pre, dy, 1, w))
    ref = dz * host(w)
    assert (np.abs(dx - ref)[ok] <= ref[ok] * (HALF["bf16"] + 2.0 ** -14)).all()
