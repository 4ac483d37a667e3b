"""Products through the kernels that the rules choose for large calls, and weight gradients whose sums are exact:
a row that is left out, or counted twice, at a border of tiles or splits changes a whole number."""
import pytest
import torch

import paper_2607_05095_amd as fast
from tests.parity import tdtype
from tests.test_gpu_layer import DT
from tests.test_gpu_linear import ACT, KINDS, check_bwd, check_fwd

pytestmark = pytest.mark.gpu


# k >= 1024, 512 columns or more and 256 tiles or more of 256 x 256: 129 x 3 of them, every remainder odd.  The
# second shape is the first one's rows' gradient.
@pytest.mark.parametrize("kind,res,wide", [("silu", True, True), ("none", False, False), ("gelu", False, True),
                                           ("relu", True, False)])
def test_linear_long_products_into_wide_rows(kind, res, wide):
    check_fwd(32801, 1030, 515, "bf16", kind, res, wide, seed=3)


@pytest.mark.parametrize("kind,wide", [("none", True), ("relu", False), ("silu", True)])
def test_linear_long_products_into_wide_rows_of_gradients(kind, wide):
    check_bwd(32801, 515, 1030, "bf16", kind, wide, seed=5)


# rows of less than a chunk of k into tiles of 128 x 128
@pytest.mark.parametrize("n,K,M,dt", [(33001, 1, 33, "bf16"), (33001, 5, 33, "bf16"), (16500, 7, 65, "bf16"), (70001, 3, 16, "bf16"),
                                      (33001, 1, 65, "f32"), (22000, 2, 70, "f32"), (70001, 3, 31, "f32")])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_many_short_rows(n, K, M, dt, wide):
    check_fwd(n, K, M, dt, KINDS[(n + K) % 4], M % 2 == 1, wide, seed=7)
    check_bwd(n, M, K, dt, KINDS[(n + M) % 4], wide, seed=8)


# 32 x 32 results a workgroup: up to 256 of them and more, k of up to 1024 bytes and more
@pytest.mark.parametrize("n", [800, 830, 2000])
@pytest.mark.parametrize("K,M", [(250, 300), (600, 300), (1030, 310)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_few_results(n, K, M, dt):
    check_fwd(n, K, M, dt, KINDS[(n + K) % 4], K > 300, n == 830, seed=9)
    check_bwd(n, M, K, dt, KINDS[(n + M + K) % 4], n == 800, seed=10)


def small(n, F, dt, seed, ld=None):
    """whole numbers of -3 .. 3"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(-3, 4, (n, F), generator=g, device="cuda").to(tdtype(dt))
    if ld is None:
        return t
    base = torch.full((n, ld), float("nan"), dtype=tdtype(dt), device="cuda")
    base[:, :F] = t
    return base[:, :F]


# splits of 256 rows and of thousands; both sides of a split's, a tile's and the longest split's border
ROWS = [1, 63, 64, 65, 255, 256, 257, 511, 513, 8300, 16383, 16384, 16385, 16390, 33001, 65537]


@pytest.mark.parametrize("K,M", [(20, 50), (130, 258), (1030, 515), (1, 300), (300, 1)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "relu"])
def test_linear_weight_gradients_are_exact_in_whole_numbers(K, M, dt, kind):
    """|dw| <= 9 * 65537 < 2^24: every sum is a whole number that fp32 holds, whatever its order."""
    print(f"[linear] whole K={K} M={M} {dt} {kind}", flush=True)
    for n in ROWS:
        ldx, ldy = (K + 3, M + 5) if n % 2 else (K, M)
        x, dy = small(n, K, dt, n, ldx), small(n, M, dt, n + 1, ldy)
        pre = small(n, M, dt, n + 2) if kind == "relu" else None
        dz = dy.double() if pre is None else dy.double() * (pre > 0)
        dw, db = torch.full((M + 1, K), 0.5, device="cuda"), torch.full((M + 1,), 0.5, device="cuda")
        wsb = fast.fast_linear_bwd_workspace(n, K, M, DT[dt], ACT[kind])
        ws = torch.full((wsb + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # (nothing but no number)
        fast.fast_linear_bwd(n, K, M, DT[dt], x, ldx, None, ACT[kind], pre, dy, ldy, None, K, dw, db, ws, wsb)
        want = (dz.t().contiguous() @ x.double().contiguous()).float()
        assert torch.equal(dw[:M], want), (n, (dw[:M] != want).nonzero()[:3].tolist())
        assert torch.equal(db[:M], dz.sum(0).float()), n
        assert (dw[M] == 0.5).all() and float(db[M]) == 0.5 and (ws[wsb:] == 0xFF).all()


@pytest.mark.parametrize("K,M,dt", [(272, 256, "bf16"), (257, 129, "bf16"), (64, 65, "f32"), (129, 200, "f32"), (1100, 520, "bf16")])
def test_linear_rows_and_their_gradients_are_exact_in_whole_numbers(K, M, dt):
    """The same of y and dx: at most 9 * 1100 < 2^24, in bf16 rounded once."""
    n = 33001
    print(f"[linear] whole rows K={K} M={M} {dt}", flush=True)
    x, w, dy = small(n, K, dt, 1, K + 3), small(M, K, dt, 2), small(n, M, dt, 3, M + 5)
    y, dx = (torch.full((n + 1, F), 0.5, dtype=tdtype(dt), device="cuda") for F in (M, K))
    fast.fast_linear_fwd(n, K, M, DT[dt], x, K + 3, w, None, 0, None, M, y, M)
    wsb = fast.fast_linear_bwd_workspace(n, K, M, DT[dt], 0)
    ws = torch.full((wsb + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    fast.fast_linear_bwd(n, K, M, DT[dt], None, K, w, 0, None, dy, M + 5, dx, K, None, None, ws, wsb)
    assert torch.equal(y[:n], (x.double().contiguous() @ w.double().t().contiguous()).to(tdtype(dt)))
    assert torch.equal(dx[:n], (dy.double().contiguous() @ w.double()).to(tdtype(dt)))
    assert (y[n] == 0.5).all() and (dx[n] == 0.5).all()
