"""GPU parity of the cached rows at the ends of the number range: finite rows read back
finite, up to the largest value of either storage type."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64 as p64
from tests.parity import tdtype, to_dev

pytestmark = pytest.mark.gpu

DT = {"f32": fast.F32, "bf16": fast.BF16}
FMT = {8: fast.MXFP8, 4: fast.MXFP4}


def finite_codes(x, fmt):
    """p64.quantize, but of the codes whose value is below 2^128: the one next to it is the
    largest of those."""
    c, s = p64.quantize(x, fmt)
    over = np.abs(p64.values(c, s, fmt)) >= 2.0 ** 128
    return c - over.astype(np.uint8), s


@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_the_largest_finite_rows_read_back_finite(fmt, dt):
    print(f"[cache] largest rows fmt={fmt} {dt}", flush=True)
    top = float(torch.finfo(tdtype(dt)).max)
    # the largest value, the borders between the codes below 2^128, and ordinary values beside them
    v = [top, 255 * 2.0 ** 120, 252 * 2.0 ** 120, 248 * 2.0 ** 120, 247 * 2.0 ** 120, 244 * 2.0 ** 120,
         240 * 2.0 ** 120, 232 * 2.0 ** 120, 225 * 2.0 ** 120, 224 * 2.0 ** 120, 223 * 2.0 ** 120, 7 * 2.0 ** 125,
         1.5 * 2.0 ** 127, 1.51 * 2.0 ** 127, 1.25 * 2.0 ** 127, 2.0 ** 127, 2.0 ** 126, 0.0]
    n, parts, width = 2 * len(v), 3, 70
    x = np.random.default_rng(fmt).normal(size=(n, parts, width)) * 2.0 ** 118
    for i, a in enumerate(v):                     # in a whole group, a short one, and filling a group
        x[2 * i, 0, 5], x[2 * i, 1, 69], x[2 * i, 2, 32:64] = a, -a, a
        x[2 * i + 1, 0, 40], x[2 * i + 1, 1, 64], x[2 * i + 1, 2, :32] = -a, a, -a
    src = torch.from_numpy(x.astype(np.float32)).to(tdtype(dt))
    s64 = src.double().numpy()
    assert np.isfinite(s64).all()
    c, s = finite_codes(s64, fmt)
    cache = torch.zeros(n, p64.record(parts, width, fmt)[3], dtype=torch.uint8, device="cuda")
    ids = torch.arange(n, device="cuda")
    fast.fast_cache_write(ids, n, n, None, parts, width, DT[dt], src.cuda(), FMT[fmt], cache, n, True)
    np.testing.assert_array_equal(cache.cpu().numpy(), p64.pack(c, s, fmt))
    want = p64.values(c, s, fmt)
    # at most the larger of a share of the value and half the smallest step
    step = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, -1)[..., :width]
    half = np.maximum(np.abs(s64) / 16, step / 1024) if fmt == 8 else np.maximum(np.abs(s64) / 4, step / 4)
    assert (np.abs(want - s64) <= half).all()
    for od in ("f32", "bf16"):
        out = torch.empty(n, parts, width, dtype=tdtype(od), device="cuda")
        fast.fast_cache_gather(ids, n, n, None, parts, width, FMT[fmt], cache, n, DT[od], out)
        assert torch.isfinite(out).all()
        np.testing.assert_array_equal(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("fmt", [8, 4])
def test_attention_over_the_largest_finite_rows(fmt):
    """One edge a segment returns its V row, whatever its size."""
    H, dh, n = 2, 50, 6
    kv = torch.zeros(n, 2 * H, dh)
    kv[:, H:] = torch.finfo(torch.float32).max * torch.tensor([1.0, -1.0, 0.5, 0.97, -0.99, 0.3])[:, None, None]
    c, s = finite_codes(kv.double().numpy(), fmt)
    cache = torch.zeros(n, fast.fast_cache_row_bytes(2 * H, dh, FMT[fmt]), dtype=torch.uint8, device="cuda")
    ids = torch.arange(n, device="cuda")
    fast.fast_cache_write(ids, n, n, None, 2 * H, dh, fast.F32, kv.cuda(), FMT[fmt], cache, n, True)
    g = fast.tcsr(torch.arange(n + 1, dtype=torch.int32, device="cuda"), n)
    wsb = fast.fast_edge_attention_cached_workspace(n, n, H, dh)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    out = torch.empty(n, H, dh, device="cuda")
    fast.fast_edge_attention_fwd_cached(g, H, dh, fast.F32, torch.ones(n, H, dh, device="cuda"), ids, n, None,
                                        FMT[fmt], cache, n, 1.0, 0.2, out, None, ws, wsb)
    np.testing.assert_array_equal(out.double().cpu().numpy(), p64.values(c, s, fmt)[:, H:])
