"""The gated recurrence's bits: a segment's results do not depend on what its neighbours' gates are."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests.parity import tdtype, to_dev
from tests.test_gpu_layer import DT

pytestmark = pytest.mark.gpu


def both(off, xg, dt, h0, dh, dlast, T):
    """forward and backward -> h, h_last, states, dxg, dh0"""
    E, _, D = xg.shape
    N = len(off) - 1
    blk = fast.tcsr(to_dev(np.asarray(off, np.int32)), E)
    new = lambda *s, t=torch.float32: torch.full(s, 7.0, dtype=t, device="cuda")
    h, last = new(E, D, t=xg.dtype), new(N, D)
    keep = torch.zeros(fast.fast_gated_scan_state_rows(E), D, device="cuda")
    dxg, dh0 = new(E, 2, D, t=xg.dtype), new(N, D)
    wsb = fast.fast_gated_scan_workspace(N, E, D)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda")
    x, g = xg[:, 0], xg[:, 1]
    fast.fast_gated_scan_fwd(blk, D, T, x, g, 2 * D, dt, h0, 0, h, last, keep, ws, wsb)
    fast.fast_gated_scan_bwd(blk, D, T, x, g, 2 * D, dt, h0, 0, keep, dh, dlast, dxg[:, 0], dxg[:, 1], 2 * D, dh0, ws, wsb)
    return h, last, keep, dxg, dh0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("length", [1, 9, 100, 300])
def test_gated_scan_bits_do_not_depend_on_neighbours(dt, length):
    """Ten equal segments beside each other in a wave (and, where they are cut, in workgroups of their own); in
    the second call every other one has gates so low that they are evaluated in another way."""
    print(f"[scan] neighbours {dt} {length}", flush=True)
    D, N = 12, 10
    E = N * length
    r = np.random.default_rng(length)
    f = lambda *s: torch.from_numpy(r.normal(size=s).astype(np.float32))
    xg = f(E, 2, D)
    xg[:, 1] *= 6
    span = torch.from_numpy(r.exponential(size=E).astype(np.float32))
    h0, dh, dl = f(N, D).cuda(), f(E, D).to(tdtype(dt)).cuda(), f(N, D).cuda()
    off = np.arange(N + 1) * length
    low = xg.clone()
    # (within a row too: every third column of the first event of the other segments)
    for v in range(1, N, 2):
        low[off[v]:off[v + 1], 1, ::3] = -90.0
    a, b = (both(off, t.to(tdtype(dt)).cuda(), span.cuda(), h0, dh, dl, DT[dt]) for t in (xg, low))
    same = torch.ones(E, D, dtype=torch.bool)
    rows = torch.ones(N, D, dtype=torch.bool)
    for v in range(1, N, 2):
        same[off[v]:off[v + 1], ::3] = False
        rows[v, ::3] = False
    same, rows = same.cuda(), rows.cuda()
    assert torch.equal(a[0][same], b[0][same]), "h"
    assert torch.equal(a[1][rows], b[1][rows]), "h_last"
    for k in (0, 1):
        assert torch.equal(a[3][:, k][same], b[3][:, k][same]), "dx or dgate"
    assert torch.equal(a[4][rows], b[4][rows]), "dh0"
