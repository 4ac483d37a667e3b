"""The gated recurrence and infinite values: a segment that is cut carries them as one that is walked whole does."""
import numpy as np
import pytest
import torch

from tests.parity import tdtype
from tests.test_gpu_gated_scan_gates import both
from tests.test_gpu_layer import DT, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("span", [False, True])
@pytest.mark.parametrize("length", [60, 400, 9000])
def test_gated_scan_carries_an_infinity(dt, span, length):
    """Fast gates (a = 0.1 an event): over a piece of a long segment the product of a lies below every fp32
    number, yet an infinite state stays what it is, forward and back.  Gates that are 0 in fp32 forget it: then
    0 times an infinity is no number, in a segment of any length."""
    print(f"[scan] infinity {dt} span={span} {length}", flush=True)
    D = 5
    r = np.random.default_rng(length)
    xg = torch.from_numpy(r.normal(size=(length, 2, D)).astype(np.float32))
    xg[:, 1] = 2.1972
    xg[3, 0, 1], xg[3, 0, 2] = float("inf"), float("-inf")
    xg = xg.to(tdtype(dt))
    dh = torch.from_numpy(r.normal(size=(length, D)).astype(np.float32))
    at = length - 5
    dh[at, 3] = float("-inf")
    dh = dh.to(tdtype(dt))
    times = torch.ones(length).cuda() if span else None
    h, last, _, dxg, dh0 = (host(t) for t in both([0, length], xg.cuda(), times, None, dh.cuda(), None, DT[dt]))
    assert np.isfinite(h[:, [0, 3, 4]]).all() and np.isfinite(h[:3]).all()
    assert (h[3:, 1] == np.inf).all() and (h[3:, 2] == -np.inf).all()
    assert last[0, 1] == np.inf and last[0, 2] == -np.inf
    assert np.isfinite(dxg[:, 0, [0, 1, 2, 4]]).all() and np.isfinite(dxg[at + 1:, 0, 3]).all()
    assert (dxg[:at + 1, 0, 3] == -np.inf).all() and dh0[0, 3] == -np.inf
    # gates that are 0: the state after them is the event's own (here: no number, of 0 times the infinity)
    xg[length // 2, 1] = 200.0
    h, last, *_ = (host(t) for t in both([0, length], xg.cuda(), times, None, dh.cuda(), None, DT[dt]))
    assert (h[3:length // 2, 1] == np.inf).all() and np.isnan(h[length // 2:, 1]).all() and np.isnan(last[0, 1])
    assert np.isfinite(h[:, [0, 3, 4]]).all()
