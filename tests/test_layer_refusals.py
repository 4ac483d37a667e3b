"""Refusals of the layer operators that need no GPU: argument errors that the host can see are
returned before anything is enqueued."""
import ctypes

import pytest

import paper_2607_05095_amd as fast
from tests.test_layer_abi import ATT, BIG, CG, CW, FAKE, ROT, UNSUPPORTED, call


# ------------------------------------------------------------------ alignment
@pytest.mark.parametrize("name,defaults", [("fast_cache_write", CW), ("fast_cache_gather", CG)])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_a_misaligned_slot_map_is_refused(name, defaults, off):
    assert call(name, defaults, dict(map=FAKE + off)) == UNSUPPORTED


@pytest.mark.parametrize("kw,offsets", [(dict(map=FAKE + 2), FAKE), (dict(), FAKE + 1), (dict(), FAKE + 2)])
def test_cached_attention_refuses_misaligned_indices(kw, offsets):
    a = dict(ATT, **kw)
    a["g"] = ctypes.byref(fast.TCSR(4, 40, offsets, None, None, None, None))
    assert fast.lib().fast_edge_attention_fwd_cached(*a.values()) == UNSUPPORTED


# ------------------------------------------------------------------ spans
@pytest.mark.parametrize("name", ["fast_rotary_fwd", "fast_rotary_bwd"])
@pytest.mark.parametrize("kw", [dict(n=BIG - 1, ldx=BIG - 1, ldy=BIG - 1), dict(n=BIG - 1, ldx=BIG - 1),
                                dict(n=BIG - 1, ldy=BIG - 1), dict(n=1 << 30, ldx=1 << 30, ldy=1 << 30, dt=1)])
def test_rows_that_span_more_than_an_address_space_are_refused(name, kw):
    """Before their ends, which 64 bits may not hold, are compared."""
    a = dict(ROT, H=1, dh=2, pairs=1, ldx=2, ldy=2)
    a.update(kw)
    assert call(name, a, {}) == UNSUPPORTED
    assert "apart" in fast.fast_last_error()
