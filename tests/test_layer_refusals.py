"""Refusals of the layer operators that need no GPU: argument errors that the host can see are
returned before anything is enqueued."""
import ctypes

import pytest

import paper_2607_05095_amd as fast
from tests.test_layer_abi import (ATT, BIG, CG, CW, FAKE, INVALID, NORM, NORM_B, OK, ROT, UNSUPPORTED,
                                  call)


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


# ------------------------------------------------------------------ overlaps
NORM_BYTES = 5 * 10 * 4                          # rows of NORM and NORM_B


@pytest.mark.parametrize("kw", [
    dict(y=FAKE + 4), dict(y=FAKE - 4), dict(y=FAKE + NORM_BYTES - 4), dict(y=FAKE - NORM_BYTES + 4),
    dict(res=FAKE + 4096, y=FAKE + 4096 + 8), dict(res=FAKE + 4096, y=FAKE + 4096, sum=FAKE + 40),
    dict(res=FAKE + 4096, y=FAKE, sum=FAKE + 4096 + 40), dict(res=FAKE + 4096, y=FAKE + 8192, sum=FAKE + 8192 + 4),
    dict(res=FAKE + 4096, y=FAKE + 8192, sum=FAKE + 8192 - 4)])
def test_layer_norm_refuses_shifted_outputs(kw):
    """An output that lies across an input or the other output: rows read what other rows wrote."""
    assert call("fast_layer_norm_fwd", NORM, kw) == INVALID
    assert "overlap" in fast.fast_last_error()


@pytest.mark.parametrize("kw", [dict(dx=FAKE + 4), dict(dx=FAKE - NORM_BYTES + 4),
                                dict(dy=FAKE + 4096, dx=FAKE + 4096 + 4), dict(h=FAKE + 4096, dx=FAKE + 4096 - 4),
                                dict(dsum=FAKE + 4096, dx=FAKE + 4096 + NORM_BYTES - 4)])
def test_layer_norm_bwd_refuses_a_shifted_gradient(kw):
    assert call("fast_layer_norm_bwd", NORM_B, kw) == INVALID
    assert "overlap" in fast.fast_last_error()


def test_arrays_that_touch_do_not_overlap():
    """Nor do those in one place: such calls get as far as the limit of a launch."""
    n, D = BIG - 1, 500
    for y in (FAKE + n * D * 4, FAKE):
        assert call("fast_layer_norm_fwd", NORM, dict(n=n, D=D, y=y)) == UNSUPPORTED
        assert "threads" in fast.fast_last_error()
    assert call("fast_layer_norm_fwd", NORM, dict(n=n, D=D, y=FAKE + n * D * 4 - 4)) == INVALID
    assert call("fast_layer_norm_fwd", NORM, dict(n=0, y=FAKE + 4)) == OK


# ------------------------------------------------------------------ tensors
def test_rows_of_a_view_are_what_the_call_says():
    """_rows_as_said looks at shapes and strides alone; ctypes callers have no views."""
    import torch
    H, dh = 2, 6
    F = H * dh
    kv = torch.zeros(5, 2, H, dh)
    wide = torch.zeros(5, H, 2 * dh)
    good = [(kv, 2 * F), (kv[:, 1], 2 * F), (kv[:, :1], 2 * F), (kv[::2], 4 * F), (kv[:1, 1], 99), (kv[:, 1].flatten(1), 2 * F),
            (torch.zeros(5, 40)[:, :F], 40), (kv[:, 0].unflatten(0, (5, 1)), 2 * F), (torch.zeros(5, F), F)]
    for t, ld in good:
        fast._rows_as_said(t, F, ld)
    bad = [(kv[:, 0].transpose(1, 2), 2 * F),           # a head's elements apart
           (wide[..., :dh], 2 * F), (wide[..., ::2], 2 * F),
           (kv[:, 1].transpose(0, 1), 2 * F), (torch.zeros(5, 40)[:, :F], F), (kv[:, 1], F),
           (torch.zeros(F, 5).t(), F), (kv[:, 0].expand(5, H, dh)[:, :1].expand(5, H, dh), 2 * F)]
    for t, ld in bad:
        with pytest.raises(fast.FastError):
            fast._rows_as_said(t, F, ld)


def test_offsets_of_the_host_are_refused():
    """The graph's offsets live where the call's other tensors have to."""
    import torch
    g = fast.tcsr(torch.tensor([0, 3], dtype=torch.int32), 3)
    with pytest.raises(fast.FastError, match="not on the current GPU"):
        fast.fast_edge_attention_fwd_cached(g, 2, 50, fast.F32, FAKE, FAKE, 10, FAKE, fast.MXFP8, FAKE, 10, 1.0, 0.2,
                                            FAKE, None, FAKE, 1 << 20, 0)
