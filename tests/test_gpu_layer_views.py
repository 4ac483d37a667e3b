"""Tensors that are not laid out as a call reads them are refused by the binding, whatever the
argument: transposed and sliced ones, and rows that are not as far apart as the call says."""
import pytest
import torch

import paper_2607_05095_amd as fast

pytestmark = pytest.mark.gpu

N, D, H, DH, E = 6, 12, 2, 6, 9


def dense(dtype, *shape):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def spread(t):
    """The same shape, every second element of a larger array."""
    return torch.zeros(*t.shape, 2, dtype=t.dtype, device=t.device)[..., 0]


def calls():
    f, i32, i64, u8 = torch.float32, torch.int32, torch.int64, torch.uint8
    row = fast.fast_cache_row_bytes(2 * H, DH, fast.MXFP8)
    wsb = fast.fast_edge_attention_cached_workspace(N, E, H, DH)
    lnb = fast.fast_layer_norm_bwd_workspace(N, D)
    cwb = fast.fast_cache_write_workspace(N, 8)
    g = fast.tcsr(dense(i32, N + 1), E)
    return {
        "norm": (fast.fast_layer_norm_fwd, [N, D, 0, dense(f, N, D), dense(f, N, D), dense(f, D), dense(f, D), 1e-5,
                                            dense(f, N, D), dense(f, N, D), dense(f, N), dense(f, N)]),
        "norm bwd": (fast.fast_layer_norm_bwd, [N, D, 0, dense(f, N, D), dense(f, D), dense(f, N), dense(f, N),
                                                dense(f, N, D), dense(f, N, D), dense(f, N, D), dense(f, D),
                                                dense(f, D), dense(u8, lnb), lnb]),
        "rotary": (fast.fast_rotary_fwd, [N, H, DH, 0, dense(f, N, D), D, dense(f, N, 1), 1, dense(i32, 3),
                                          dense(f, 3), 3, 0, dense(f, N, D), D]),
        "rotary bwd": (fast.fast_rotary_bwd, [N, H, DH, 0, dense(f, N, D), D, dense(f, N, 1), 1, dense(i32, 3),
                                              dense(f, 3), 3, 0, dense(f, N, D), D]),
        "write": (fast.fast_cache_write, [dense(i64, N), N, 8, dense(i32, 8), 2 * H, DH, 0, dense(f, N, 2 * H, DH),
                                          fast.MXFP8, dense(u8, 8, row), 8, False, dense(u8, cwb), cwb]),
        "gather": (fast.fast_cache_gather, [dense(i64, N), N, 8, dense(i32, 8), 2 * H, DH, fast.MXFP8,
                                            dense(u8, 8, row), 8, 0, dense(f, N, 2 * H, DH)]),
        "attention": (fast.fast_edge_attention_fwd_cached, [g, H, DH, 0, dense(f, N, H, DH), dense(i64, E), 8,
                                                            dense(i32, 8), fast.MXFP8, dense(u8, 8, row), 8, 1.0, 0.2,
                                                            dense(f, N, H, DH), dense(f, N, H), dense(u8, wsb), wsb]),
    }


@pytest.mark.parametrize("name", ["norm", "norm bwd", "rotary", "rotary bwd", "write", "gather", "attention"])
def test_every_argument_that_is_not_laid_out_as_read_is_refused(name):
    f, args = calls()[name]
    f(*args)                                         # as they are: fine
    tensors = [k for k, t in enumerate(args) if torch.is_tensor(t)]
    assert len(tensors) >= 4
    for k in tensors:
        for bad in (spread(args[k]), args[k].cpu()):
            with pytest.raises(fast.FastError):
                f(*args[:k], bad, *args[k + 1:])
    torch.cuda.synchronize()


def test_offsets_and_transposed_rows_are_refused():
    f, args = calls()["attention"]
    for off in (torch.zeros(N + 1, 2, dtype=torch.int32, device="cuda")[:, 0], torch.zeros(N + 1, dtype=torch.int32)):
        with pytest.raises(fast.FastError):
            f(fast.tcsr(off, E), *args[1:])
    for name in ("rotary", "rotary bwd"):
        f, args = calls()[name]
        for k in (4, 12):
            for bad in (torch.zeros(D, N, device="cuda").t(), torch.zeros(N, 2 * D, device="cuda")[:, :D],
                        torch.zeros(N, DH, H, device="cuda").transpose(1, 2)):
                with pytest.raises(fast.FastError):
                    f(*args[:k], bad, *args[k + 1:])
        kv = torch.randn(N, 2, D, device="cuda")     # rows of a view, as far apart as the call says
        x = kv[:, 1].clone()
        f(*args[:4], kv[:, 1], 2 * D, *args[6:12], kv[:, 1], 2 * D)
        assert torch.equal(kv[:, 1], x)              # by angles of zero
