"""Thin Python binding of libfast.so, the gfx950 temporal-subgraph operators.

Every function has the name and argument order of the C entry point in
include/fast.h.  Arguments are torch tensors resident on the GPU (or None
for optional pointers); the binding only marshals pointers, sizes and the
current HIP stream, and raises FastError for a non-OK status.  All
computation happens in the HIP kernels; there is no fallback path: if the
library is missing the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os

__all__ = [
    "FastError", "lib", "TCSR", "tcsr", "TemporalGraphDesc", "temporal_graph", "F32", "BF16",
    "dtype_of", "fast_sample_recent_workspace", "fast_sample_recent",
    "fast_version", "fast_last_error",
    "fast_csr_offsets_workspace", "fast_csr_offsets", "fast_check_tcsr",
    "fast_csr_offsets_batched_workspace", "fast_csr_offsets_batched", "fast_time_encode_batched",
    "fast_dedup_gather_workspace", "fast_dedup_gather", "fast_dedup_gather_noalloc",
    "NOALLOC_SCRATCH_BYTES",
    "fast_access_count_workspace", "fast_access_count",
    "fast_greedy_hot_set_workspace", "fast_greedy_hot_set", "fast_hot_set_budget",
    "fast_time_encode", "fast_time_encode_bwd_workspace", "fast_time_encode_bwd",
    "fast_edge_softmax_fwd", "fast_edge_softmax_bwd",
    "fast_temporal_aggregate_fwd", "fast_temporal_aggregate_bwd",
    "fast_edge_attention_fwd", "fast_edge_attention_bwd",
    "fast_edge_attention_fwd_packed", "fast_edge_attention_bwd_packed",
    "fast_edge_attention_fwd_indexed", "fast_edge_attention_bwd_indexed",
    "fast_occurrence_csr_workspace", "fast_occurrence_csr",
    "fast_index_add_rows_workspace", "fast_index_add_rows",
    "fast_edge_attention_bwd_indexed_coef",
    "fast_index_add_scaled_rows_workspace", "fast_index_add_scaled_rows",
    "fast_layer_norm_fwd", "fast_layer_norm_bwd_workspace", "fast_layer_norm_bwd",
    "fast_rotary_fwd", "fast_rotary_bwd", "MXFP8", "MXFP4", "fast_cache_row_bytes",
    "fast_cache_write_workspace", "fast_cache_write", "fast_cache_gather",
    "fast_edge_attention_cached_workspace", "fast_edge_attention_fwd_cached",
    "ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_SILU", "fast_linear_fwd", "fast_linear_bwd_workspace",
    "fast_linear_bwd", "fast_gated_scan_state_rows", "fast_gated_scan_workspace",
    "fast_gated_scan_fwd", "fast_gated_scan_bwd", "STATE_F32", "STATE_MXFP8", "AdamWTensor",
    "adamw_tensors", "fast_adamw", "fast_grad_norm_workspace", "fast_grad_norm",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; FAST_LIB names another build of the same sources (the
# sanitizer build of the host code)
LIB_PATH = os.environ.get("FAST_LIB") or os.path.join(_HERE, "libfast.so")

F32, BF16 = 0, 1
MXFP8, MXFP4 = 0, 1   # fast_cache_format_t
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3   # fast_act_t
STATE_F32, STATE_MXFP8 = 0, 1   # fast_state_format_t
NOALLOC_SCRATCH_BYTES = 128 << 20   # FAST_NOALLOC_SCRATCH_BYTES of include/fast.h
_STATUS = {0: "FAST_OK", 1: "FAST_ERR_INVALID_ARG", 2: "FAST_ERR_UNSUPPORTED",
           3: "FAST_ERR_WORKSPACE", 4: "FAST_ERR_HIP"}


class FastError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class TCSR(C.Structure):
    """fast_tcsr_t: a sampled temporal subgraph of one layer block (device pointers)."""
    _fields_ = [
        ("num_dst", C.c_int64),
        ("num_edges", C.c_int64),
        ("dst_offsets", C.c_void_p),
        ("src_ids", C.c_void_p),
        ("edge_t", C.c_void_p),
        ("edge_ids", C.c_void_p),
        ("dst_t", C.c_void_p),
    ]


class TemporalGraphDesc(C.Structure):
    """fast_temporal_graph_t: a T-CSR temporal graph (device pointers)."""
    _fields_ = [
        ("num_nodes", C.c_int64),
        ("num_entries", C.c_int64),
        ("indptr", C.c_void_p),
        ("nbr", C.c_void_p),
        ("ts", C.c_void_p),
        ("eid", C.c_void_p),
    ]


class AdamWTensor(C.Structure):
    """fast_adamw_tensor_t: one tensor of an AdamW step (device pointers)."""
    _fields_ = [
        ("w", C.c_void_p),
        ("grad", C.c_void_p),
        ("m", C.c_void_p),
        ("v", C.c_void_p),
        ("m_scale", C.c_void_p),
        ("v_scale", C.c_void_p),
        ("copy", C.c_void_p),
        ("n", C.c_int64),
        ("decay", C.c_float),
    ]


_p, _i64, _i32, _f32, _sz = C.c_void_p, C.c_int64, C.c_int, C.c_float, C.c_size_t
_f64 = C.c_double
_G = C.POINTER(TCSR)
_TG = C.POINTER(TemporalGraphDesc)
_SIGS = {
    "fast_last_error": (C.c_char_p, []),
    "fast_version": (C.c_char_p, []),
    "fast_csr_offsets_workspace": (_sz, [_i64]),
    "fast_csr_offsets": (_i32, [_p, _i64, _p, _p, _sz, _p]),
    "fast_csr_offsets_batched_workspace": (_sz, [_i32, _p]),
    "fast_csr_offsets_batched": (_i32, [_i32, _p, _p, _p, _p, _sz, _p]),
    "fast_time_encode_batched": (_i32, [_i32, _p, _p, _p, _i32, _p, _i32, _p]),
    "fast_check_tcsr": (_i32, [_G, _i64, _i64, _p, _p]),
    "fast_dedup_gather_workspace": (_sz, [_i64, _i64]),
    "fast_dedup_gather": (_i32, [_p, _i64, _i64, _p, _i64, _i32, _i32, _p, _p, _p, _p,
                                 _p, _p, _p, _p, _sz, _p]),
    "fast_dedup_gather_noalloc": (_i32, [_p, _i64, _i64, _p, _i64, _i32, _i32, _p, _p, _p, _p,
                                         _p, _p, _p, _p]),
    "fast_sample_recent_workspace": (_sz, [_i64]),
    "fast_sample_recent": (_i32, [_TG, _p, _p, _i64, _i32, _p, _p, _p, _p, _p, _sz, _p]),
    "fast_access_count_workspace": (_sz, [_i64]),
    "fast_access_count": (_i32, [_p, _p, _i64, _i64, _p, _p, _sz, _p]),
    "fast_greedy_hot_set_workspace": (_sz, [_i64, _i64, _i32]),
    "fast_hot_set_budget": (_i32, [C.c_double, _i64, _i64, _p]),
    "fast_greedy_hot_set": (_i32, [_p, _i64, _p, _i64, _i32, _i64, _p, _p, _p, _p, _p, _p, _p,
                                   _sz, _p]),
    "fast_time_encode": (_i32, [_G, _p, _p, _i32, _p, _i32, _p]),
    "fast_time_encode_bwd_workspace": (_sz, [_i64, _i32]),
    "fast_time_encode_bwd": (_i32, [_G, _p, _p, _i32, _p, _i32, _p, _p, _p, _sz, _p]),
    "fast_edge_softmax_fwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _f32, _f32, _p, _p, _p]),
    "fast_edge_softmax_bwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _f32, _f32, _p, _p, _p, _p, _p]),
    "fast_temporal_aggregate_fwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _p]),
    "fast_temporal_aggregate_bwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _p, _p, _p]),
    "fast_edge_attention_fwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _f32, _f32, _p, _p, _p]),
    "fast_edge_attention_bwd": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _f32, _f32, _p, _p,
                                       _p, _p, _p, _p]),
    "fast_edge_attention_fwd_packed": (_i32, [_G, _i32, _i32, _i32, _p, _p, _f32, _f32, _p, _p, _p]),
    "fast_edge_attention_bwd_packed": (_i32, [_G, _i32, _i32, _i32, _p, _p, _f32, _f32, _p, _p, _p,
                                              _p, _p]),
    "fast_edge_attention_fwd_indexed": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _i64, _p, _p,
                                               _i64, _f32, _f32, _p, _p, _p]),
    "fast_edge_attention_bwd_indexed": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _i64, _p, _p,
                                               _i64, _f32, _f32, _p, _p, _p, _p, _p, _p]),
    "fast_occurrence_csr_workspace": (_sz, [_i64, _i64]),
    "fast_occurrence_csr": (_i32, [_p, _i64, _i64, _p, _p, _p, _sz, _p]),
    "fast_index_add_rows_workspace": (_sz, [_i64, _i64, _i32]),
    "fast_index_add_rows": (_i32, [_p, _p, _i64, _i64, _i32, _i32, _p, _p, _p, _sz, _p]),
    "fast_edge_attention_bwd_indexed_coef": (_i32, [_G, _i32, _i32, _i32, _p, _p, _p, _i64, _p, _p,
                                                    _i64, _f32, _f32, _p, _p, _p, _p, _p, _p]),
    "fast_index_add_scaled_rows_workspace": (_sz, [_i64, _i64, _i32, _i32]),
    "fast_index_add_scaled_rows": (_i32, [_p, _p, _i64, _i64, _p, _i64, _i32, _i32, _i32, _p, _p,
                                          _p, _p, _sz, _p]),
    "fast_layer_norm_fwd": (_i32, [_i64, _i32, _i32, _p, _p, _p, _p, _f32, _p, _p, _p, _p, _p]),
    "fast_layer_norm_bwd_workspace": (_sz, [_i64, _i32]),
    "fast_layer_norm_bwd": (_i32, [_i64, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _sz,
                                   _p]),
    "fast_rotary_fwd": (_i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _i32, _p, _p, _i32, _i32, _p,
                               _i64, _p]),
    "fast_rotary_bwd": (_i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _i32, _p, _p, _i32, _i32, _p,
                               _i64, _p]),
    "fast_cache_row_bytes": (_sz, [_i32, _i32, _i32]),
    "fast_cache_write_workspace": (_sz, [_i64, _i64]),
    "fast_cache_write": (_i32, [_p, _i64, _i64, _p, _i32, _i32, _i32, _p, _i32, _p, _i64, _i32, _p,
                                _sz, _p]),
    "fast_cache_gather": (_i32, [_p, _i64, _i64, _p, _i32, _i32, _i32, _p, _i64, _i32, _p, _p]),
    "fast_edge_attention_cached_workspace": (_sz, [_i64, _i64, _i32, _i32]),
    "fast_edge_attention_fwd_cached": (_i32, [_G, _i32, _i32, _i32, _p, _p, _i64, _p, _i32, _p,
                                              _i64, _f32, _f32, _p, _p, _p, _sz, _p]),
    "fast_linear_fwd": (_i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _p, _i32, _p, _i64, _p, _i64, _p,
                               _p]),
    "fast_linear_bwd_workspace": (_sz, [_i64, _i32, _i32, _i32, _i32]),
    "fast_linear_bwd": (_i32, [_i64, _i32, _i32, _i32, _p, _i64, _p, _i32, _p, _p, _i64, _p, _i64, _p,
                               _p, _p, _sz, _p]),
    "fast_gated_scan_state_rows": (_i64, [_i64]),
    "fast_gated_scan_workspace": (_sz, [_i64, _i64, _i32]),
    "fast_gated_scan_fwd": (_i32, [_G, _i32, _i32, _p, _p, _i64, _p, _p, _i64, _p, _p, _p, _p, _sz,
                                   _p]),
    "fast_gated_scan_bwd": (_i32, [_G, _i32, _i32, _p, _p, _i64, _p, _p, _i64, _p, _p, _p, _p, _p,
                                   _i64, _p, _p, _sz, _p]),
    "fast_adamw": (_i32, [_p, _i32, _i32, _i32, _f64, _f64, _f64, _f64, _i64, C.c_uint32, _p, _p, _p,
                          _p]),
    "fast_grad_norm_workspace": (_sz, [_i64, _i32]),
    "fast_grad_norm": (_i32, [_p, _i32, _i32, _f32, _p, _p, _p, _sz, _p]),
}

_lib = None


def lib():
    """Load libfast.so (built in-tree by build.py); raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FastError(-1, f"{LIB_PATH} is not built; run python -m paper_2607_05095_amd.build")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    # the raw handle of torch.cuda.current_stream(), without building a Stream object (2.8 -> 0.4 us a call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(st: int):
    if st != 0:
        raise FastError(st, fast_last_error())


def _rows_as_said(t, F, ld):
    """A view's rows are F elements side by side, ld apart; raises otherwise."""
    if t.dim() == 2 and t.shape[1] == F and t.stride() == (ld, 1):
        return
    side = 1                             # elements side by side, from the last dimension on
    outer = []
    for size, step in zip(reversed(t.shape), reversed(t.stride())):
        if size == 1:
            continue
        if side < F:
            if step != side:
                break
            side *= size
        else:
            outer.append(step)
    if side < F or (len(outer) == 1 and outer[0] != ld):
        raise FastError(1, f"tensor of shape {tuple(t.shape)}, strides {tuple(t.stride())}: its rows "
                           f"are not {F} elements side by side, {ld} apart")


def _resident(dense=(), rows=()):
    """Tensors of a call live on the current device, and are contiguous or, as (tensor, stride, F) in
    `rows`, views of rows of F elements that far apart; raises otherwise."""
    import torch
    dev = None                           # (asked of the runtime directly: with a tensor there it is up)
    for t in dense:
        if t is None or isinstance(t, int):
            continue
        if dev is None and t.is_cuda:
            dev = torch._C._cuda_getDevice()
        if t.get_device() != dev:
            raise FastError(1, f"tensor on {t.device}, not on the current GPU")
        if not t.is_contiguous():
            raise FastError(1, f"tensor of shape {tuple(t.shape)} is not contiguous")
    for t, ld, F in rows:
        if t is None or isinstance(t, int):
            continue
        if dev is None and t.is_cuda:
            dev = torch._C._cuda_getDevice()
        if t.get_device() != dev:
            raise FastError(1, f"tensor on {t.device}, not on the current GPU")
        if not t.is_contiguous():        # contiguous tensors hold rows of any stride
            _rows_as_said(t, F, ld)


def dtype_of(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise FastError(2, f"unsupported tensor dtype {t.dtype}")


def tcsr(dst_offsets, num_edges: int, src_ids=None, edge_t=None, edge_ids=None, dst_t=None) -> TCSR:
    """Builds a fast_tcsr_t over device tensors.  The struct keeps a reference
    to each tensor, so a temporary passed here (`x.cuda()`) is not returned to
    torch's caching allocator, and reused, while the struct is alive."""
    g = TCSR(dst_offsets.shape[0] - 1, int(num_edges), _ptr(dst_offsets), _ptr(src_ids),
             _ptr(edge_t), _ptr(edge_ids), _ptr(dst_t))
    g._keep = tuple(t for t in (dst_offsets, src_ids, edge_t, edge_ids, dst_t)
                    if t is not None and not isinstance(t, int))
    return g


def temporal_graph(indptr, nbr, ts, eid) -> TemporalGraphDesc:
    """Builds a fast_temporal_graph_t over device tensors; the struct keeps a
    reference to each tensor while it is alive."""
    g = TemporalGraphDesc(indptr.shape[0] - 1, int(nbr.shape[0]), _ptr(indptr), _ptr(nbr),
                          _ptr(ts), _ptr(eid))
    g._keep = (indptr, nbr, ts, eid)
    return g


# ------------------------------------------------------------------ entry points
def fast_last_error() -> str:
    return lib().fast_last_error().decode()


def fast_version() -> str:
    return lib().fast_version().decode()


def fast_csr_offsets_workspace(n: int) -> int:
    return lib().fast_csr_offsets_workspace(n)


def fast_csr_offsets(counts, n, offsets, ws, ws_bytes, stream=None):
    _check(lib().fast_csr_offsets(_ptr(counts), n, _ptr(offsets), _ptr(ws), ws_bytes,
                                  _stream(stream)))


def _host_ptrs(xs):
    """A host array of device pointers (None for a NULL entry)."""
    return (C.c_void_p * max(len(xs), 1))(*[_ptr(x) for x in xs])


def _host_i64(xs):
    return (C.c_int64 * max(len(xs), 1))(*[int(x) for x in xs])


def fast_csr_offsets_batched_workspace(n) -> int:
    return lib().fast_csr_offsets_batched_workspace(len(n), _host_i64(n))


def fast_csr_offsets_batched(counts, n, offsets, ws, ws_bytes, stream=None):
    """counts, n, offsets: sequences of equal length (one entry per block)."""
    if not (len(counts) == len(n) == len(offsets)):
        raise ValueError("counts, n and offsets must have one entry per block")
    _check(lib().fast_csr_offsets_batched(len(n), _host_ptrs(counts), _host_i64(n),
                                          _host_ptrs(offsets), _ptr(ws), ws_bytes,
                                          _stream(stream)))


def fast_time_encode_batched(graphs, omega, phi, d_t, te, te_dtype, stream=None):
    """graphs: TCSR descriptors, te: outputs, one per block."""
    if len(graphs) != len(te):
        raise ValueError("graphs and te must have one entry per block")
    gs = (C.POINTER(TCSR) * max(len(graphs), 1))(*[C.pointer(g) for g in graphs])
    _check(lib().fast_time_encode_batched(len(graphs), gs, _ptr(omega), _ptr(phi), d_t,
                                          _host_ptrs(te), te_dtype, _stream(stream)))


def fast_check_tcsr(g: TCSR, src_bound, edge_bound, violations, stream=None):
    _check(lib().fast_check_tcsr(C.byref(g), src_bound, edge_bound, _ptr(violations),
                                 _stream(stream)))


def fast_dedup_gather_workspace(n: int, id_bound: int) -> int:
    return lib().fast_dedup_gather_workspace(n, id_bound)


def fast_dedup_gather(ids, n, id_bound, table, table_rows, D, dtype, slot_map, uni, inv,
                      num_unique, rows, miss, num_miss, ws, ws_bytes, stream=None):
    _check(lib().fast_dedup_gather(_ptr(ids), n, id_bound, _ptr(table), table_rows, D, dtype,
                                   _ptr(slot_map), _ptr(uni), _ptr(inv), _ptr(num_unique),
                                   _ptr(rows), _ptr(miss), _ptr(num_miss), _ptr(ws), ws_bytes,
                                   _stream(stream)))


def fast_dedup_gather_noalloc(ids, n, id_bound, table, table_rows, D, dtype, slot_map, uni, inv,
                              num_unique, rows, miss, num_miss, stream=None):
    _check(lib().fast_dedup_gather_noalloc(_ptr(ids), n, id_bound, _ptr(table), table_rows, D,
                                           dtype, _ptr(slot_map), _ptr(uni), _ptr(inv),
                                           _ptr(num_unique), _ptr(rows), _ptr(miss),
                                           _ptr(num_miss), _stream(stream)))


def fast_sample_recent_workspace(num_roots: int) -> int:
    return lib().fast_sample_recent_workspace(num_roots)


def fast_sample_recent(g: TemporalGraphDesc, roots, root_t, num_roots, k, dst_offsets, src_ids,
                       edge_t, edge_ids, ws, ws_bytes, stream=None):
    _check(lib().fast_sample_recent(C.byref(g), _ptr(roots), _ptr(root_t), num_roots, k,
                                    _ptr(dst_offsets), _ptr(src_ids), _ptr(edge_t),
                                    _ptr(edge_ids), _ptr(ws), ws_bytes, _stream(stream)))


def fast_access_count_workspace(id_bound: int) -> int:
    return lib().fast_access_count_workspace(id_bound)


def fast_access_count(ids, batch_offsets, num_batches, id_bound, freq, ws, ws_bytes, stream=None):
    """batch_offsets: a host sequence of num_batches + 1 int64 offsets into ids."""
    offs = (C.c_int64 * (num_batches + 1))(*[int(x) for x in batch_offsets])
    _check(lib().fast_access_count(_ptr(ids), C.cast(offs, C.c_void_p), num_batches, id_bound,
                                   _ptr(freq), _ptr(ws), ws_bytes, _stream(stream)))


def fast_greedy_hot_set_workspace(num_nodes: int, num_edges: int, max_freq: int) -> int:
    return lib().fast_greedy_hot_set_workspace(num_nodes, num_edges, max_freq)


def fast_greedy_hot_set(freq_v, num_nodes, freq_e, num_edges, max_freq, budget, hot_v, num_hot_v,
                        slot_v, hot_e, num_hot_e, slot_e, ws, ws_bytes, stream=None):
    _check(lib().fast_greedy_hot_set(_ptr(freq_v), num_nodes, _ptr(freq_e), num_edges, max_freq,
                                     budget, _ptr(hot_v), _ptr(num_hot_v), _ptr(slot_v),
                                     _ptr(hot_e), _ptr(num_hot_e), _ptr(slot_e), _ptr(ws),
                                     ws_bytes, _stream(stream)))


def fast_hot_set_budget(alpha: float, num_nodes: int, num_edges: int) -> int:
    """Returns the budget the library computes (a host call)."""
    out = C.c_int64(0)
    _check(lib().fast_hot_set_budget(float(alpha), num_nodes, num_edges, C.byref(out)))
    return out.value


def fast_time_encode(g: TCSR, omega, phi, d_t, te, te_dtype, stream=None):
    _check(lib().fast_time_encode(C.byref(g), _ptr(omega), _ptr(phi), d_t, _ptr(te), te_dtype,
                                  _stream(stream)))


def fast_time_encode_bwd_workspace(num_dst: int, d_t: int) -> int:
    return lib().fast_time_encode_bwd_workspace(num_dst, d_t)


def fast_time_encode_bwd(g: TCSR, omega, phi, d_t, dte, dte_dtype, domega, dphi, ws, ws_bytes,
                         stream=None):
    _check(lib().fast_time_encode_bwd(C.byref(g), _ptr(omega), _ptr(phi), d_t, _ptr(dte),
                                      dte_dtype, _ptr(domega), _ptr(dphi), _ptr(ws), ws_bytes,
                                      _stream(stream)))


def fast_edge_softmax_fwd(g: TCSR, H, dh, dtype, Q, K, scale, neg_slope, alpha, lse, stream=None):
    _check(lib().fast_edge_softmax_fwd(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K), scale,
                                       neg_slope, _ptr(alpha), _ptr(lse), _stream(stream)))


def fast_edge_softmax_bwd(g: TCSR, H, dh, dtype, Q, K, scale, neg_slope, alpha, dalpha, dQ, dK,
                          stream=None):
    _check(lib().fast_edge_softmax_bwd(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K), scale,
                                       neg_slope, _ptr(alpha), _ptr(dalpha), _ptr(dQ), _ptr(dK),
                                       _stream(stream)))


def fast_temporal_aggregate_fwd(g: TCSR, H, dh, dtype, alpha, V, out, stream=None):
    _check(lib().fast_temporal_aggregate_fwd(C.byref(g), H, dh, dtype, _ptr(alpha), _ptr(V),
                                             _ptr(out), _stream(stream)))


def fast_temporal_aggregate_bwd(g: TCSR, H, dh, dtype, alpha, V, dout, dalpha, dV, stream=None):
    _check(lib().fast_temporal_aggregate_bwd(C.byref(g), H, dh, dtype, _ptr(alpha), _ptr(V),
                                             _ptr(dout), _ptr(dalpha), _ptr(dV), _stream(stream)))


def fast_edge_attention_fwd(g: TCSR, H, dh, dtype, Q, K, V, scale, neg_slope, out, lse,
                            stream=None):
    _check(lib().fast_edge_attention_fwd(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K), _ptr(V),
                                         scale, neg_slope, _ptr(out), _ptr(lse), _stream(stream)))


def fast_edge_attention_bwd(g: TCSR, H, dh, dtype, Q, K, V, scale, neg_slope, lse, dout, dQ, dK,
                            dV, stream=None):
    _check(lib().fast_edge_attention_bwd(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K), _ptr(V),
                                         scale, neg_slope, _ptr(lse), _ptr(dout), _ptr(dQ),
                                         _ptr(dK), _ptr(dV), _stream(stream)))


def fast_edge_attention_fwd_packed(g: TCSR, H, dh, dtype, Q, KV, scale, neg_slope, out, lse,
                                   stream=None):
    _check(lib().fast_edge_attention_fwd_packed(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(KV),
                                                scale, neg_slope, _ptr(out), _ptr(lse),
                                                _stream(stream)))


def fast_edge_attention_bwd_packed(g: TCSR, H, dh, dtype, Q, KV, scale, neg_slope, lse, dout, dQ,
                                   dKV, stream=None):
    _check(lib().fast_edge_attention_bwd_packed(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(KV),
                                                scale, neg_slope, _ptr(lse), _ptr(dout),
                                                _ptr(dQ), _ptr(dKV), _stream(stream)))


def fast_edge_attention_fwd_indexed(g: TCSR, H, dh, dtype, Q, K, k_index, k_rows, V, v_index,
                                    v_rows, scale, neg_slope, out, lse, stream=None):
    _check(lib().fast_edge_attention_fwd_indexed(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K),
                                                 _ptr(k_index), k_rows, _ptr(V), _ptr(v_index),
                                                 v_rows, scale, neg_slope, _ptr(out), _ptr(lse),
                                                 _stream(stream)))


def fast_edge_attention_bwd_indexed(g: TCSR, H, dh, dtype, Q, K, k_index, k_rows, V, v_index,
                                    v_rows, scale, neg_slope, lse, dout, dQ, dK_edge, dV_edge,
                                    stream=None):
    _check(lib().fast_edge_attention_bwd_indexed(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K),
                                                 _ptr(k_index), k_rows, _ptr(V), _ptr(v_index),
                                                 v_rows, scale, neg_slope, _ptr(lse), _ptr(dout),
                                                 _ptr(dQ), _ptr(dK_edge), _ptr(dV_edge),
                                                 _stream(stream)))


def fast_occurrence_csr_workspace(n: int, num_rows: int) -> int:
    return lib().fast_occurrence_csr_workspace(n, num_rows)


def fast_occurrence_csr(index, n, num_rows, occ_off, occ, ws, ws_bytes, stream=None):
    _check(lib().fast_occurrence_csr(_ptr(index), n, num_rows, _ptr(occ_off), _ptr(occ), _ptr(ws),
                                     ws_bytes, _stream(stream)))


def fast_index_add_rows_workspace(n: int, num_rows: int, D: int) -> int:
    return lib().fast_index_add_rows_workspace(n, num_rows, D)


def fast_index_add_rows(occ_off, occ, n, num_rows, D, src_dtype, src, dst, ws, ws_bytes,
                        stream=None):
    _check(lib().fast_index_add_rows(_ptr(occ_off), _ptr(occ), n, num_rows, D, src_dtype, _ptr(src),
                                     _ptr(dst), _ptr(ws), ws_bytes, _stream(stream)))


def fast_edge_attention_bwd_indexed_coef(g: TCSR, H, dh, dtype, Q, K, k_index, k_rows, V, v_index,
                                         v_rows, scale, neg_slope, lse, dout, dQ, g_edge,
                                         alpha_edge, stream=None):
    _check(lib().fast_edge_attention_bwd_indexed_coef(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(K),
                                                      _ptr(k_index), k_rows, _ptr(V),
                                                      _ptr(v_index), v_rows, scale, neg_slope,
                                                      _ptr(lse), _ptr(dout), _ptr(dQ),
                                                      _ptr(g_edge), _ptr(alpha_edge),
                                                      _stream(stream)))


def fast_index_add_scaled_rows_workspace(n: int, num_rows: int, H: int, dh: int) -> int:
    return lib().fast_index_add_scaled_rows_workspace(n, num_rows, H, dh)


def fast_index_add_scaled_rows(occ_off, occ, n, num_rows, dst_offsets, num_dst, H, dh, src_dtype,
                               scal, src, dst, ws, ws_bytes, stream=None):
    _check(lib().fast_index_add_scaled_rows(_ptr(occ_off), _ptr(occ), n, num_rows,
                                            _ptr(dst_offsets), num_dst, H, dh, src_dtype,
                                            _ptr(scal), _ptr(src), _ptr(dst), _ptr(ws), ws_bytes,
                                            _stream(stream)))


def fast_layer_norm_fwd(n, D, dtype, x, res, gamma, beta, eps, y, sum=None, mean=None, rstd=None,
                        stream=None):
    _resident((x, res, gamma, beta, y, sum, mean, rstd))
    _check(lib().fast_layer_norm_fwd(n, D, dtype, _ptr(x), _ptr(res), _ptr(gamma), _ptr(beta), eps,
                                     _ptr(y), _ptr(sum), _ptr(mean), _ptr(rstd), _stream(stream)))


def fast_layer_norm_bwd_workspace(n: int, D: int) -> int:
    return lib().fast_layer_norm_bwd_workspace(n, D)


def fast_layer_norm_bwd(n, D, dtype, h, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, ws,
                        ws_bytes, stream=None):
    _resident((h, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, ws))
    _check(lib().fast_layer_norm_bwd(n, D, dtype, _ptr(h), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                     _ptr(dy), _ptr(dsum), _ptr(dx), _ptr(dgamma), _ptr(dbeta),
                                     _ptr(ws), ws_bytes, _stream(stream)))


def fast_rotary_fwd(n, H, dh, dtype, x, ldx, pos, axes, axis, omega, pairs, interleaved, y, ldy,
                    stream=None):
    """x and y may be views whose rows are ldx and ldy elements apart."""
    _resident((pos, axis, omega), ((x, ldx, H * dh), (y, ldy, H * dh)))
    _check(lib().fast_rotary_fwd(n, H, dh, dtype, _ptr(x), ldx, _ptr(pos), axes, _ptr(axis),
                                 _ptr(omega), pairs, int(interleaved), _ptr(y), ldy,
                                 _stream(stream)))


def fast_rotary_bwd(n, H, dh, dtype, dy, lddy, pos, axes, axis, omega, pairs, interleaved, dx, lddx,
                    stream=None):
    _resident((pos, axis, omega), ((dy, lddy, H * dh), (dx, lddx, H * dh)))
    _check(lib().fast_rotary_bwd(n, H, dh, dtype, _ptr(dy), lddy, _ptr(pos), axes, _ptr(axis),
                                 _ptr(omega), pairs, int(interleaved), _ptr(dx), lddx,
                                 _stream(stream)))


def fast_cache_row_bytes(parts: int, width: int, format: int) -> int:
    return lib().fast_cache_row_bytes(parts, width, format)


def fast_cache_write_workspace(n: int, cache_rows: int) -> int:
    return lib().fast_cache_write_workspace(n, cache_rows)


def fast_cache_write(ids, n, id_bound, slot_map, parts, width, dtype, src, format, cache, cache_rows,
                     distinct, ws=None, ws_bytes=0, stream=None):
    _resident((ids, slot_map, src, cache, ws))
    _check(lib().fast_cache_write(_ptr(ids), n, id_bound, _ptr(slot_map), parts, width, dtype,
                                  _ptr(src), format, _ptr(cache), cache_rows, int(distinct),
                                  _ptr(ws), ws_bytes, _stream(stream)))


def fast_cache_gather(ids, n, id_bound, slot_map, parts, width, format, cache, cache_rows, dtype,
                      rows, stream=None):
    _resident((ids, slot_map, cache, rows))
    _check(lib().fast_cache_gather(_ptr(ids), n, id_bound, _ptr(slot_map), parts, width, format,
                                   _ptr(cache), cache_rows, dtype, _ptr(rows), _stream(stream)))


def fast_edge_attention_cached_workspace(num_dst: int, num_edges: int, H: int, dh: int) -> int:
    return lib().fast_edge_attention_cached_workspace(num_dst, num_edges, H, dh)


def fast_edge_attention_fwd_cached(g: TCSR, H, dh, dtype, Q, ids, id_bound, slot_map, format, cache,
                                   cache_rows, scale, neg_slope, out, lse, ws, ws_bytes,
                                   stream=None):
    _resident((*getattr(g, "_keep", ())[:1], Q, ids, slot_map, cache, out, lse, ws))   # its offsets first
    _check(lib().fast_edge_attention_fwd_cached(C.byref(g), H, dh, dtype, _ptr(Q), _ptr(ids),
                                                id_bound, _ptr(slot_map), format, _ptr(cache),
                                                cache_rows, scale, neg_slope, _ptr(out),
                                                _ptr(lse), _ptr(ws), ws_bytes, _stream(stream)))


def fast_linear_fwd(n, in_, out, dtype, x, ldx, w, bias, act, res, ldres, y, ldy, pre=None, stream=None):
    """x, res and y may be views whose rows are ldx, ldres and ldy elements apart."""
    _resident((w, bias, pre), ((x, ldx, in_), (res, ldres, out), (y, ldy, out)))
    _check(lib().fast_linear_fwd(n, in_, out, dtype, _ptr(x), ldx, _ptr(w), _ptr(bias), act, _ptr(res),
                                 ldres, _ptr(y), ldy, _ptr(pre), _stream(stream)))


def fast_linear_bwd_workspace(n: int, in_: int, out: int, dtype: int, act: int) -> int:
    return lib().fast_linear_bwd_workspace(n, in_, out, dtype, act)


def fast_linear_bwd(n, in_, out, dtype, x, ldx, w, act, pre, dy, lddy, dx, lddx, dw, dbias, ws,
                    ws_bytes, stream=None):
    _resident((w, pre, dw, dbias, ws), ((x, ldx, in_), (dx, lddx, in_), (dy, lddy, out)))
    _check(lib().fast_linear_bwd(n, in_, out, dtype, _ptr(x), ldx, _ptr(w), act, _ptr(pre), _ptr(dy),
                                 lddy, _ptr(dx), lddx, _ptr(dw), _ptr(dbias), _ptr(ws), ws_bytes,
                                 _stream(stream)))


def fast_gated_scan_state_rows(num_edges: int) -> int:
    return lib().fast_gated_scan_state_rows(num_edges)


def fast_gated_scan_workspace(num_dst: int, num_edges: int, D: int) -> int:
    return lib().fast_gated_scan_workspace(num_dst, num_edges, D)


def fast_gated_scan_fwd(g: TCSR, D, dtype, x, gate, ldx, dt, h0, longest, h, h_last, states, ws,
                        ws_bytes, stream=None):
    """x and gate may be views whose rows are ldx elements apart."""
    _resident((*getattr(g, "_keep", ())[:1], dt, h0, h, h_last, states, ws), ((x, ldx, D), (gate, ldx, D)))
    _check(lib().fast_gated_scan_fwd(C.byref(g), D, dtype, _ptr(x), _ptr(gate), ldx, _ptr(dt),
                                     _ptr(h0), longest, _ptr(h), _ptr(h_last), _ptr(states), _ptr(ws),
                                     ws_bytes, _stream(stream)))


def fast_gated_scan_bwd(g: TCSR, D, dtype, x, gate, ldx, dt, h0, longest, states, dh, dh_last, dx,
                        dgate, lddx, dh0, ws, ws_bytes, stream=None):
    _resident((*getattr(g, "_keep", ())[:1], dt, h0, states, dh, dh_last, dh0, ws),
              ((x, ldx, D), (gate, ldx, D), (dx, lddx, D), (dgate, lddx, D)))
    _check(lib().fast_gated_scan_bwd(C.byref(g), D, dtype, _ptr(x), _ptr(gate), ldx, _ptr(dt),
                                     _ptr(h0), longest, _ptr(states), _ptr(dh), _ptr(dh_last),
                                     _ptr(dx), _ptr(dgate), lddx, _ptr(dh0), _ptr(ws), ws_bytes,
                                     _stream(stream)))


def adamw_tensors(w, grad, m, v, m_scale=None, v_scale=None, copy=None, decay=None):
    """Builds the host array of fast_adamw_tensor_t over lists of device tensors, one entry per
    tensor (m_scale, v_scale, copy: None, or lists; decay: a number, a list, or None for 0).  Built once
    and passed to every step; it holds addresses and keeps a reference to each tensor, so a program whose
    gradients move builds it anew.  w fp32; all grads fp32 or all bf16; m and v fp32, or all of them codes
    of a byte (uint8, float8_e4m3fn) with scales of a byte (uint8, float8_e8m0fnu); copy bf16."""
    import torch
    n = len(w)
    lists = [w, grad, m, v, m_scale, v_scale, copy]
    for k, x in enumerate(lists):
        if x is None and k >= 4:
            lists[k] = [None] * n
        elif x is None or len(x) != n:
            raise ValueError("one entry per tensor")
    if decay is None or isinstance(decay, (int, float)):
        decay = [float(decay or 0)] * n
    elif len(decay) != n:
        raise ValueError("one decay per tensor")
    a = (AdamWTensor * max(n, 1))()
    f32, bf16 = torch.float32, torch.bfloat16
    code, power = (torch.uint8, torch.float8_e4m3fn), (torch.uint8, torch.float8_e8m0fnu)
    half = any(t is not None and t.dtype == bf16 for t in lists[1])
    low = any(t is not None and t.dtype in code for t in lists[2])
    types = ((f32,), (bf16,) if half else (f32,), *2 * [code if low else (f32,)], power, power, (bf16,))
    for j, ts in enumerate(zip(*lists)):
        size = ts[0].numel()
        for t, want in zip(ts, (size, size, size, size, (size + 31) // 32, (size + 31) // 32, size)):
            if t is not None and t.numel() != want:
                raise FastError(1, f"tensor {j}: an array of {t.numel()} elements, {want} wanted")
        for t, want, name in zip(ts, types, ("w", "grad", "m", "v", "m_scale", "v_scale", "copy")):
            if t is not None and t.dtype not in want:
                raise FastError(1, f"tensor {j}: {name} of {t.dtype}, {' or '.join(map(str, want))} wanted")
        a[j] = AdamWTensor(*[_ptr(t) for t in ts], size, decay[j])
    a._count, a._grad, a._format = n, BF16 if half else F32, STATE_MXFP8 if low else STATE_F32
    a._keep = tuple(t for x in lists for t in x if t is not None)
    _resident(a._keep)
    return a


def _listed(tensors, grad_dtype, format):
    """A list's types are those that a call names; raises otherwise."""
    if tensors._count and (tensors._grad != grad_dtype or tensors._format != format):
        raise FastError(1, f"grad_dtype {grad_dtype}, format {format}: the list holds grads of dtype "
                           f"{tensors._grad}, states of format {tensors._format}")


def fast_adamw(tensors, grad_dtype, format, lr, beta1, beta2, eps, step, seed=0, lr_dev=None,
               step_dev=None, scale=None, stream=None):
    """tensors: from adamw_tensors."""
    _listed(tensors, grad_dtype, format)
    _resident((*tensors._keep[:1], lr_dev, step_dev, scale))
    _check(lib().fast_adamw(tensors, tensors._count, grad_dtype, format, lr, beta1, beta2, eps, step,
                            seed, _ptr(lr_dev), _ptr(step_dev), _ptr(scale), _stream(stream)))


def fast_grad_norm_workspace(total: int, count: int) -> int:
    return lib().fast_grad_norm_workspace(total, count)


def fast_grad_norm(tensors, grad_dtype, max_norm, norm, scale, ws, ws_bytes, stream=None):
    """tensors: from adamw_tensors."""
    _listed(tensors, grad_dtype, tensors._format)
    _resident((*tensors._keep[:1], norm, scale, ws))
    _check(lib().fast_grad_norm(tensors, tensors._count, grad_dtype, max_norm, _ptr(norm), _ptr(scale),
                                _ptr(ws), ws_bytes, _stream(stream)))
