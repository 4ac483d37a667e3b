"""Layer operators without a GPU: refusals before any launch, workspace and record
sizes, and the plain 64-bit definitions that the GPU tests compare with (gradients
against differences, formats against their definition)."""
import ctypes

import numpy as np
import pytest

import paper_2607_05095_amd as fast
from tests import plain64 as p64

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x10000  # an aligned stand-in address, never dereferenced on these paths
BIG = 1 << 31


def call(name, defaults, kw):
    L = fast.lib()
    a = dict(defaults)
    a.update(kw)
    return getattr(L, name)(*a.values())


NORM = dict(n=5, D=10, dt=0, x=FAKE, res=None, gamma=FAKE, beta=FAKE, eps=1e-5, y=FAKE, sum=None,
            mean=FAKE, rstd=FAKE, st=None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(D=0), INVALID), (dict(dt=2), INVALID), (dict(x=None), INVALID),
    (dict(y=None), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(sum=FAKE), INVALID), (dict(D=8193), UNSUPPORTED), (dict(n=BIG), UNSUPPORTED),
    (dict(x=FAKE + 2), UNSUPPORTED), (dict(dt=1, y=FAKE + 1), UNSUPPORTED),
    (dict(gamma=FAKE + 2), UNSUPPORTED), (dict(n=0, x=None, y=None), OK)])
def test_layer_norm_fwd_refusals(kw, status):
    assert call("fast_layer_norm_fwd", NORM, kw) == status
    assert (fast.fast_last_error() == "") == (status == OK)


def test_layer_norm_sum_and_y_in_one_array_refused():
    assert call("fast_layer_norm_fwd", NORM, dict(res=FAKE + 4096, sum=FAKE, y=FAKE)) == INVALID


NORM_B = dict(n=5, D=10, dt=0, h=FAKE, gamma=FAKE, mean=FAKE, rstd=FAKE, dy=FAKE, dsum=None, dx=FAKE,
              dgamma=FAKE, dbeta=FAKE, ws=FAKE, wsb=1 << 20, st=None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(D=-3), INVALID), (dict(dt=9), INVALID), (dict(h=None), INVALID),
    (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(dy=None), INVALID),
    (dict(dx=None), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=1), WORKSPACE),
    (dict(ws=FAKE + 4), UNSUPPORTED), (dict(dsum=FAKE + 1), UNSUPPORTED), (dict(D=8193), UNSUPPORTED),
    (dict(n=0, dgamma=None, dbeta=None, ws=None), OK)])
def test_layer_norm_bwd_refusals(kw, status):
    assert call("fast_layer_norm_bwd", NORM_B, kw) == status


def test_launches_past_the_thread_limit_are_refused():
    """Sizes whose launch would need 2^32 threads: refused before anything is enqueued."""
    assert call("fast_layer_norm_fwd", NORM, dict(n=BIG - 1, D=500)) == UNSUPPORTED
    assert call("fast_rotary_fwd", ROT, dict(n=BIG - 1, H=8, dh=16, ldx=256, ldy=256, pairs=8, x=FAKE,
                                             y=FAKE + 4 * 128)) == UNSUPPORTED
    assert call("fast_cache_write", CW, dict(n=BIG - 1, parts=8, width=32, distinct=1)) == UNSUPPORTED
    assert call("fast_cache_gather", CG, dict(n=BIG - 1, parts=8, width=32)) == UNSUPPORTED
    a = dict(ATT, dh=256, Q=FAKE, ws=FAKE, wsb=1 << 40)
    a["g"] = ctypes.byref(fast.TCSR(BIG - 1, 10, FAKE, None, None, None, None))
    assert fast.lib().fast_edge_attention_fwd_cached(*a.values()) == UNSUPPORTED


def test_layer_norm_workspace():
    assert fast.fast_layer_norm_bwd_workspace(0, 8) > 0
    assert fast.fast_layer_norm_bwd_workspace(-1, 8) == 0
    assert fast.fast_layer_norm_bwd_workspace(4, 0) == 0
    assert fast.fast_layer_norm_bwd_workspace(4, 8193) == 0
    # a partial row of two fp64 sums per column and workgroup, a small share of the rows
    assert fast.fast_layer_norm_bwd_workspace(10 ** 7, 100) < 10 ** 7 * 100 * 4 // 10


ROT = dict(n=5, H=2, dh=8, dt=0, x=FAKE, ldx=16, pos=FAKE, axes=2, axis=FAKE, omega=FAKE, pairs=4,
           inter=0, y=FAKE + 4096, ldy=16, st=None)


@pytest.mark.parametrize("name", ["fast_rotary_fwd", "fast_rotary_bwd"])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(H=0), INVALID), (dict(dh=0), INVALID), (dict(dt=4), INVALID),
    (dict(pairs=5), INVALID), (dict(pairs=-1), INVALID), (dict(axes=0), INVALID),
    (dict(ldx=15), INVALID), (dict(ldy=15), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(pos=None), INVALID), (dict(omega=None), INVALID),
    (dict(y=FAKE + 4), INVALID),                       # shifted by one element
    (dict(y=FAKE, ldy=32), INVALID),                   # in place with another stride
    (dict(ldx=32, ldy=32, y=FAKE + 60), INVALID),      # one element into the gap
    (dict(H=65), UNSUPPORTED), (dict(dh=257, ldx=600, ldy=600), UNSUPPORTED),
    (dict(x=FAKE + 2), UNSUPPORTED), (dict(pos=FAKE + 1), UNSUPPORTED), (dict(n=BIG), UNSUPPORTED),
    (dict(n=0, x=None, y=None, pos=None, omega=None), OK)])
def test_rotary_refusals(name, kw, status):
    assert call(name, ROT, kw) == status


CW = dict(ids=FAKE, n=4, bound=100, map=FAKE, parts=2, width=40, dt=0, src=FAKE, fmt=0, cache=FAKE,
          rows=50, distinct=0, ws=FAKE, wsb=1 << 20, st=None)
CG = dict(ids=FAKE, n=4, bound=100, map=FAKE, parts=2, width=40, fmt=0, cache=FAKE, rows=50, dt=0,
          out=FAKE, st=None)
COMMON = [(dict(n=-1), INVALID), (dict(bound=-1), INVALID), (dict(rows=-1), INVALID),
          (dict(dt=2), INVALID), (dict(fmt=2), INVALID), (dict(parts=0), INVALID), (dict(width=0), INVALID),
          (dict(ids=None), INVALID), (dict(cache=None), INVALID), (dict(parts=129), UNSUPPORTED),
          (dict(width=1025), UNSUPPORTED), (dict(parts=128, width=65), UNSUPPORTED),
          (dict(n=BIG), UNSUPPORTED), (dict(rows=BIG), UNSUPPORTED), (dict(cache=FAKE + 8), UNSUPPORTED),
          (dict(ids=FAKE + 4), UNSUPPORTED), (dict(n=0, ids=None, cache=None), OK),
          (dict(rows=0, cache=None), OK)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(src=None), INVALID), (dict(src=FAKE + 2), UNSUPPORTED), (dict(ws=None), WORKSPACE),
    (dict(wsb=199), WORKSPACE), (dict(ws=FAKE + 8), UNSUPPORTED)])
def test_cache_write_refusals(kw, status):
    assert call("fast_cache_write", CW, kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [(dict(out=None), INVALID), (dict(out=FAKE + 2), UNSUPPORTED)])
def test_cache_gather_refusals(kw, status):
    assert call("fast_cache_gather", CG, kw) == status


@pytest.mark.parametrize("fmt", [8, 4])
def test_cache_record_sizes(fmt):
    f = fast.MXFP8 if fmt == 8 else fast.MXFP4
    for parts in (1, 2, 3, 4, 8, 16, 128):
        for width in (1, 7, 8, 31, 32, 33, 50, 64, 100, 128, 172, 200, 256, 1000):
            if parts * width <= 8192:
                assert fast.fast_cache_row_bytes(parts, width, f) == p64.record(parts, width, fmt)[3]
    assert fast.fast_cache_row_bytes(0, 4, f) == 0
    assert fast.fast_cache_row_bytes(4, 1025, f) == 0
    assert fast.fast_cache_row_bytes(128, 65, f) == 0
    assert fast.fast_cache_row_bytes(4, 4, 5) == 0
    assert fast.fast_cache_write_workspace(10, 100) >= 400
    assert fast.fast_cache_write_workspace(-1, 100) == 0


ATT = dict(g="ok", H=2, dh=50, dt=0, Q=FAKE, ids=FAKE, bound=10, map=FAKE, fmt=0, cache=FAKE, rows=10,
           scale=1.0, slope=0.2, out=FAKE, lse=None, ws=FAKE, wsb=1 << 20, st=None)


@pytest.mark.parametrize("kw,status", [
    (dict(g=None), INVALID), (dict(g=(-1, 4)), INVALID), (dict(g=(4, -1)), INVALID),
    (dict(g=(0, 4)), INVALID), (dict(g=(4, 4, None)), INVALID), (dict(H=0), INVALID), (dict(dh=0), INVALID),
    (dict(dt=3), INVALID), (dict(fmt=3), INVALID), (dict(bound=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(Q=None), INVALID), (dict(out=None), INVALID), (dict(ids=None), INVALID),
    (dict(cache=None), INVALID), (dict(H=65, dh=4), UNSUPPORTED), (dict(dh=257), UNSUPPORTED),
    (dict(H=8, dh=129), UNSUPPORTED), (dict(g=(4, BIG)), UNSUPPORTED), (dict(rows=BIG), UNSUPPORTED),
    (dict(Q=FAKE + 2), UNSUPPORTED), (dict(cache=FAKE + 8), UNSUPPORTED), (dict(ids=FAKE + 4), UNSUPPORTED),
    (dict(ws=FAKE + 4), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(wsb=8), WORKSPACE),
    (dict(g=(0, 0), Q=None, out=None, ws=None), OK)])
def test_cached_attention_refusals(kw, status):
    a = dict(ATT)
    a.update(kw)
    g = a["g"]
    if g is not None:
        g = (4, 40, FAKE) if g == "ok" else (tuple(g) + (FAKE,))[:3]
        g = fast.TCSR(g[0], g[1], g[2], None, None, None, None)
        a["g"] = ctypes.byref(g)
    assert fast.lib().fast_edge_attention_fwd_cached(*a.values()) == status


def test_cached_attention_workspace():
    ws = fast.fast_edge_attention_cached_workspace
    assert ws(0, 0, 2, 50) > 0 and ws(1, 10, 2, 50) > 0
    for bad in ((-1, 1, 2, 50), (1, -1, 2, 50), (1, BIG, 2, 50), (1, 1, 0, 50), (1, 1, 2, 257), (1, 1, 64, 17)):
        assert ws(*bad) == 0


def test_binding_refuses_host_and_strided_tensors():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(fast.FastError):
        fast.fast_layer_norm_fwd(4, 8, fast.F32, x, None, None, None, 1e-5, x)
    assert set(n for n in fast.__all__ if "layer_norm" in n) == {
        "fast_layer_norm_fwd", "fast_layer_norm_bwd", "fast_layer_norm_bwd_workspace"}


# ---------------------------------------------------------------- the definitions themselves
def _difference(f, x, d, eps=1e-5):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


def test_plain_norm_gradients_match_differences():
    r = np.random.default_rng(1)
    h, dy, ds = r.normal(size=(3, 5, 9))
    ga, be = r.normal(size=(2, 9))
    _, mu, rs = p64.layer_norm(h, ga, be, 1e-3)
    dx, dg, db = p64.layer_norm_bwd(h, ga, mu, rs, dy, ds)
    for grad, x, f in ((dx, h, lambda v: (dy * p64.layer_norm(v, ga, be, 1e-3)[0]).sum() + (ds * v).sum()),
                       (dg, ga, lambda v: (dy * p64.layer_norm(h, v, be, 1e-3)[0]).sum()),
                       (db, be, lambda v: (dy * p64.layer_norm(h, ga, v, 1e-3)[0]).sum())):
        d = r.normal(size=x.shape)
        assert abs(_difference(f, x, d) - (grad * d).sum()) < 1e-6


@pytest.mark.parametrize("inter", [False, True])
def test_plain_rotary_turns_and_its_gradient(inter):
    r = np.random.default_rng(2)
    x, dy = r.normal(size=(2, 4, 3, 11))
    pos, om = r.uniform(0, 50, (4, 2)), r.uniform(0, 2, 4)
    ax = np.array([0, 1, 1, 0])
    f = lambda v: (dy * p64.rotary(v, pos, ax, om, 4, inter)).sum()
    d = r.normal(size=x.shape)
    assert abs(_difference(f, x, d) - (p64.rotary(dy, pos, ax, om, 4, inter, -1.0) * d).sum()) < 1e-6
    # turned queries and keys meet in the difference of their positions
    q, k = r.normal(size=(2, 4, 3, 11))
    shift = pos + np.array([3.0, -7.0])
    dot = lambda p, s: (p64.rotary(q, p, ax, om, 4, inter) * p64.rotary(k, s, ax, om, 4, inter)).sum()
    np.testing.assert_allclose(dot(pos, pos * 0.5), dot(shift, pos * 0.5 + np.array([3.0, -7.0])), rtol=1e-12)


@pytest.mark.parametrize("fmt", [8, 4])
def test_plain_formats(fmt):
    g = p64.grid(fmt)
    if fmt == 8:
        import torch
        t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
        np.testing.assert_array_equal(np.concatenate([g, -g]), t)
    codes, sc = p64.quantize(np.concatenate([g[~np.isnan(g)], -g[~np.isnan(g)]]).reshape(1, 1, -1)[..., :32]
                             if fmt == 4 else g[~np.isnan(g)].reshape(1, 1, -1)[..., -32:], fmt)
    assert (sc == 127).all()                                  # the format's own values keep scale 1
    r = np.random.default_rng(3)
    x = r.normal(size=(50, 2, 70)) * 2.0 ** r.integers(-30, 30, (50, 2, 1))
    c, s = p64.quantize(x, fmt)
    v = p64.values(c, s, fmt)
    top = np.repeat(np.stack([np.abs(x[..., a:a + 32]).max(-1) for a in (0, 32, 64)], -1), 32, -1)[..., :70]
    # half a step: 2^-4 of a normal value, or half the smallest step of a group of largest value top
    half = np.maximum(np.abs(x) * 2.0 ** -4, top * 2.0 ** -17) if fmt == 8 else np.maximum(
        np.abs(x) * 0.25, top / 3 * 0.25)
    assert (np.abs(v - x) <= half).all()
    np.testing.assert_array_equal(p64.unpack(p64.pack(c, s, fmt), 2, 70, fmt), v)


def test_a_workspace_for_the_largest_sizes_serves_all_smaller_ones():
    r = np.random.default_rng(0)
    size = lambda top: int(10 ** r.uniform(0, np.log10(top)))
    for _ in range(4000):
        D, n = size(8192), size(1e8)
        n2 = min(n, max(0, n - size(n)) if r.random() < 0.5 else size(n))
        assert fast.fast_layer_norm_bwd_workspace(n2, D) <= fast.fast_layer_norm_bwd_workspace(n, D), (n2, n, D)
        H, dh = [(1, 1), (2, 50), (4, 32), (8, 128), (64, 16)][r.integers(5)]
        N, E = size(1e7), size(1e8)
        N2, E2 = (min(k, max(0, k - size(k)) if r.random() < 0.5 else size(k)) for k in (N, E))
        big, small = (fast.fast_edge_attention_cached_workspace(a, b, H, dh) for a, b in ((N, E), (N2, E2)))
        assert small <= big, (N2, E2, N, E, H, dh)
    # and at the borders of the ways a call is carried out
    for H, dh in ((2, 50), (4, 32), (64, 16)):
        for N in (1, 31, 32, 64, 2048, 4096, 4097, 100000):
            E = np.unique([b + d for b in (64, 128, 256, 1024, 4096, 8192, 65536, 131072, 245760, 491520, 983040,
                                           64 * N, 128 * N, 2048 * N) for d in (-1, 0, 1)])
            ws = [fast.fast_edge_attention_cached_workspace(N, int(e), H, dh) for e in E]
            assert ws == sorted(ws), (H, dh, N)
