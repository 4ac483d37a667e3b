"""GPU parity of the AdamW step and the gradients' norm against the plain 64-bit definition, through
the C ABI.  States in 8 bits are compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests import plain64_train as p64
from tests.parity import tdtype
from tests.plain64 import HALF, U
from tests.test_gpu_layer import DT, host, within

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-3, 0.9, 0.999, 1e-8
SIZES = [1, 3, 31, 32, 33, 100, 1000, 1023, 1024, 1025, 4096, 5001, 0, 37]


def views(n, dtype, shift):
    """a tensor of n elements, `shift` elements off its allocation's start, guards around it"""
    t = torch.full((n + 2 * shift + 2,), 7, dtype=dtype, device="cuda")
    return t, t[shift:shift + n]


def model(sizes, grad, low, copy, shift, seed):
    r = np.random.default_rng(seed)
    d = dict(all=[], w=[], g=[], m=[], v=[], ms=[], vs=[], copy=[], host=[])
    for j, n in enumerate(sizes):
        w = r.normal(size=n).astype(np.float32)
        g = torch.from_numpy((0.01 * r.normal(size=n)).astype(np.float32)).to(tdtype(grad))
        m = (0.003 * r.normal(size=n)).astype(np.float32)
        v = ((0.01 * r.normal(size=n)) ** 2 + 1e-9).astype(np.float32)
        h = dict(w=w.astype(np.float64), g=g.double().numpy(), m=m.astype(np.float64), v=v.astype(np.float64))

        def put(name, values, dtype):
            base, t = views(len(values), dtype, shift)
            t.copy_(values if isinstance(values, torch.Tensor) else torch.from_numpy(values))
            d[name].append(t)
            d["all"].append((base, shift, len(values)))
        put("w", w, torch.float32)
        put("g", g, tdtype(grad))
        if low:
            half = np.full(n, 0x8000)
            for name, val, root in (("m", m, False), ("v", np.sqrt(v), True)):
                c, s = p64.to_codes(val.astype(np.float64), half, root)
                put(name, c, torch.uint8)
                put(name + "s", s, torch.uint8)
                h[name] = p64.from_codes(c, s) ** (2 if root else 1)
        else:
            put("m", m, torch.float32)
            put("v", v, torch.float32)
        if copy:
            put("copy", np.zeros(n, np.float32), torch.bfloat16)
        d["host"].append(h)
    d["decay"] = [0.01 if j % 2 else 0.0 for j in range(len(sizes))]
    d["list"] = fast.adamw_tensors(d["w"], d["g"], d["m"], d["v"], d["ms"] or None, d["vs"] or None, d["copy"] or None,
                                   d["decay"])
    return d


def compare(d, sizes, t, seed, low, scale=1.0, lr=LR):
    for j, n in enumerate(sizes):
        h = d["host"][j]
        g = h["g"] * scale
        w, m, v = p64.adamw(h["w"], g, h["m"], h["v"], t, lr, B1, B2, EPS, d["decay"][j])
        if low:
            m32, root = m.astype(np.float32).astype(np.float64), np.sqrt(v).astype(np.float32).astype(np.float64)
            bits = p64.rounding_bits(seed, t, j, n).astype(np.int64)
            for name, val, r, up in (("m", m32, bits & 0xFFFF, False), ("v", root, bits >> 16, True)):
                c, s = p64.to_codes(val, r, up)
                np.testing.assert_array_equal(d[name][j].cpu().numpy(), c)
                np.testing.assert_array_equal(d[name + "s"][j].cpu().numpy(), s)
                h[name] = p64.from_codes(c, s) ** (2 if up else 1)
        else:
            # a product's and a sum's rounding each, and that of 1 - beta
            within(d["m"][j], m, 4 * U * (np.abs(B1 * h["m"]) + np.abs((1 - B1) * g)), "m")
            within(d["v"][j], v, 5 * U * (B2 * h["v"] + (1 - B2) * g * g), "v")
            h["m"], h["v"] = host(d["m"][j]), host(d["v"][j])
        tm = 4 * U * (np.abs(B1 * h["m"]) + np.abs((1 - B1) * g)) if not low else 2 * U * np.abs(m)
        den = np.sqrt(v / (1 - B2 ** t)) + EPS
        tol = lr * ((tm / (1 - B1 ** t) + 12 * U * np.abs(m) / (1 - B1 ** t)) / den + 3 * U * np.abs(h["w"]) * 0.01)
        # m after the step stands for m above: what the step's own rounding moved is in tm
        within(d["w"][j], w, 2 * tol + 2 * U * np.abs(w), "w")
        h["w"] = host(d["w"][j])
        if d["copy"]:
            assert torch.equal(d["copy"][j], d["w"][j].bfloat16())
    for base, shift, n in d["all"]:
        assert (base[:shift] == 7).all() and (base[shift + n:] == 7).all()


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("low", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_adamw_steps(grad, low, shift):
    print(f"[adamw] {grad} low={low} shift={shift}", flush=True)
    d = model(SIZES, grad, low, shift != 3, shift, 1)
    form = fast.STATE_MXFP8 if low else fast.STATE_F32
    for t in (1, 2, 3):
        fast.fast_adamw(d["list"], DT[grad], form, LR, B1, B2, EPS, t, 12345)
        compare(d, SIZES, t, 12345, low)


@pytest.mark.parametrize("low", [False, True], ids=["32", "8"])
def test_adamw_many_tensors_and_large_ones(low):
    """More tensors than a launch takes; more elements than a workgroup's single round."""
    sizes = [5 + 7 * k for k in range(130)]
    d = model(sizes, "f32", low, True, 0, 2)
    form = fast.STATE_MXFP8 if low else fast.STATE_F32
    fast.fast_adamw(d["list"], 0, form, LR, B1, B2, EPS, 7, 99)
    compare(d, sizes, 7, 99, low)
    sizes = [100, 4200001 if not low else 4200001, 77]
    print("[adamw] large", flush=True)
    n = sizes[1]
    w, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda") * 0.01
    if not low:
        m, v = torch.randn(n, device="cuda") * 0.003, torch.rand(n, device="cuda") * 1e-4
        w0, m0, v0 = w.double(), m.double(), v.double()
        fast.fast_adamw(fast.adamw_tensors([w], [g], [m], [v], decay=0.01), 0, form, LR, B1, B2, EPS, 1000)
        m1 = B1 * m0 + (1 - B1) * g.double()
        v1 = B2 * v0 + (1 - B2) * g.double() ** 2
        w1 = w0 - LR * (0.01 * w0 + m1 / (1 - B1 ** 1000) / ((v1 / (1 - B2 ** 1000)).sqrt() + EPS))
        assert ((m - m1).abs() <= 4 * U * (m0.abs() + g.abs())).all()
        assert ((v - v1).abs() <= 6 * U * v1).all()
        assert ((w - w1).abs() <= 2 * U * w1.abs() + LR * 40 * U * (w0.abs() + (m0.abs() + g.abs()) / v1.sqrt())).all()
    else:
        z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")
        m, v, ms, vs = z(n), z(n), z((n + 31) // 32), z((n + 31) // 32)
        fast.fast_adamw(fast.adamw_tensors([w], [g], [m], [v], [ms], [vs]), 0, form, LR, B1, B2, EPS, 1, 5)
        for at in (0, 32 * 40000, n - 65):                 # pieces of it, with their own places
            at -= at % 32
            k = min(64, n - at)
            bits = p64.rounding_bits(5, 1, 0, n)[at:at + k].astype(np.int64)
            gd = host(g)[at:at + k]
            for c, s, val, r, up in ((m, ms, (1 - B1) * gd, bits & 0xFFFF, False),
                                     (v, vs, np.sqrt((1 - B2) * gd * gd), bits >> 16, True)):
                rc, rs = p64.to_codes(val.astype(np.float32).astype(np.float64), r, up)
                np.testing.assert_array_equal(c[at:at + k].cpu().numpy(), rc)
                np.testing.assert_array_equal(s[at // 32:at // 32 + len(rs)].cpu().numpy(), rs)


def test_adamw_random_rounding_keeps_the_mean():
    """A thousand steps without gradients: every root falls by sqrt(beta2) a step in the mean, though no single
    step reaches the next code.  The mean of 10^5 roots, each of a spread below 0.3, is within 0.005 of its
    own mean but in one of 10^6 runs; the rule's bias (2^-16 of an eighth at most a step) adds 0.002."""
    n = 100000
    z = lambda k, x=0: torch.full((k,), x, dtype=torch.uint8, device="cuda")
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v, ms, vs = z(n), z(n, 0x38), z(n // 32), z(n // 32, 127)         # roots of 1
    ts = fast.adamw_tensors([w], [g], [m], [v], [ms], [vs])
    for t in range(1, 1001):
        fast.fast_adamw(ts, 0, fast.STATE_MXFP8, LR, B1, B2, EPS, t, 3)
    root = p64.from_codes(v.cpu().numpy(), vs.cpu().numpy())
    assert abs(root.mean() - B2 ** 500) <= 0.007
    assert (w == 0).all() and (p64.from_codes(m.cpu().numpy(), ms.cpu().numpy()) == 0).all()


def test_adamw_nonfinite_groups_and_extremes_in_8_bits():
    n = 160
    g = torch.zeros(n, device="cuda")
    g[5], g[40] = float("nan"), float("inf")
    g[64:96] = torch.logspace(-44, -30, 32)
    g[96:128] = torch.logspace(-40, 38, 32, dtype=torch.float64).float()
    g[128:160] = 3e38 * torch.linspace(-1, 1, 32)
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")
    w, m, v, ms, vs = torch.ones(n, device="cuda"), z(n), z(n), z(5), z(5)
    fast.fast_adamw(fast.adamw_tensors([w], [g], [m], [v], [ms], [vs]), 0, fast.STATE_MXFP8, LR, 0.0, 0.0, EPS, 1, 8)
    assert ms[:2].tolist() == [255, 255] and vs[:2].tolist() == [255, 255]
    assert (m[:64] == 0).all() and (v[:64] == 0).all()
    bits = p64.rounding_bits(8, 1, 0, n).astype(np.int64)[64:]
    val = host(g)[64:]
    for c, s, x, r, up in ((m, ms, val, bits & 0xFFFF, False), (v, vs, np.abs(val), bits >> 16, True)):
        rc, rs = p64.to_codes(x, r, up)
        np.testing.assert_array_equal(c[64:].cpu().numpy(), rc)
        np.testing.assert_array_equal(s[2:].cpu().numpy(), rs)
        assert np.isfinite(p64.from_codes(rc, rs).astype(np.float32)).all()
    assert (v[64:160].cpu().numpy()[np.abs(val) > 0] > 0).all()
    # the next step reads the marked groups back as not a number, and only those
    g.zero_()
    fast.fast_adamw(fast.adamw_tensors([w], [g], [m], [v], [ms], [vs]), 0, fast.STATE_MXFP8, LR, 0.5, 0.5, EPS, 2, 8)
    assert torch.isnan(w[:64]).all() and torch.isfinite(w[64:]).all()


def test_adamw_scale_skips_a_step():
    for low in (False, True):
        d = model([100, 33], "bf16", low, True, 0, 4)
        form = fast.STATE_MXFP8 if low else fast.STATE_F32
        before = [t.clone() for k in ("w", "m", "v", "ms", "vs", "copy") for t in d[k]]
        for bad in (float("nan"), float("inf"), float("-inf")):
            fast.fast_adamw(d["list"], 1, form, LR, B1, B2, EPS, 5, 1, scale=torch.full((1,), bad, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(before, [t for k in ("w", "m", "v", "ms", "vs", "copy") for t in d[k]]))
        sc = torch.full((1,), 0.25, device="cuda")
        fast.fast_adamw(d["list"], 1, form, LR, B1, B2, EPS, 5, 1, scale=sc)
        compare(d, [100, 33], 5, 1, low, scale=0.25)


def test_adamw_captured_reads_step_and_rate_from_the_device():
    for low in (False, True):
        d = model([1000, 77], "f32", low, False, 0, 6)
        form = fast.STATE_MXFP8 if low else fast.STATE_F32
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")

        def one():
            step.add_(1)
            fast.fast_adamw(d["list"], 0, form, 123.0, B1, B2, EPS, 0, 17, lr, step)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one()
        for t in range(1, 5):
            lr.fill_(LR * t)
            graph.replay() if t != 3 else one()
            torch.cuda.synchronize()
            compare(d, [1000, 77], t, 17, low, lr=float(lr))


@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_grad_norm(grad):
    for sizes in (SIZES, [5 + k for k in range(300)], [300001], []):
        print(f"[norm] {len(sizes)} tensors {grad}", flush=True)
        r = np.random.default_rng(len(sizes))
        g = [torch.from_numpy(r.normal(size=n).astype(np.float32)).to(tdtype(grad)) for n in sizes]
        want = float(np.sqrt(sum(float((x.double() ** 2).sum()) for x in g)))
        dev = [x.cuda() for x in g]
        z = [torch.zeros(n, device="cuda") for n in sizes]
        ts = fast.adamw_tensors(z, dev, z, z)
        wsb = fast.fast_grad_norm_workspace(sum(sizes), len(sizes))
        ws = torch.full((wsb + 64,), 0xAB, dtype=torch.uint8, device="cuda")
        norm, scale = torch.zeros(2, 1, device="cuda").unbind(0)
        for most in (want / 3 if want else 1.0, want * 3 + 1, float("inf")):
            fast.fast_grad_norm(ts, DT[grad], most, norm, scale, ws, wsb)
            assert abs(float(norm) - want) <= U * want * 1.01
            f = np.float32(most) / np.float32(float(norm)) if want > most else 1.0
            assert abs(float(scale) - f) <= 2 * U * abs(f)
        assert (ws[wsb:] == 0xAB).all()
        if sizes and sizes[0] > 0:
            dev[0][0] = float("inf")
            fast.fast_grad_norm(ts, DT[grad], 1.0, norm, scale, ws, wsb)
            assert torch.isinf(norm) and torch.isnan(scale)


def test_clipped_step():
    d = model([1000, 5], "f32", False, False, 0, 11)
    norm, scale = torch.zeros(2, 1, device="cuda").unbind(0)
    wsb = fast.fast_grad_norm_workspace(1005, 2)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_grad_norm(d["list"], 0, 0.1, norm, scale, ws, wsb)
    assert float(norm) > 0.1
    fast.fast_adamw(d["list"], 0, fast.STATE_F32, LR, B1, B2, EPS, 1, 0, scale=scale)
    compare(d, [1000, 5], 1, 0, False, scale=float(scale))
