"""Passes through the trained parts around the temporal operators: products of rows with weights
(bias, activation and residual in the epilogue), the gated recurrence over a segment's events, and
the AdamW step over all weights, with the norm that clips its gradients.

A case is a dict of plain values.  `prepare` makes what a program has in hand before the call,
`run` makes one pass, in the operators' plain form (elementary torch operations) or, where `own`
is set, through the framework's entry points.
"""
import math

import torch

own = False

# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------


def listed():
    return [
        # the update of one query's row
        dict(name="linear_query", op="linear", n=1, K=272, M=100, dtype="f32", act="relu", res=True, train=False),
        # K|V rows of a serving batch: node, edge and time features side by side
        dict(name="linear_serve", op="linear", n=600, K=372, M=200, dtype="bf16", act="none", res=False,
             train=False),
        # K|V rows of a training block, all three gradients
        dict(name="linear_block", op="linear", n=264000, K=272, M=256, dtype="bf16", act="none", res=False,
             train=True),
        # the same in fp32 with an activation
        dict(name="linear_events", op="linear", n=264000, K=372, M=200, dtype="f32", act="gelu", res=False,
             train=True),
        # wide hidden rows with a residual, forward and backward
        dict(name="linear_wide", op="linear", n=40000, K=2048, M=2048, dtype="bf16", act="silu", res=True,
             train=True),
        # one new event for each node of a serving batch: memory rows in and out
        dict(name="scan_step", op="scan", N=600, E=600, D=100, dtype="f32", span=True, h0=True, hub=0.0, most=1,
             train=False),
        # sampled blocks of a training step: up to twenty recent events a root
        dict(name="scan_block", op="scan", N=264000, E=2400000, D=100, dtype="f32", span=True, h0=False, hub=0.0,
             most=20, train=True),
        # four whole histories
        dict(name="scan_hubs", op="scan", N=4, E=100003, D=128, dtype="bf16", span=True, h0=True, hub=0.0, most=0,
             train=True),
        # histories of any length, three of them long, gates without time
        dict(name="scan_ragged", op="scan", N=6000, E=900001, D=256, dtype="bf16", span=False, h0=True, hub=0.1,
             most=0, train=True),
        # the weights of a two-layer model, clipped
        dict(name="adamw_model", op="adamw", count=24, total=400000, grad="f32", fmt=32, copy=True, clip=True),
        # one large table of node rows
        dict(name="adamw_table", op="adamw", count=1, total=100000000, grad="f32", fmt=32, copy=False, clip=False),
        # a larger model with states in 8 bits, clipped
        dict(name="adamw_8bit", op="adamw", count=61, total=60000001, grad="bf16", fmt=8, copy=True, clip=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "scan", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "linear":
        K, M = _logint(rng, 1, 2048), _logint(rng, 1, 2048)
        most = 2.0e10 if dtype == "f32" else 1.6e11
        n = max(1, min(_logint(rng, 1, 300000), int(most / (K * M)), 150000000 // (K + M)))
        return dict(op=op, n=n, K=K, M=M, dtype=dtype, act=rng.choice(["none", "relu", "gelu", "silu"]),
                    res=rng.random() < 0.4, train=rng.random() < 0.6)
    if op == "scan":
        D = _logint(rng, 1, 1024)
        E = max(1, min(_logint(rng, 1, 2400000), 240000000 // D))
        N = max(1, min(_logint(rng, 1, 264000), 2 * E, 60000000 // D))
        return dict(op=op, N=N, E=E, D=D, dtype=dtype, span=rng.random() < 0.6, h0=rng.random() < 0.5,
                    hub=rng.choice([0.0, 0.0, 0.2, 0.7]), most=0, train=rng.random() < 0.6)
    total = _logint(rng, 1, 60000000)
    return dict(op=op, count=min(_logint(rng, 1, 150), total), total=total, grad=dtype, fmt=rng.choice([32, 8]),
                copy=rng.random() < 0.5, clip=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

_T = {"f32": torch.float32, "bf16": torch.bfloat16}
_LR, _B1, _B2, _EPS, _CLIP = 1e-3, 0.9, 0.999, 1e-8, 1.0


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _segments(g, N, E, hub, most):
    """offsets of N ragged segments of E edges, some empty; `hub`: the share of the edges that three
    segments hold; `most`: no segment is longer (0: any length)"""
    if most == 1:
        return torch.arange(N + 1, dtype=torch.int32, device="cuda")
    w = torch.rand(N, generator=g, device="cuda").double()
    w = torch.where(w < 0.05, torch.zeros_like(w), w + 0.3)
    if float(w.sum()) == 0:
        w += 1
    w /= w.sum()
    if hub > 0:
        w *= 1 - hub
        w[torch.randint(N, (3,), generator=g, device="cuda")] += hub / 3
    off = torch.round(torch.cumsum(w / w.sum(), 0) * E).clamp(max=E).to(torch.int32)
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), off]).contiguous()


def _sizes(case):
    """sizes of the tensors: wide matrices among narrow vectors, odd ones among them"""
    n, total = case["count"], case["total"]
    w = [(1, 40, 3, 400)[k % 4] + k % 7 for k in range(n)]
    size = [max(1, (total - n) * x // sum(w)) for x in w]
    size[-1] = max(1, total - sum(size[:-1]))
    return size


def _act_of(fast, kind):
    return {"none": fast.ACT_NONE, "relu": fast.ACT_RELU, "gelu": fast.ACT_GELU, "silu": fast.ACT_SILU}[kind]


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    op = case["op"]
    new = lambda *sh, t=torch.float32: torch.empty(*sh, dtype=t, device="cuda")
    if op == "linear":
        n, K, M, dt = case["n"], case["K"], case["M"], _T[case["dtype"]]
        s["x"] = _randn(g, n, K, dtype=dt)
        s["w"] = (_randn(g, M, K) / math.sqrt(K)).to(dt)
        s["b"] = 0.1 * _randn(g, M)
        s["r"] = _randn(g, n, M, dtype=dt) if case["res"] else None
        s["dy"] = _randn(g, n, M, dtype=dt) if case["train"] else None
        # what a forward left for the backward: not this pass's own, whose values next to a border between
        # two numbers of the type may round to either
        s["z"] = _randn(g, n, M, dtype=dt) if case["train"] and case["act"] != "none" else None
        if own:
            import paper_2607_05095_amd as fast
            s["y"] = new(n, M, t=dt)
            s["pre"] = torch.empty_like(s["z"]) if s["z"] is not None else None
            if case["train"]:
                s["dx"], s["dw"], s["db"] = new(n, K, t=dt), new(M, K), new(M)
                s["wsb"] = fast.fast_linear_bwd_workspace(
                    n, K, M, fast.F32 if case["dtype"] == "f32" else fast.BF16, _act_of(fast, case["act"]))
                s["ws"] = new(max(s["wsb"], 16), t=torch.uint8)
    elif op == "scan":
        N, E, D, dt = case["N"], case["E"], case["D"], _T[case["dtype"]]
        s["off"] = _segments(g, N, E, case["hub"], case["most"])
        E = s["E"] = int(s["off"][-1])
        s["longest"] = int((s["off"][1:] - s["off"][:-1]).max())
        # x and its gate side by side, as one product makes them
        s["xg"] = torch.stack((_randn(g, E, D), _randn(g, E, D) - 1), 1).to(dt)
        s["dt"] = torch.empty(E, device="cuda").exponential_(generator=g) if case["span"] else None
        s["h0"] = _randn(g, N, D) if case["h0"] else None
        if case["train"]:
            s["dh"] = _randn(g, E, D, dtype=dt)
            s["dlast"] = _randn(g, N, D)
        if own:
            import paper_2607_05095_amd as fast
            s["g"] = fast.tcsr(s["off"], E)
            s["h"], s["last"] = new(E, D, t=dt), new(N, D)
            s["keep"] = None
            if case["train"]:
                s["keep"] = new(fast.fast_gated_scan_state_rows(E), D)
                s["dxg"] = new(E, 2, D, t=dt)
                s["dh0"] = new(N, D) if case["h0"] else None
            s["wsb"] = fast.fast_gated_scan_workspace(N, E, D)
            s["ws"] = new(max(s["wsb"], 16), t=torch.uint8)
    else:
        # all tensors of a kind in one buffer, each from a multiple of 32 elements on
        size, gt = _sizes(case), _T[case["grad"]]
        s["step"], s["seed"] = 1000, seed & _M32
        rows = [(n + 31) // 32 for n in size]
        first = [32 * sum(rows[:k]) for k in range(len(rows))]
        of = torch.repeat_interleave(torch.tensor(rows, device="cuda"))            # the tensor of a group of 32
        s["place"] = 32 * torch.arange(len(of), device="cuda") - torch.tensor(first, device="cuda")[of]
        s["of"] = of
        live = (s["place"][:, None] + torch.arange(32, device="cuda") < torch.tensor(size, device="cuda")[of][:, None])
        live = live.view(-1)
        n = live.shape[0]
        s["w"] = _randn(g, n) * live
        s["g"] = (0.01 * _randn(g, n) * live).to(gt)
        s["m"] = 0.003 * _randn(g, n) * live
        s["v"] = ((0.01 * _randn(g, n)) ** 2 + 1e-6) * live
        decay = [0.01 if k % 2 else 0.0 for k in range(len(size))]
        s["decay"] = torch.tensor(decay, device="cuda")[of][:, None]
        s["copy_w"] = s["w"].to(torch.bfloat16) if case["copy"] else None
        s["norm"], s["scale"] = new(1), new(1)
        if case["fmt"] == 8:
            half = torch.full((n // 32, 32), 0x8000, device="cuda")
            s["m"], s["ms"] = _quantize(s["m"].view(-1, 32), half)
            s["v"], s["vs"] = _quantize(s["v"].sqrt().view(-1, 32), half, True)
        if own:
            import paper_2607_05095_amd as fast

            def parts(name, unit=1):
                if s.get(name) is None:
                    return None
                return [s[name][f // unit:f // unit + (m + unit - 1) // unit] for f, m in zip(first, size)]
            s["list"] = fast.adamw_tensors(parts("w"), parts("g"), parts("m"), parts("v"), parts("ms", 32),
                                           parts("vs", 32), parts("copy_w"), decay)
            s["wsb"] = fast.fast_grad_norm_workspace(case["total"], case["count"])
            s["ws"] = new(max(s["wsb"], 16), t=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------
# plain form: products
# ------------------------------------------------------------------------------------------------

_CHUNK = 8192                          # rows whose products are added in 32 bits; 64 beyond


def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    return z / (1 + torch.exp(-z))


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    p = 1 / (1 + torch.exp(-z))
    return p * (1 + z * (1 - p))


def _over_rows(a, b):
    """a^T b over many rows"""
    n = a.shape[0] // _CHUNK * _CHUNK
    t = (a[n:].t() @ b[n:]).double()
    if n:
        at = a[:n].view(-1, _CHUNK, a.shape[1]).transpose(1, 2).contiguous()
        t = t + torch.bmm(at, b[:n].view(-1, _CHUNK, b.shape[1])).sum(0, dtype=torch.float64)
    return t.float()


def _linear_plain(s):
    dt, kind = s["x"].dtype, s["act"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["b"]
    y = z if kind == "none" else _act(z, kind)
    if s["r"] is not None:
        y = y + s["r"].float()
    if not s["train"]:
        return (y.to(dt),)
    dz = s["dy"].float()
    if kind != "none":
        dz = dz * _act_slope(s["z"].float(), kind)
    out = (y.to(dt), (dz @ w).to(dt), _over_rows(dz, x), dz.sum(0, dtype=torch.float64).float())
    return out if kind == "none" else out + (z.to(dt),)


# ------------------------------------------------------------------------------------------------
# plain form: recurrence
# ------------------------------------------------------------------------------------------------


def _runs(a, b, first, longest):
    """t = a t_before + b along rows, from `first` (each row's place in its run) on: pairs combined
    over distances 1, 2, 4, ..."""
    d = 1
    while d < longest:
        ok = (first[d:] >= d)[:, None]
        b = torch.cat((b[:d], torch.where(ok, a[d:] * b[:-d] + b[d:], b[d:])))
        a = torch.cat((a[:d], torch.where(ok, a[d:] * a[:-d], a[d:])))
        d *= 2
    return a, b


def _scan_plain(s):
    N, E, D, dt = s["N"], s["E"], s["D"], s["xg"].dtype
    off = s["off"].long()
    size = off[1:] - off[:-1]
    seg = torch.repeat_interleave(torch.arange(N, device="cuda"), size, output_size=E)
    place = torch.arange(E, device="cuda") - off[seg]
    x, gate = s["xg"][:, 0].float(), s["xg"][:, 1].float()
    rate = gate.clamp(min=0) + torch.log1p(torch.exp(-gate.abs()))
    span = s["dt"][:, None] if s["dt"] is not None else torch.ones((), device="cuda")
    a, u = torch.exp(-rate * span), -torch.expm1(-rate * span)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros(N, D, device="cuda")
    pa, pb = _runs(a, u * x, place, s["longest"])
    h = pa * h0[seg] + pb
    some = (size > 0)[:, None]
    end = (off[1:] - 1).clamp(min=0)
    last = torch.where(some, h[end], h0)
    if not s["train"]:
        return h.to(dt), last
    before = torch.where((place > 0)[:, None], torch.cat((h[:1], h[:-1])), h0[seg])
    # back: what reaches h_t is dh_t plus a of the next event times what reaches that
    left = (size[seg] - 1 - place)
    dh = s["dh"].float() + torch.where((left == 0)[:, None], s["dlast"][seg], torch.zeros((), device="cuda"))
    nxt = torch.cat((a[1:], a[:1]))
    _, back = _runs(nxt.flip(0), dh.flip(0), left.flip(0), s["longest"])
    delta = back.flip(0)
    dx = u * delta
    dgate = delta * (x - before) * a * span * torch.sigmoid(gate)
    out = (h.to(dt), last, torch.stack((dx.to(dt), dgate.to(dt)), 1))
    if s["h0"] is None:
        return out
    start = off[:-1].clamp(max=max(E - 1, 0))
    return out + (torch.where(some, a[start] * delta[start], s["dlast"]),)


# ------------------------------------------------------------------------------------------------
# plain form: AdamW.  States in 8 bits: groups of 32 elements of a tensor, m and the square root of v,
# each a code of e4m3 times the power of two 2^k that is the smallest for which the group's largest is
# at most 448; between two codes the upper is taken where the fraction is above 16 bits of a hash, and
# a root that is not zero never becomes zero
# ------------------------------------------------------------------------------------------------

_M32 = 0xffffffff


def _mix(x):
    """32 bits of a hash, in 64-bit integers"""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & _M32
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & _M32
    return x ^ (x >> 16)


def _pow2(k):
    """2^k in 64 bits, exactly"""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _quantize(x, r16, root=False):
    """x [groups, 32] (fp32) and 16 random bits each -> (codes of float8, k + 127 in a byte)"""
    mant, ex = torch.frexp(x.abs().amax(-1))
    k = torch.where(mant > 0, ex - 9 + (mant * 2 > 1.75).int(), torch.full_like(ex, -127)).clamp(min=-127)
    s = x.double() * _pow2(-k)[:, None]
    e = (torch.frexp(s.abs())[1] - 1).clamp(min=-6)
    step = _pow2(torch.where(s == 0, torch.full_like(e, -6), e) - 3)
    t = s.abs() / step
    low = torch.floor(t)
    c = low + (t - low > r16.double() / 65536)
    if root:
        c = torch.where((t > 0) & (c == 0), torch.ones_like(c), c)
    val = (c * step * torch.where(s < 0, -1.0, 1.0)).float()
    return val.to(torch.float8_e4m3fn).view(-1), (k + 127).to(torch.uint8)


def _values(codes, scale):
    """-> what they stand for, [groups, 32]"""
    return codes.view(-1, 32).double() * _pow2(scale.int() - 127)[:, None]


def _random16(s):
    """two numbers of 16 bits per element, from seed, step, tensor and place"""
    top = _mix(s["seed"] ^ (s["step"] * 0x9E3779B9 & _M32))
    h = _mix(_mix(_mix(top ^ s["of"]))[:, None] ^ (s["place"][:, None] + torch.arange(32, device="cuda")))
    return h & 0xffff, h >> 16


def _adamw_plain(s):
    s["step"] += 1
    t = s["step"]
    low = s["fmt"] == 8
    g = s["g"].view(-1, 32).float()
    w = s["w"].view(-1, 32)
    wide = torch.float64 if low else torch.float32     # 64 bits next to a border between codes
    if s["clip"]:
        norm = (g.double() ** 2).sum().sqrt().float()
        g = g.to(wide) * torch.where(norm > _CLIP, _CLIP / norm, torch.ones((), device="cuda")).to(wide)
        s["norm"].copy_(norm)
    g = g.to(wide)
    old_m = _values(s["m"], s["ms"]) if low else s["m"].view(-1, 32)
    old_v = _values(s["v"], s["vs"]) ** 2 if low else s["v"].view(-1, 32)
    m = (_B1 * old_m + (1 - _B1) * g).float()
    v = _B2 * old_v + (1 - _B2) * g * g
    root = torch.sqrt(v).float()
    step = (m / (1 - _B1 ** t)) / (root / math.sqrt(1 - _B2 ** t) + _EPS)
    w.copy_(w - _LR * (s["decay"] * w + step))
    if s["copy_w"] is not None:
        s["copy_w"].copy_(s["w"])
    if low:
        r1, r2 = _random16(s)
        s["m"], s["ms"] = _quantize(m, r1)
        s["v"], s["vs"] = _quantize(root, r2, True)
    else:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    return _held(s)


def _held(s):
    """weights and states; those of 8 bits as numbers of float8 and their groups' powers of two"""
    out = (s["norm"],) if s["clip"] else ()
    out += (s["w"], s["m"], s["v"])
    if s["copy_w"] is not None:
        out += (s["copy_w"],)
    return out + ((s["ms"], s["vs"]) if s["fmt"] == 8 else ())


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------


def run(s):
    op = s["op"]
    if not own:
        return {"linear": _linear_plain, "scan": _scan_plain, "adamw": _adamw_plain}[op](s)
    import paper_2607_05095_amd as fast
    if op == "linear":
        n, K, M, dt = s["n"], s["K"], s["M"], fast.F32 if s["dtype"] == "f32" else fast.BF16
        act = _act_of(fast, s["act"])
        fast.fast_linear_fwd(n, K, M, dt, s["x"], K, s["w"], s["b"], act, s["r"], M, s["y"], M, s["pre"])
        if not s["train"]:
            return (s["y"],)
        fast.fast_linear_bwd(n, K, M, dt, s["x"], K, s["w"], act, s["z"], s["dy"], M, s["dx"], K, s["dw"], s["db"],
                             s["ws"], s["wsb"])
        out = (s["y"], s["dx"], s["dw"], s["db"])
        return out if s["pre"] is None else out + (s["pre"],)
    if op == "scan":
        D, dt = s["D"], fast.F32 if s["dtype"] == "f32" else fast.BF16
        x, gate = s["xg"][:, 0], s["xg"][:, 1]
        fast.fast_gated_scan_fwd(s["g"], D, dt, x, gate, 2 * D, s["dt"], s["h0"], s["most"], s["h"], s["last"],
                                 s["keep"], s["ws"], s["wsb"])
        if not s["train"]:
            return s["h"], s["last"]
        dx, dgate = s["dxg"][:, 0], s["dxg"][:, 1]
        fast.fast_gated_scan_bwd(s["g"], D, dt, x, gate, 2 * D, s["dt"], s["h0"], s["most"], s["keep"], s["dh"],
                                 s["dlast"], dx, dgate, 2 * D, s["dh0"], s["ws"], s["wsb"])
        out = (s["h"], s["last"], s["dxg"])
        return out if s["h0"] is None else out + (s["dh0"],)
    gt = fast.F32 if s["grad"] == "f32" else fast.BF16
    s["step"] += 1
    if s["clip"]:
        fast.fast_grad_norm(s["list"], gt, _CLIP, s["norm"], s["scale"], s["ws"], s["wsb"])
    fast.fast_adamw(s["list"], gt, fast.STATE_F32 if s["fmt"] == 32 else fast.STATE_MXFP8, _LR, _B1, _B2, _EPS,
                    s["step"], s["seed"], None, None, s["scale"] if s["clip"] else None)
    return _held(s)


def work(case):
    op = case["op"]
    if op == "linear":
        n, K, M, b = case["n"], case["K"], case["M"], 4 if case["dtype"] == "f32" else 2
        keeps = case["act"] != "none"
        by = (n * K + M * K + n * M * (1 + case["res"])) * b + 4 * M
        fl = 2 * n * K * M
        if case["train"]:
            by += n * M * b * keeps                                    # pre out
            by += (2 * n * K + M * K + n * M * (1 + keeps)) * b + 4 * M * K + 4 * M
            fl *= 3
        return {"bytes": by, "flops": fl}
    if op == "scan":
        N, E, D, b = case["N"], case["E"], case["D"], 4 if case["dtype"] == "f32" else 2
        by = 3 * E * D * b + 4 * E * case["span"] + 4 * (N + 1) + 4 * N * D * (1 + case["h0"])
        if case["train"]:
            by += 5 * E * D * b + 4 * E * case["span"] + 4 * (N + 1) + 4 * N * D * (1 + 2 * case["h0"])
        return {"bytes": by, "flops": (60 if case["train"] else 20) * E * D}
    n, g = case["total"], 4 if case["grad"] == "f32" else 2
    state = 16 if case["fmt"] == 32 else 4 + 4 / 32
    return {"bytes": n * (8 + state + g * (1 + case["clip"]) + 2 * case["copy"]), "flops": 20 * n}


# ------------------------------------------------------------------------------------------------
# from the definitions in 64 bits
# ------------------------------------------------------------------------------------------------


def _exact_linear(case, s):
    x, w, kind = s["x"].double(), s["w"].double(), case["act"]
    z = torch.addmm(s["b"].double(), x, w.t())
    y = z
    if kind != "none":
        y = {"relu": z.clamp(min=0), "gelu": z * torch.special.ndtr(z), "silu": z * torch.sigmoid(z)}[kind]
    if s["r"] is not None:
        y = y + s["r"].double()
    if not case["train"]:
        return (y,)
    dz = s["dy"].double()
    if kind != "none":
        p = s["z"].double()
        half, sg = torch.special.ndtr(p), torch.sigmoid(p)
        bell = torch.exp(-p.square() / 2) * 0.3989422804014326779
        slope = {"relu": torch.heaviside(p, torch.zeros_like(p)), "gelu": half + p * bell,
                 "silu": sg + p * sg * torch.sigmoid(-p)}[kind]
        dz = dz * slope
    out = (y, dz.mm(w), dz.t().mm(x), dz.sum(0))
    return out if kind == "none" else out + (z,)


def _exact_scan(case, s):
    if s["longest"] > 50000:
        return None
    N, E, D = case["N"], s["E"], case["D"]
    off = s["off"].long()
    size = off[1:] - off[:-1]
    order = torch.argsort(size, descending=True)
    start = off[order]
    times = torch.arange(s["longest"], device="cuda")
    longer = (N - torch.searchsorted(size.sort().values, times, right=True)).tolist()      # segments of over t events
    x, gate = s["xg"][:, 0], s["xg"][:, 1]
    h0 = s["h0"].double() if s["h0"] is not None else torch.zeros(N, D, dtype=torch.float64, device="cuda")

    def event(rows):
        gt = gate[rows].double()
        lam = torch.nn.functional.softplus(gt, threshold=700)
        if s["dt"] is not None:
            span = s["dt"][rows].double()[:, None]
        else:
            span = torch.ones((), dtype=torch.float64, device="cuda")
        keep = torch.exp(-lam * span)
        return gt, span, keep

    h = torch.empty(E, D, dtype=torch.float64, device="cuda")
    state = h0[order].clone()
    for t, n in enumerate(longer):
        rows = start[:n] + t
        _, _, keep = event(rows)
        state[:n] = keep * state[:n] + (1 - keep) * x[rows].double()
        h[rows] = state[:n]
    last = torch.empty_like(state)
    last[order] = state
    if not case["train"]:
        return h, last
    d = s["dlast"].double()[order].clone()
    dxg = torch.empty(E, 2, D, dtype=torch.float64, device="cuda")
    for t in range(len(longer) - 1, -1, -1):
        n = longer[t]
        rows = start[:n] + t
        gt, span, keep = event(rows)
        d[:n] += s["dh"][rows].double()
        prev = h[rows - 1] if t else h0[order[:n]]
        dxg[rows, 0] = (1 - keep) * d[:n]
        dxg[rows, 1] = d[:n] * (x[rows].double() - prev) * keep * span * torch.sigmoid(gt)
        d[:n] *= keep
    dh0 = torch.empty_like(d)
    dh0[order] = d
    return (h, last, dxg) + ((dh0,) if s["h0"] is not None else ())


def _grid():
    v = [m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return torch.tensor(v[:-1], dtype=torch.float64, device="cuda")


def _codes64(x, r, root):
    """one tensor's numbers as 8 bits hold them: codes and powers of two"""
    n = x.shape[0]
    grid = _grid()
    group = torch.arange(n, device="cuda") // 32
    top = torch.zeros((n + 31) // 32, dtype=torch.float64, device="cuda").scatter_reduce_(0, group, x.abs(), "amax")
    k = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(min=-127)
    k = torch.where(top > 448 * _pow2(k), k + 1, k)                # logarithms may be off
    k = torch.where((top <= 224 * _pow2(k)) & (k > -127), k - 1, k)
    a = x.abs() / _pow2(k)[group]
    i = torch.searchsorted(grid, a, right=True).sub(1).clamp(max=len(grid) - 2)
    part = (a - grid[i]) / (grid[i + 1] - grid[i])
    up = part > r.double() / 65536
    if root:
        up |= (i == 0) & (a > 0)
    return torch.copysign(grid[i + up.long()], x), k.int() + 127


def _exact_adamw(case, s):
    t = s["step"] + 1
    low = case["fmt"] == 8
    g = s["g"].double()
    out = []
    if case["clip"]:
        norm = g.square().sum().sqrt().float()
        out.append(norm.double().view(1))
        if float(norm) > _CLIP:
            g = g * float(torch.tensor(_CLIP, dtype=torch.float32) / norm.cpu())
    if low:
        m0, v0 = (s[c].double() * _pow2(s[c + "s"].int() - 127).repeat_interleave(32) for c in ("m", "v"))
        v0 = v0.square()
    else:
        m0, v0 = s["m"].double(), s["v"].double()
    m = m0 + (1 - _B1) * (g - m0)
    v = v0 + (1 - _B2) * (g.square() - v0)
    w = s["w"].double()
    decay = s["decay"].double().expand(-1, 32).reshape(-1)
    w = w * (1 - _LR * decay) - _LR * (m / (1 - _B1 ** t)) / ((v / (1 - _B2 ** t)).sqrt() + _EPS)
    after = []
    if low:
        key = _mix(_mix(_mix(s["seed"] ^ (t * 0x9E3779B9 % (1 << 32))) ^ s["of"]))
        bits = _mix(key.repeat_interleave(32) ^ (s["place"].repeat_interleave(32) +
                                                 torch.arange(w.shape[0], device="cuda") % 32))
        m, ms = _codes64(m.float().double(), bits % 65536, False)
        v, vs = _codes64(v.sqrt().float().double(), bits // 65536, True)
        after = [ms.to(torch.uint8), vs.to(torch.uint8)]
    return out + [w, m, v] + ([w] if case["copy"] else []) + after


def exact(case, seed):
    """what run returns for prepare(case, seed), laid out the same, in 64 bits"""
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"linear": _exact_linear, "scan": _exact_scan, "adamw": _exact_adamw}[case["op"]](case, s)
