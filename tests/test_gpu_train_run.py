"""Products, gated recurrence and AdamW together, as programs run them: a training step of a memory
model with its gradients and the step over its weights, captured and not, and the memory kept event
by event while serving."""
import numpy as np
import pytest
import torch

import paper_2607_05095_amd as fast
from tests.parity import to_dev
from tests.plain64 import U

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-2, 0.9, 0.99, 1e-8
LENGTHS = [5, 0, 1, 300, 17, 8, 0, 150, 40, 3]
IN, D, OUT = 50, 36, 30


class Model:
    """features -> [x | gate] -> recurrence over each segment -> gelu rows, and back"""

    def __init__(self, seed):
        r = np.random.default_rng(seed)
        f = lambda *s: torch.from_numpy(r.normal(size=s).astype(np.float32))
        self.off = np.concatenate([[0], np.cumsum(LENGTHS)]).astype(np.int32)
        self.N, self.E = len(LENGTHS), int(self.off[-1])
        self.feat, self.h0, self.dy, self.dl = f(self.E, IN), f(self.N, D), f(self.E, OUT), f(self.N, D)
        self.dt = torch.from_numpy(r.exponential(size=self.E).astype(np.float32))
        self.w = [f(2 * D, IN) / IN ** 0.5, 0.1 * f(2 * D), f(OUT, D) / D ** 0.5, 0.1 * f(OUT)]
        self.m = [0.1 * f(*w.shape) for w in self.w]
        self.v = [1 + f(*w.shape) ** 2 for w in self.w]

    def device(self):
        d = dict(off=to_dev(self.off))
        for k in ("feat", "h0", "dy", "dl", "dt"):
            d[k] = getattr(self, k).cuda()
        for k in ("w", "m", "v"):
            d[k] = [t.cuda() for t in getattr(self, k)]
        z = lambda *s: torch.full(s, 7.0, device="cuda")
        E, N = self.E, self.N
        d.update(xg=z(E, 2, D), h=z(E, D), last=z(N, D), keep=z(fast.fast_gated_scan_state_rows(E), D), y=z(E, OUT),
                 pre=z(E, OUT), dh=z(E, D), dxg=z(E, 2, D), dh0=z(N, D), df=z(E, IN), norm=z(1), scale=z(1),
                 g=[z(*w.shape) for w in self.w], step=torch.zeros(1, dtype=torch.int64, device="cuda"))
        d["copy"] = [torch.zeros(w.shape, dtype=torch.bfloat16, device="cuda") for w in self.w]
        flat = lambda ts: [t.view(-1) for t in ts]
        d["list"] = fast.adamw_tensors(flat(d["w"]), flat(d["g"]), flat(d["m"]), flat(d["v"]), copy=flat(d["copy"]),
                                       decay=[0.1, 0.0, 0.1, 0.0])
        d["blk"] = fast.tcsr(d["off"], E)
        sizes = [fast.fast_linear_bwd_workspace(E, D, OUT, 0, fast.ACT_GELU),
                 fast.fast_linear_bwd_workspace(E, IN, 2 * D, 0, fast.ACT_NONE), fast.fast_gated_scan_workspace(N, E, D),
                 fast.fast_grad_norm_workspace(sum(w.numel() for w in self.w), 4)]
        d["wsb"] = max(sizes)
        d["ws"] = torch.empty(d["wsb"], dtype=torch.uint8, device="cuda")    # one for all: the calls run in order
        return d

    def run(self, d, stream=None):
        E, ws, wsb = self.E, d["ws"], d["wsb"]
        x, gate = d["xg"][:, 0], d["xg"][:, 1]
        fast.fast_linear_fwd(E, IN, 2 * D, 0, d["feat"], IN, d["w"][0], d["w"][1], fast.ACT_NONE, None, 2 * D, d["xg"], 2 * D)
        fast.fast_gated_scan_fwd(d["blk"], D, 0, x, gate, 2 * D, d["dt"], d["h0"], 0, d["h"], d["last"], d["keep"], ws, wsb)
        fast.fast_linear_fwd(E, D, OUT, 0, d["h"], D, d["w"][2], d["w"][3], fast.ACT_GELU, None, OUT, d["y"], OUT, d["pre"])
        fast.fast_linear_bwd(E, D, OUT, 0, d["h"], D, d["w"][2], fast.ACT_GELU, d["pre"], d["dy"], OUT, d["dh"], D, d["g"][2],
                             d["g"][3], ws, wsb)
        fast.fast_gated_scan_bwd(d["blk"], D, 0, x, gate, 2 * D, d["dt"], d["h0"], 0, d["keep"], d["dh"], d["dl"],
                                 d["dxg"][:, 0], d["dxg"][:, 1], 2 * D, d["dh0"], ws, wsb)
        fast.fast_linear_bwd(E, IN, 2 * D, 0, d["feat"], IN, d["w"][0], fast.ACT_NONE, None, d["dxg"], 2 * D, d["df"], IN,
                             d["g"][0], d["g"][1], ws, wsb)
        fast.fast_grad_norm(d["list"], 0, 5.0, d["norm"], d["scale"], ws, wsb)
        d["step"].add_(1)
        fast.fast_adamw(d["list"], 0, fast.STATE_F32, LR, B1, B2, EPS, 1, 0, None, d["step"], d["scale"])


def test_training_step_and_its_gradients():
    """Against 64-bit autograd on the host.  Three fp32 stages forward and back, each within about 100 U of its
    operands' magnitude (at most about 20 here): 5000 U of the largest gradient."""
    print("[run] memory model, one step", flush=True)
    M = Model(1)
    d = M.device()
    M.run(d)
    leaves = [t.double().requires_grad_() for t in (M.feat, M.h0, *M.w)]
    feat, h0, w1, b1, w2, b2 = leaves
    xg = feat @ w1.t() + b1
    x, gate = xg[:, :D], xg[:, D:]
    a = torch.exp(-torch.nn.functional.softplus(gate) * M.dt.double()[:, None])
    rows, last = [], []
    for v in range(M.N):
        s = h0[v]
        for e in range(M.off[v], M.off[v + 1]):
            s = a[e] * s + (1 - a[e]) * x[e]
            rows.append(s)
        last.append(s)
    h, last = torch.stack(rows), torch.stack(last)
    z = h @ w2.t() + b2
    y = z * 0.5 * torch.erfc(-z / 2 ** 0.5)
    ((y * M.dy.double()).sum() + (last * M.dl.double()).sum()).backward()
    got = [("y", d["y"], y), ("h", d["h"], h), ("last", d["last"], last), ("df", d["df"], feat.grad),
           ("dh0", d["dh0"], h0.grad)] + [(f"g{k}", d["g"][k], leaves[2 + k].grad) for k in range(4)]
    for name, t, want in got:
        err = (t.double().cpu() - want.detach()).abs().max()
        assert err <= 5000 * U * want.abs().max(), (name, float(err), float(want.abs().max()))
    norm = float(torch.sqrt(sum((leaves[2 + k].grad ** 2).sum() for k in range(4))))
    assert abs(float(d["norm"]) - norm) <= 5000 * U * norm and norm > 5
    for k in range(4):
        g = leaves[2 + k].grad * (5.0 / norm)
        m = B1 * M.m[k].double() + (1 - B1) * g
        v = B2 * M.v[k].double() + (1 - B2) * g * g
        decay = 0.1 if k % 2 == 0 else 0.0
        w = M.w[k].double()
        want = w - LR * (decay * w + (m / (1 - B1)) / ((v / (1 - B2)).sqrt() + EPS))
        assert ((d["w"][k].double().cpu() - want).abs() <= U * want.abs() * 2 + LR * 1e-3 * (1 + g.abs())).all()
        assert torch.equal(d["copy"][k], d["w"][k].bfloat16())


def test_training_steps_captured_and_replayed():
    print("[run] memory model, captured", flush=True)
    M = Model(2)
    one, two = M.device(), M.device()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                          # (warm, on its own copy)
        M.run(M.device())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.run(one)
    assert int(one["step"]) == 0
    for t in range(1, 5):
        for k in ("xg", "h", "y", "dh", "dxg", "df"):
            one[k].fill_(-1)
        graph.replay()
        M.run(two)
        torch.cuda.synchronize()
        assert int(one["step"]) == t
        for k in ("y", "last", "df", "dh0", "norm"):
            assert torch.equal(one[k], two[k]), (t, k)
        for k in ("w", "m", "v", "g", "copy"):
            assert all(torch.equal(a, b) for a, b in zip(one[k], two[k])), (t, k)
    assert not torch.equal(one["w"][0], M.w[0].cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_memory_kept_event_by_event(dtype):
    """Batches of one event per node against the whole histories at once: the same bits (segments that are
    not cut walk their events in the same order)."""
    print("[run] serving", flush=True)
    V, D, steps = 300, 50, 20
    code = fast.F32 if dtype == torch.float32 else fast.BF16
    g = torch.Generator(device="cuda").manual_seed(3)
    xg = torch.randn(V, steps, 2, D, generator=g, device="cuda").to(dtype)
    dt = torch.rand(V, steps, generator=g, device="cuda")
    there = torch.rand(V, steps, generator=g, device="cuda") < 0.7
    memory = torch.randn(V, D, generator=g, device="cuda")
    off = torch.zeros(V + 1, dtype=torch.int32, device="cuda")
    off[1:] = there.sum(1).cumsum(0)
    E = int(off[-1])
    allx = xg[there]
    h, last = torch.empty(E, D, dtype=dtype, device="cuda"), torch.empty(V, D, device="cuda")
    wsb = fast.fast_gated_scan_workspace(V, E, D)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    fast.fast_gated_scan_fwd(fast.tcsr(off, E), D, code, allx[:, 0], allx[:, 1], 2 * D, dt[there], memory, steps, h, last,
                             None, ws, wsb)
    outs = torch.empty(V, steps, D, dtype=dtype, device="cuda")
    for t in range(steps):
        nodes = there[:, t].nonzero().view(-1)
        n = len(nodes)
        rows = memory[nodes]                               # the nodes' memories, updated in place
        ev = xg[nodes, t].contiguous()
        o = torch.empty(n, D, dtype=dtype, device="cuda")
        one = fast.tcsr(torch.arange(n + 1, dtype=torch.int32, device="cuda"), n)
        b = fast.fast_gated_scan_workspace(n, n, D)
        fast.fast_gated_scan_fwd(one, D, code, ev[:, 0], ev[:, 1], 2 * D, dt[nodes, t].contiguous(), rows, 1, o, rows, None,
                                 ws, max(b, 1))
        memory[nodes] = rows
        outs[nodes, t] = o
    assert torch.equal(memory, last) and torch.equal(outs[there], h)
