"""Calls of the products, the recurrence and the AdamW step that are refused before any launch: sizes whose launches do
not fit, workspaces among a call's arrays, lists of tensors of other types than the step takes.  Without a GPU."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2607_05095_amd as fast
from tests.test_train_abi import BWD, INVALID, NORM, SB, SF, UNSUPPORTED, at, call, scan_call, tensors

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAR = 1 << 48                            # from one array to the next, where a case's arrays are large


# ------------------------------------------------------------------ lists of tensors
F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8
LISTS = dict(w=[F32, F32], grad=[F32, F32], m=[F32, F32], v=[F32, F32])
LOW = dict(w=[F32, F32], grad=[BF16, BF16], m=[U8, U8], v=[U8, U8], m_scale=[U8, U8], v_scale=[U8, U8], copy=[BF16, BF16])


def lists(types, n=96, **kw):
    d = {k: [torch.zeros((n + 31) // 32 if "scale" in k else n, dtype=t) for t in ts] for k, ts in dict(types, **kw).items()}
    return lambda: fast.adamw_tensors(**d)


@pytest.mark.parametrize("types,kw,name", [
    (LISTS, dict(w=[F32, BF16]), "tensor 1: w of torch.bfloat16"), (LISTS, dict(w=[torch.float64, F32]), "tensor 0: w of"),
    (LISTS, dict(grad=[F32, BF16]), "tensor 0: grad of torch.float32"), (LISTS, dict(grad=[torch.float16, F32]), "tensor 0: grad of"),
    (LISTS, dict(grad=[BF16, torch.float64]), "tensor 1: grad of"), (LISTS, dict(m=[F32, U8]), "tensor 0: m of torch.float32"),
    (LISTS, dict(m=[BF16, BF16]), "tensor 0: m of"), (LISTS, dict(v=[F32, BF16]), "tensor 1: v of"),
    (LISTS, dict(v=[U8, U8]), "tensor 0: v of"), (LOW, dict(v=[F32, F32]), "tensor 0: v of"), (LOW, dict(m=[U8, F32]), "tensor 1: m of"),
    (LOW, dict(m_scale=[F32, U8]), "tensor 0: m_scale of"), (LOW, dict(v_scale=[U8, torch.int32]), "tensor 1: v_scale of"),
    (LISTS, dict(copy=[F32, BF16]), "tensor 0: copy of"), (LISTS, dict(copy=[BF16, torch.float16]), "tensor 1: copy of")])
def test_adamw_tensors_of_other_types_are_refused(types, kw, name):
    """A step reads and writes each array at its own type's size: one of a smaller type would be passed by."""
    with pytest.raises(fast.FastError) as e:
        lists(types, **kw)()
    assert name in str(e.value)


def test_adamw_tensors_of_the_types_named_are_taken():
    """What is left to refuse here is that there is no GPU."""
    for types, kw in ((LISTS, {}), (LOW, {}), (LISTS, dict(grad=[BF16, BF16], copy=[BF16, BF16])),
                      (LOW, dict(m=2 * [torch.float8_e4m3fn], v_scale=2 * [torch.float8_e8m0fnu]))):
        with pytest.raises(fast.FastError) as e:
            lists(types, **kw)()
        assert "not on the current GPU" in str(e.value)
    assert fast.adamw_tensors([], [], [], [])._count == 0


def test_adamw_and_norm_refuse_a_list_of_other_types(monkeypatch):
    """A call names the types of grads and states; they are those that its list was built of."""
    monkeypatch.setattr(fast, "_resident", lambda *a: None)
    wide, low = lists(LISTS)(), lists(LOW)()
    step = dict(lr=1e-3, beta1=.9, beta2=.999, eps=1e-8, step=1)
    for ts, grad, form in ((wide, fast.BF16, fast.STATE_F32), (wide, fast.F32, fast.STATE_MXFP8),
                           (low, fast.F32, fast.STATE_MXFP8), (low, fast.BF16, fast.STATE_F32)):
        with pytest.raises(fast.FastError) as e:
            fast.fast_adamw(ts, grad, form, **step)
        assert "the list holds" in str(e.value)
    for ts, grad in ((wide, fast.BF16), (low, fast.F32)):
        with pytest.raises(fast.FastError) as e:
            fast.fast_grad_norm(ts, grad, 1.0, at(1), at(2), at(3), 1 << 20)
        assert "the list holds" in str(e.value)


# ------------------------------------------------------------------ launches
@pytest.mark.parametrize("kw", [
    # dz: 64 rows a workgroup of 256 threads
    dict(n=(1 << 30) - 63, K=1, M=1, act=3), dict(n=1 << 30, K=1, M=1, act=2, dw=None), dict(n=1 << 30, K=1, M=1, act=1, dx=None),
    dict(n=(1 << 31) - 1, K=1, M=1, act=1, dx=None, dw=None),
    # the weight gradient: 2^17 splits of 128 tiles, 256 threads each
    dict(n=(1 << 31) - 16383, K=1, M=16384, act=0, pre=None, dx=None), dict(n=(1 << 31) - 16383, K=1, M=16384, act=0, pre=None, dw=None)])
def test_linear_bwd_refuses_launches_of_2_32_threads(kw):
    a = {k: FAR * (j + 1) for j, k in enumerate(("x", "w", "pre", "dy", "dx", "dw", "db", "ws"))}
    a.update(dt=1, ldx=kw["K"], lddx=kw["K"], lddy=kw["M"], wsb=1 << 62)
    a.update(kw)
    assert call("fast_linear_bwd", BWD, a) == UNSUPPORTED
    assert "2^32 threads" in fast.fast_last_error()


# ------------------------------------------------------------------ workspaces
def test_linear_bwd_refuses_a_workspace_among_its_arrays():
    """On each array, and one whose end reaches into the next."""
    need = fast.fast_linear_bwd_workspace(5, 10, 6, 0, 1)
    for kw in ([dict(ws=at(k)) for k in (1, 2, 3, 4, 5, 6, 7)] + [dict(ws=at(k) - need // 256 * 256 + 256) for k in (1, 4, 6)] +
               [dict(dw=at(8) + need - 4), dict(dx=at(8) + need - 4), dict(db=at(8) + 512)]):
        assert call("fast_linear_bwd", BWD, kw) == INVALID, kw
        assert "the workspace overlaps" in fast.fast_last_error()


@pytest.mark.parametrize("name,defaults,arrays", [("fast_gated_scan_fwd", SF, (1, 2, 3, 4, 5, 6, 7, 20)),
                                                  ("fast_gated_scan_bwd", SB, (1, 2, 3, 4, 7, 9, 10, 11, 12, 13, 20))])
def test_gated_scan_refuses_a_workspace_among_its_arrays(name, defaults, arrays):
    need = fast.fast_gated_scan_workspace(4, 200, 10)
    for kw in [dict(ws=at(k)) for k in arrays] + [dict(ws=at(k) - need // 256 * 256 + 256) for k in arrays[:3]]:
        assert scan_call(name, defaults, kw) == INVALID, kw
        assert "the workspace overlaps" in fast.fast_last_error()


def test_grad_norm_refuses_a_workspace_among_grads():
    other = dict(grad=at(12))
    for ws in (at(2), at(2) + 392, at(12) + 8):
        a = dict(NORM, t=tensors({}, other), count=2, ws=ws)
        assert fast.lib().fast_grad_norm(*a.values()) == INVALID
        assert "the workspace overlaps" in fast.fast_last_error()


# ------------------------------------------------------------------ small threads
SMALL = """
import ctypes, threading
import paper_2607_05095_amd as fast
from tests.test_train_abi import STEP, tensors
f = fast.lib().fast_adamw
a = list(dict(STEP, t=tensors({}, {}), count=2).values())
f(*a)                                    # (refused: one tensor twice)
got = []
threading.stack_size(96 << 10)
t = threading.Thread(target=lambda: got.append(f(*a)))
t.start()
t.join()
print("status", got)
"""


def test_adamw_runs_on_a_small_stack():
    """A thread of 96 KB; the call's list of ranges, 115 KB at its longest, is elsewhere."""
    r = subprocess.run([sys.executable, "-c", SMALL], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "status [1]" in r.stdout, (r.returncode, r.stdout, r.stderr[-500:])
