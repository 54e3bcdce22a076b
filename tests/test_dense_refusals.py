"""What the dense operators refuse, before anything is enqueued (no GPU needed), and the plain
forms that their GPU tests rest on."""
import math

import pytest
import torch

import paper_2510_03275_amd as P
from paper_2510_03275_amd import binding as Bd
from tests import dense_common as D

ARG, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -6, -9
A = 4096           # a 16-byte aligned address that no refused call reads
F16, BF16, F32 = P.SDQ_F16, P.SDQ_BF16, P.SDQ_F32


def _call(name, args, **change):
    vals = dict(args)
    vals.update(change)
    return getattr(Bd.lib(), name)(*vals.values())


QUANT = dict(x=A, xt=F16, m=2, k=8, q=A, s=A, stream=None)
LINEAR = dict(x=A, xt=F16, xs=None, m=2, w=A, ws=A, n=4, k=8, y=A, yt=F16, acc=0, space=A, bytes=1 << 30, stream=None)
GATED8 = dict(x=A, xt=F16, xs=None, m=2, g=A, gs=A, u=A, us=A, f=4, k=8, act=0, h=A, ht=F16, space=A, bytes=1 << 30,
              stream=None)
GATED = dict(x=A, t=F16, m=2, gate=A, up=A, f=4, k=8, act=0, h=A, g=None, u=None, kt=F16, space=A, bytes=1 << 30,
             stream=None)
BACK = dict(dh=A, x=A, t=F16, m=2, gate=A, up=A, f=4, k=8, act=0, g=A, u=A, kt=F16, dx=A, dgate=A, dup=A, acc=0,
            space=A, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("name,args,change,status", [
    ("sdq_int8_quantize", QUANT, dict(x=None), ARG), ("sdq_int8_quantize", QUANT, dict(q=None), ARG),
    ("sdq_int8_quantize", QUANT, dict(s=None), ARG), ("sdq_int8_quantize", QUANT, dict(xt=3), ARG),
    ("sdq_int8_quantize", QUANT, dict(m=-1), ARG), ("sdq_int8_quantize", QUANT, dict(k=0), ARG),
    ("sdq_int8_quantize", QUANT, dict(x=A + 2), ARG), ("sdq_int8_quantize", QUANT, dict(m=1 << 40), SHAPE),
    ("sdq_int8_linear", LINEAR, dict(x=None), ARG), ("sdq_int8_linear", LINEAR, dict(w=None), ARG),
    ("sdq_int8_linear", LINEAR, dict(ws=None), ARG), ("sdq_int8_linear", LINEAR, dict(y=None), ARG),
    ("sdq_int8_linear", LINEAR, dict(xt=3), ARG), ("sdq_int8_linear", LINEAR, dict(yt=-1), ARG),
    ("sdq_int8_linear", LINEAR, dict(m=-1), ARG), ("sdq_int8_linear", LINEAR, dict(n=-1), ARG),
    ("sdq_int8_linear", LINEAR, dict(k=0), ARG), ("sdq_int8_linear", LINEAR, dict(k=131072), SHAPE),
    ("sdq_int8_linear", LINEAR, dict(m=1 << 31), SHAPE), ("sdq_int8_linear", LINEAR, dict(m=1 << 29, n=1 << 29), SHAPE),
    ("sdq_int8_linear", LINEAR, dict(w=A + 1), ARG), ("sdq_int8_linear", LINEAR, dict(y=A + 8), ARG),
    ("sdq_int8_linear", LINEAR, dict(space=None), WORKSPACE), ("sdq_int8_linear", LINEAR, dict(bytes=15), WORKSPACE),
    ("sdq_int8_linear", LINEAR, dict(space=A + 4), ARG),
    ("sdq_int8_gated_linear", GATED8, dict(act=2), ARG), ("sdq_int8_gated_linear", GATED8, dict(u=None), ARG),
    ("sdq_int8_gated_linear", GATED8, dict(gs=None), ARG), ("sdq_int8_gated_linear", GATED8, dict(ht=5), ARG),
    ("sdq_int8_gated_linear", GATED8, dict(h=A + 2), ARG), ("sdq_int8_gated_linear", GATED8, dict(k=131072), SHAPE),
    ("sdq_int8_gated_linear", GATED8, dict(bytes=0), WORKSPACE),
    ("sdq_gated_linear", GATED, dict(t=F32), UNSUPPORTED), ("sdq_gated_linear", GATED, dict(t=7), ARG),
    ("sdq_gated_linear", GATED, dict(act=-1), ARG), ("sdq_gated_linear", GATED, dict(g=A), ARG),
    ("sdq_gated_linear", GATED, dict(up=None), ARG), ("sdq_gated_linear", GATED, dict(x=A + 2), ARG),
    ("sdq_gated_linear", GATED, dict(g=A, u=A, kt=BF16), ARG), ("sdq_gated_linear_backward", BACK, dict(kt=BF16), ARG),
    ("sdq_gated_linear_backward", BACK, dict(kt=3), ARG), ("sdq_gated_linear", GATED, dict(g=A, u=A + 2), ARG), ("sdq_gated_linear", GATED, dict(k=-3), ARG),
    ("sdq_gated_linear_backward", BACK, dict(t=F32), UNSUPPORTED), ("sdq_gated_linear_backward", BACK, dict(act=9), ARG),
    ("sdq_gated_linear_backward", BACK, dict(dgate=None), ARG), ("sdq_gated_linear_backward", BACK, dict(g=None), ARG),
    ("sdq_gated_linear_backward", BACK, dict(dh=None), ARG), ("sdq_gated_linear_backward", BACK, dict(gate=None), ARG),
    ("sdq_gated_linear_backward", BACK, dict(x=None), ARG), ("sdq_gated_linear_backward", BACK, dict(dx=A + 2), ARG),
    ("sdq_gated_linear_backward", BACK, dict(bytes=31), WORKSPACE),
    ("sdq_gated_linear_backward", BACK, dict(space=None), WORKSPACE),
    ("sdq_gated_linear_backward", BACK, dict(m=1 << 29, f=1 << 29), SHAPE),
])
def test_refused(name, args, change, status):
    assert _call(name, args, **change) == status
    assert Bd.lib().sdq_last_error()


def test_no_ops():
    assert _call("sdq_int8_quantize", QUANT, m=0, x=None, q=None, s=None) == 0
    assert _call("sdq_int8_linear", LINEAR, m=0, x=None, y=None, space=None, bytes=0) == 0
    assert _call("sdq_int8_linear", LINEAR, n=0, w=None, y=None, space=None, bytes=0) == 0
    assert _call("sdq_int8_gated_linear", GATED8, f=0, h=None) == 0
    assert _call("sdq_gated_linear", GATED, m=0, x=None, h=None) == 0
    assert _call("sdq_gated_linear_backward", BACK, dx=None, dgate=None, dup=None) == 0


def test_workspace_bytes():
    for fn in (P.sdq_int8_linear_workspace_bytes, P.sdq_int8_gated_linear_workspace_bytes):
        assert fn(0, 5, 8) == 0 and fn(5, 0, 8) == 0 and fn(1, 1, 131072) == 0 and fn(-1, 4, 4) == 0
        assert fn(3, 100, 1000) >= 3 * 1000 + 12
        assert fn(300, 100, 1000) >= 300 * 1000 + 1200
    assert P.sdq_gated_linear_workspace_bytes(0, 4, 4) == 0 and P.sdq_gated_linear_workspace_bytes(1, 4, -4) == 0
    assert P.sdq_gated_linear_backward_workspace_bytes(100, 50, 8) >= 2 * 100 * 50 * 2
    assert P.sdq_gated_linear_backward_workspace_bytes(1 << 40, 50, 8) == 0


def test_host_tensors_are_refused():
    x = torch.zeros(2, 8)
    w = P.Int8Rows(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4))
    h = torch.zeros(4, 8, dtype=torch.float16)
    for fn in (lambda: P.int8_quantize(x), lambda: P.int8_linear(x, w), lambda: P.int8_gated_linear(x, w, w),
               lambda: P.gated_linear(h, h, h), lambda: P.gated_linear_backward(h, h, h, h, h, h)):
        with pytest.raises(ValueError):
            fn()


@pytest.mark.parametrize("act", [0, 1])
def test_plain_gradients_are_the_formulas(act):
    """act' of the plain form against differences and against torch's activations."""
    g = torch.linspace(-9, 9, 721, dtype=torch.float64)
    a, da = D.act_ref(g, act)
    num = (D.act_ref(g + 1e-6, act)[0] - D.act_ref(g - 1e-6, act)[0]) / 2e-6
    assert float((da - num).abs().max()) < 1e-8
    want = torch.nn.functional.silu(g) if act == 0 else torch.nn.functional.gelu(g, approximate="tanh")
    assert float((a - want).abs().max()) < 1e-12
    assert float(da.abs().max()) < 1.2              # as the bound of the gated block takes it


def test_plain_quantiser():
    x = torch.tensor([[0.5, 1.5, 2.5, -0.5, -1.5, 127.0], [0, 0, 0, 0, 0, 0], [1, math.inf, 0, 0, 0, 0]])
    q, s = D.quantize_ref(x)
    assert q[0].tolist() == [0, 2, 2, 0, -2, 127] and float(s[0]) == 1.0
    assert not q[1].any() and float(s[1]) == 2.0 ** -126 and not q[2].any() and math.isnan(float(s[2]))


def test_native_and_ctypes_calls_answer_alike(monkeypatch):
    """The native calls of the per-token entry points and the ctypes ones that stand in for them."""
    import sys
    import types
    stream = types.SimpleNamespace(cuda_stream=0)
    x, w, s = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    names = ("_call_int8_linear", "_call_int8_gated_linear", "_call_gated_linear")
    native = [getattr(Bd, n) for n in names]
    monkeypatch.setitem(sys.modules, "paper_2510_03275_amd._sdqcall", None)
    monkeypatch.delattr(P, "_sdqcall", raising=False)
    plain = Bd._native_dense_calls()
    seen = []
    for calls in (native, plain):
        for n, c in zip(names, calls):
            monkeypatch.setattr(Bd, n, c)
        got = []
        for fn in (lambda: P.sdq_int8_linear(x, w, s, torch.zeros(2, 4), None, stream),      # 2 rows of 8: no workspace
                   lambda: P.sdq_int8_linear(x.new_zeros(0, 8), w, s, torch.zeros(0, 4), None, stream),
                   lambda: P.sdq_int8_gated_linear(x, w, s, w, s, 5, x, x, stream),
                   lambda: P.sdq_int8_gated_linear(torch.zeros(99, 600), w.new_zeros(4, 600), s, w.new_zeros(4, 600), s, 0,
                                                   x, x, stream),
                   lambda: P.sdq_gated_linear(x, x, x, 7, x, x, stream),
                   lambda: P.sdq_gated_linear(x, x, x, 0, x, x, stream, g=x)):
            try:
                fn()
                got.append(0)
            except P.SdqError as e:
                got.append((e.status, str(e)))
        seen.append(got)
    assert seen[0] == seen[1]
    assert [g if g == 0 else g[0] for g in seen[0]] == [WORKSPACE, 0, ARG, WORKSPACE, ARG, ARG]
