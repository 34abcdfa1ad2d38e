"""What the log-probability calls refuse is refused on the host, before anything is enqueued."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2509_23472_amd as L
from paper_2509_23472_amd import _lib, api
from paper_2509_23472_amd._lib import LoractLogprobParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SMALL, UNSUPPORTED = -1, -2, -3
X, T, LP, ST, TL, TI, WS, DL, DE, GR = (i << 40 for i in range(1, 11))


def test_parameter_structure(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    body = 'printf("%zu\\n", sizeof(loract_logprob_params));' + "".join('printf("%%zu\\n", offsetof(loract_logprob_params, %s));' % f[0]
                                                                        for f in LoractLogprobParams._fields_)
    src.write_text('#include "%s/include/loract.h"\n#include <stdio.h>\nint main(void) { %s return 0; }\n' % (ROOT, body))
    subprocess.run(["gcc", str(src), "-o", str(exe)], check=True)
    want = [int(v) for v in subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    assert [ctypes.sizeof(LoractLogprobParams)] + [getattr(LoractLogprobParams, f[0]).offset for f in LoractLogprobParams._fields_] == want
    values = [1, 2, 3, 4, 5, 6, 7, 8, 0.5]
    assert api._LOGPROB_PARAMS.pack(*values) == bytes(LoractLogprobParams(*values))


def _p(**kw):
    base = dict(m=100, n=32000, ld=32000, ldg=32000, dtype=1, target_bits=64, top=5, reserved=0, temperature=1.0)
    base.update(kw)
    return LoractLogprobParams(**base)


def _forward(p, x=X, t=T, lp=LP, st=ST, tl=TL, ti=TI, ws=WS, size=1 << 40):
    return _lib.load().loract_token_logprobs(x, t, ctypes.byref(p), lp, st, tl, ti, ws, size, None)


def _backward(p, x=X, t=T, st=ST, dl=DL, de=DE, gr=GR):
    return _lib.load().loract_token_logprobs_backward(x, t, ctypes.byref(p), st, dl, de, gr, None)


def _grad(p, x=X, t=T, dl=DL, de=DE, lp=LP, st=ST, gr=GR, ws=WS, size=1 << 40):
    return _lib.load().loract_token_logprobs_grad(x, t, ctypes.byref(p), dl, de, lp, st, gr, ws, size, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(m=0)), (INVALID, dict(n=0)), (INVALID, dict(ld=31999)), (INVALID, dict(dtype=2)), (INVALID, dict(target_bits=16)), (INVALID, dict(reserved=1)),
    (INVALID, dict(temperature=0.0)), (INVALID, dict(temperature=-1.0)), (INVALID, dict(temperature=NAN)), (INVALID, dict(temperature=INF)),
    (INVALID, dict(temperature=1e-300)), (UNSUPPORTED, dict(m=(1 << 30) + 1)), (UNSUPPORTED, dict(n=(1 << 30) + 1, ld=1 << 31, ldg=1 << 31))])
def test_refused_parameters(code, kw):
    p = _p(**kw)
    assert _forward(p) == code and _backward(p) == code and _grad(p) == code
    assert _lib.load().loract_token_logprobs_workspace_bytes(ctypes.byref(p), ctypes.byref(ctypes.c_size_t())) == code


def test_refused_operands():
    p = _p()
    for kw in (dict(x=None), dict(st=None), dict(tl=None), dict(ti=None), dict(t=None), dict(x=X + 1), dict(t=T + 4), dict(lp=LP + 2), dict(st=ST + 1), dict(tl=TL + 2),
               dict(ti=TI + 1), dict(ws=WS + 8)):
        assert _forward(p, **kw) == INVALID, kw
    assert _forward(_p(top=-1)) == INVALID and _forward(_p(n=4, top=5)) == INVALID and _forward(_p(top=65)) == UNSUPPORTED
    for kw in (dict(x=None), dict(st=None), dict(gr=None), dict(t=None), dict(dl=None, de=None), dict(dl=DL + 1), dict(de=DE + 2), dict(gr=GR + 1)):
        assert _backward(p, **kw) == INVALID and _grad(p, **kw) == INVALID, kw
    assert _grad(p, dl=None, t=None) == INVALID                      # (logp without targets)
    for kw in (dict(ldg=31999),):
        assert _backward(_p(**kw)) == INVALID and _grad(_p(**kw)) == INVALID


def test_workspace():
    p, out = _p(), ctypes.c_size_t(0)
    lib = _lib.load()
    assert lib.loract_token_logprobs_workspace_bytes(ctypes.byref(p), ctypes.byref(out)) == 0 and out.value > 0
    assert _forward(p, size=0) == SMALL and _forward(p, ws=None) == SMALL and _grad(p, size=0) == SMALL
    assert lib.loract_token_logprobs_workspace_bytes(ctypes.byref(p), None) == INVALID
    assert lib.loract_token_logprobs_workspace_bytes(None, ctypes.byref(out)) == INVALID
    many = _p(m=8192)
    assert lib.loract_token_logprobs_workspace_bytes(ctypes.byref(many), ctypes.byref(out)) == 0 and out.value == 0


def test_outputs_that_share_memory():
    p = _p()
    size = 100 * 32000 * 2
    for kw in (dict(lp=X + 4), dict(st=X + size - 4), dict(tl=T), dict(ti=TL), dict(lp=ST + 1196), dict(ws=X + 16), dict(ws=ST), dict(ti=T + 796)):
        assert _forward(p, **kw) == INVALID, kw
    for kw in (dict(gr=X + 2), dict(gr=X - 64), dict(gr=T), dict(gr=DL - 64), dict(gr=DE), dict(gr=ST)):
        assert _backward(p, **kw) == INVALID and _grad(p, **kw) == INVALID, kw
    assert _backward(_p(ldg=32008), gr=X) == INVALID                 # (in place: the same strides)
    assert _grad(p, lp=DL) == INVALID and _grad(p, st=DE + 396) == INVALID and _grad(p, ws=GR) == INVALID and _grad(p, lp=GR + 64) == INVALID


def test_the_binding_refuses(monkeypatch):
    x, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        L.loract_token_logprobs(x, t)                              # not on a GPU
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or 0
    monkeypatch.setattr(api._lib, "load", lambda: Library())
    d, st = torch.zeros(4), torch.zeros(3, 4)
    L.loract_token_logprobs(x, t, top=2)
    L.loract_token_logprobs_backward(x, t, st, d)
    L.loract_token_logprobs_grad(x, t, d, d, out=x)
    assert reached == ["loract_token_logprobs", "loract_token_logprobs_backward", "loract_token_logprobs_grad"]
    for call in (lambda: L.loract_token_logprobs(x[0], t), lambda: L.loract_token_logprobs(x, t[:3]), lambda: L.loract_token_logprobs(x, t.float()),
                 lambda: L.loract_token_logprobs(x.double(), t), lambda: L.loract_token_logprobs(x[:, ::2], t), lambda: L.loract_token_logprobs(x[:, :0], t),
                 lambda: L.loract_token_logprobs(x, torch.zeros(8, dtype=torch.int64)[::2]), lambda: L.loract_token_logprobs_backward(x, t, st, None),
                 lambda: L.loract_token_logprobs_backward(x, None, st, d), lambda: L.loract_token_logprobs_backward(x, t, st[:2], d),
                 lambda: L.loract_token_logprobs_backward(x, t, st, d[:3]), lambda: L.loract_token_logprobs_backward(x, t, st, d, out=x.bfloat16()),
                 lambda: L.loract_token_logprobs_backward(x, t, st, d, out=torch.zeros(4, 11)), lambda: L.loract_token_logprobs_grad(x, t, d.double()),
                 lambda: L.loract_token_logprobs_grad(x, None, d), lambda: L.loract_token_logprobs_grad(x[0], t, d)):
        with pytest.raises((ValueError, TypeError)):
            call()
    assert len(reached) == 3
