"""CPU-side checks of the sub-layer's entry points: what is refused is refused on the host, before anything is enqueued."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2509_23472_amd import _lib
from paper_2509_23472_amd._lib import LoractLinearParams, LoractQkParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(4096)
INVALID, SMALL, UNSUPPORTED = -1, -2, -3


def test_parameter_structures_match_the_header(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    fields = [("loract_linear_params", LoractLinearParams), ("loract_qk_params", LoractQkParams)]
    body = "".join('printf("%%zu\\n", sizeof(%s));' % name + "".join('printf("%%zu\\n", offsetof(%s, %s));' % (name, f[0]) for f in t._fields_)
                   for name, t in fields)
    src.write_text('#include "%s/include/loract.h"\n#include <stdio.h>\nint main(void) { %s return 0; }\n' % (ROOT, body))
    subprocess.run(["gcc", str(src), "-o", str(exe)], check=True)
    want = [int(v) for v in subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    got = [v for _, t in fields for v in [ctypes.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]]
    assert got == want


def test_packed_parameters_are_the_structures():
    from paper_2509_23472_amd import api
    values = list(range(1, 15)) + [0.5, 0.25, 2 ** 64 - 3]
    assert api._LINEAR_PARAMS.pack(*values) == bytes(LoractLinearParams(*values))
    values = list(range(1, 9)) + [0.5] + list(range(20, 32))
    assert api._QK_PARAMS.pack(*values) == bytes(LoractQkParams(*values))


def _linear(**kw):
    base = dict(m=64, n_in=32, n_out=48, ldx=32, ldw=32, ldr=48, ldy=48, ldz=48, ldp=48, dtype=1, out_dtype=1, w_layout=0, act=0, r_lora=0,
                lora_scale=1.0, p_drop=0.0, seed=0)
    base.update(kw)
    return LoractLinearParams(**base)


def _call_linear(p, x=FAKE, w=FAKE, t=None, b=None, res=None, y=FAKE, z=None, ws=FAKE, size=1 << 40):
    return _lib.load().loract_linear(x, w, None, t, b, res, ctypes.byref(p), y, z, ws, size, None)


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(m=0)), (INVALID, dict(n_in=0)), (INVALID, dict(n_out=-1)), (INVALID, dict(ldx=31)), (INVALID, dict(ldw=31)),
    (INVALID, dict(w_layout=1, ldw=47)), (INVALID, dict(ldy=47)), (INVALID, dict(w_layout=2)), (INVALID, dict(act=4)), (INVALID, dict(act=-1)),
    (INVALID, dict(dtype=2)), (INVALID, dict(out_dtype=5)), (INVALID, dict(r_lora=-1)), (INVALID, dict(r_lora=4)), (INVALID, dict(p_drop=1.0)),
    (INVALID, dict(p_drop=-0.1)), (INVALID, dict(p_drop=float("nan"))), (UNSUPPORTED, dict(dtype=0, out_dtype=1)), (UNSUPPORTED, dict(r_lora=65)),
    (UNSUPPORTED, dict(m=(1 << 30) + 1)), (UNSUPPORTED, dict(n_in=1 << 31, ldx=1 << 31, ldw=1 << 31))])
def test_linear_refusals(code, kw):
    assert _call_linear(_linear(**kw)) == code


def test_linear_refuses_null_pointers_short_rows_and_small_workspaces():
    lib = _lib.load()
    p = _linear()
    assert _call_linear(p, x=None) == INVALID and _call_linear(p, w=None) == INVALID and _call_linear(p, y=None) == INVALID
    assert _call_linear(_linear(ldr=47), res=FAKE) == INVALID and _call_linear(_linear(ldz=47), z=FAKE) == INVALID
    assert _call_linear(_linear(r_lora=4), t=FAKE) == INVALID and _call_linear(_linear(r_lora=4), b=FAKE) == INVALID
    assert lib.loract_linear(FAKE, FAKE, None, None, None, None, None, FAKE, None, FAKE, 1 << 40, None) == INVALID
    out = ctypes.c_size_t(0)
    split = _linear(m=64, n_in=8192, ldx=8192, ldw=8192)               # few tiles, a long sum: K is split
    assert lib.loract_linear_workspace_bytes(ctypes.byref(split), ctypes.byref(out)) == 0 and out.value > 0 and out.value % 256 == 0
    assert _call_linear(split, size=out.value - 1) == SMALL and _call_linear(split, ws=None) == SMALL
    assert _call_linear(split, ws=ctypes.c_void_p(4104)) == INVALID
    assert lib.loract_linear_workspace_bytes(None, ctypes.byref(out)) == INVALID
    assert lib.loract_linear_workspace_bytes(ctypes.byref(p), None) == INVALID


def _call_backward(p, dy=FAKE, z=FAKE, t=None, dp=FAKE, db=FAKE, d_b=None, ws=FAKE, size=1 << 40):
    return _lib.load().loract_linear_backward(dy, z, t, ctypes.byref(p), dp, db, d_b, ws, size, None)


def test_linear_backward_refusals():
    for kw in (dict(m=0), dict(n_out=0), dict(ldy=47), dict(ldp=47), dict(act=9), dict(dtype=3), dict(p_drop=1.5), dict(r_lora=-2)):
        assert _call_backward(_linear(**kw)) == INVALID, kw
    assert _call_backward(_linear(r_lora=65)) == UNSUPPORTED
    assert _call_backward(_linear(), dy=None) == INVALID and _call_backward(_linear(), dp=None) == INVALID
    assert _call_backward(_linear(act=2), z=None) == INVALID and _call_backward(_linear(act=2, ldz=3)) == INVALID
    assert _call_backward(_linear(r_lora=4), d_b=FAKE) == INVALID                       # no T
    assert _call_backward(_linear(), t=FAKE, d_b=FAKE) == INVALID                       # no rank
    out = ctypes.c_size_t(0)
    p = _linear(r_lora=16)
    assert _lib.load().loract_linear_backward_workspace_bytes(ctypes.byref(p), ctypes.byref(out)) == 0 and out.value > 0
    assert _call_backward(p, ws=None) == SMALL and _call_backward(p, t=FAKE, d_b=FAKE, size=16) == SMALL
    assert _call_backward(p, ws=ctypes.c_void_p(4097)) == INVALID


def test_dropout_refusals():
    f = lambda x=FAKE, ldx=8, r=None, ldr=0, m=4, n=8, dt=0, p=0.1, y=FAKE, ldy=8: _lib.load().loract_dropout(x, ldx, r, ldr, m, n, dt, p, 0, y, ldy, None)
    for kw in (dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(r=FAKE, ldr=7), dict(m=0), dict(n=0), dict(dt=4), dict(p=1.0), dict(p=-1.0),
               dict(p=float("nan"))):
        assert f(**kw) == INVALID, kw
    assert f(m=1 << 31) == UNSUPPORTED


def _qk(**kw):
    base = dict(m=4, heads_q=2, heads_k=1, d=64, rot=64, interleaved=0, dtype=1, n_pos=8, eps=1e-6)
    base.update(kw)
    return LoractQkParams(**base)


def test_qknorm_rope_refusals():
    lib = _lib.load()

    def forward(p, q=FAKE, k=FAKE, table=FAKE, qo=FAKE, ko=FAKE):
        return lib.loract_qknorm_rope_forward(q, k, ctypes.byref(p), None, None, table, None, qo, ko, None)

    def backward(p, q=FAKE, k=FAKE, dqo=FAKE, dko=FAKE, dq=FAKE, dk=FAKE, gq=FAKE, gk=FAKE, ws=FAKE, size=1 << 40):
        return lib.loract_qknorm_rope_backward(q, k, ctypes.byref(p), None, None, FAKE, None, dqo, dko, dq, dk, gq, gk, ws, size, None)

    for kw in (dict(m=0), dict(heads_q=0), dict(heads_k=-1), dict(d=0), dict(rot=3), dict(rot=66), dict(rot=-2), dict(dtype=2), dict(eps=-1.0),
               dict(eps=float("nan")), dict(n_pos=0)):
        assert forward(_qk(**kw)) == INVALID, kw
        assert backward(_qk(**kw)) == INVALID, kw
    assert forward(_qk(d=1026, rot=2)) == UNSUPPORTED and forward(_qk(m=1 << 31)) == UNSUPPORTED
    for kw in (dict(q=None), dict(k=None), dict(table=None), dict(qo=None), dict(ko=None)):
        assert forward(_qk(), **kw) == INVALID, kw
    for kw in (dict(q=None), dict(k=None), dict(dqo=None), dict(dko=None), dict(dq=None), dict(dk=None)):
        assert backward(_qk(), **kw) == INVALID, kw
    assert backward(_qk(heads_k=0)) == INVALID                                          # a gradient of keys that are not there
    assert backward(_qk(), ws=None) == SMALL and backward(_qk(), size=8) == SMALL and backward(_qk(), ws=ctypes.c_void_p(4100)) == INVALID
    out = ctypes.c_size_t(0)
    assert lib.loract_qknorm_rope_workspace_bytes(ctypes.byref(_qk()), ctypes.byref(out)) == 0 and out.value > 0
    assert lib.loract_qknorm_rope_workspace_bytes(None, ctypes.byref(out)) == INVALID
    for args in ((None, 4, 8, 1e4, 0), (FAKE, 0, 8, 1e4, 0), (FAKE, 4, 7, 1e4, 0), (FAKE, 4, 0, 1e4, 0), (FAKE, 4, 8, 0.0, 0), (FAKE, 4, 8, 1e4, -1)):
        assert lib.loract_rope_table(*args, None) == INVALID, args


def test_binding_refuses_tensors_that_are_not_on_the_gpu_or_do_not_fit():
    import paper_2509_23472_amd as L
    x = torch.zeros(4, 8)
    for call in (lambda: L.loract_linear(x, x), lambda: L.loract_linear_backward(x), lambda: L.loract_dropout(x, 0.1, 0),
                 lambda: L.loract_qknorm_rope_forward(x.view(4, 1, 8), None, None, None, None)):
        with pytest.raises(ValueError):
            call()
