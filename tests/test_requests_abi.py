"""What loract_lora_requests refuses is refused on the host, before anything is enqueued."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2509_23472_amd as L
from paper_2509_23472_amd import _lib, api
from paper_2509_23472_amd._lib import LoractRequestsParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SMALL, UNSUPPORTED = -1, -2, -3
X, A, B, IDS, SC, R, Y, WS = (i << 40 for i in range(1, 9))


def test_parameter_structure(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    body = 'printf("%zu\\n", sizeof(loract_requests_params));' + "".join('printf("%%zu\\n", offsetof(loract_requests_params, %s));' % f[0]
                                                                         for f in LoractRequestsParams._fields_)
    src.write_text('#include "%s/include/loract.h"\n#include <stdio.h>\nint main(void) { %s return 0; }\n' % (ROOT, body))
    subprocess.run(["gcc", str(src), "-o", str(exe)], check=True)
    want = [int(v) for v in subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    assert [ctypes.sizeof(LoractRequestsParams)] + [getattr(LoractRequestsParams, f[0]).offset for f in LoractRequestsParams._fields_] == want
    values = list(range(1, 12))
    assert api._REQUESTS_PARAMS.pack(*values) == bytes(LoractRequestsParams(*values))


def _p(**kw):
    base = dict(m=100, n_in=512, n_out=256, adapters=4, ldx=512, ldr=256, ldy=256, dtype=1, out_dtype=1, r=16, reserved=0)
    base.update(kw)
    return LoractRequestsParams(**base)


def _call(p, x=X, a=A, b=B, ids=IDS, sc=SC, r=R, y=Y, ws=WS, size=1 << 50):
    return _lib.load().loract_lora_requests(x, a, b, ids, sc, r, ctypes.byref(p), y, ws, size, None)


def _query(p):
    out = ctypes.c_size_t(0)
    code = _lib.load().loract_lora_requests_workspace_bytes(ctypes.byref(p), ctypes.byref(out))
    return code, out.value


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(m=0)), (INVALID, dict(n_in=0)), (INVALID, dict(n_out=-1)), (INVALID, dict(adapters=0)), (INVALID, dict(r=0)), (INVALID, dict(reserved=1)),
    (INVALID, dict(ldx=511)), (INVALID, dict(ldy=255)), (INVALID, dict(dtype=2)), (INVALID, dict(out_dtype=-1)), (UNSUPPORTED, dict(r=65)),
    (UNSUPPORTED, dict(dtype=0)), (UNSUPPORTED, dict(m=(1 << 27) + 1)), (UNSUPPORTED, dict(n_out=(1 << 24) + 1, ldy=1 << 25, ldr=1 << 25)),
    (UNSUPPORTED, dict(n_in=(1 << 30) + 1, ldx=1 << 31)), (UNSUPPORTED, dict(adapters=(1 << 30) + 1)),
    (UNSUPPORTED, dict(m=1 << 27, n_out=1 << 24, ldy=1 << 24, ldr=1 << 24))])
def test_refused_parameters(code, kw):
    assert _call(_p(**kw)) == code and _query(_p(**kw))[0] == code


def test_refused_operands():
    p = _p()
    for kw in (dict(x=None), dict(a=None), dict(b=None), dict(ids=None), dict(y=None), dict(x=X + 1), dict(a=A + 1), dict(b=B + 1), dict(ids=IDS + 2), dict(sc=SC + 1),
               dict(r=R + 1), dict(y=Y + 1), dict(ws=WS + 8)):
        assert _call(p, **kw) == INVALID, kw
    assert _call(_p(ldr=255)) == INVALID
    code, need = _query(p)
    assert code == 0 and need >= 100 * 16 * 4
    assert _call(p, size=100) == SMALL and _call(p, ws=None) == SMALL
    assert _lib.load().loract_lora_requests_workspace_bytes(ctypes.byref(p), None) == INVALID
    assert _lib.load().loract_lora_requests_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == INVALID


def test_outputs_that_share_memory():
    p = _p()
    for kw in (dict(y=X + 64), dict(y=A), dict(y=B + 4 * 16 * 256 * 2 - 2), dict(y=IDS), dict(y=SC + 12), dict(y=R + 2), dict(y=WS), dict(ws=X), dict(ws=A + 16), dict(ws=R),
               dict(ws=IDS + 16)):
        assert _call(p, **kw) == INVALID, kw
    assert _call(_p(ldy=264), y=R) == INVALID


def test_every_size_that_is_taken_fits_a_launch():
    """The grids of both launches: fewer than 2^32 threads, fewer than 65536 rows of workgroups."""
    for m, n_out in ((1, 1 << 24), (1 << 27, 128), (1 << 20, 1 << 16), (3, 5)):
        assert _query(_p(m=m, n_out=n_out, ldy=n_out, ldr=n_out))[0] == 0


def test_the_binding_refuses(monkeypatch):
    args = dict(x=torch.zeros(4, 8), a=torch.zeros(3, 8, 2), b=torch.zeros(3, 2, 6), ids=torch.zeros(4, dtype=torch.int32), scales=torch.zeros(3))
    with pytest.raises(ValueError):
        L.loract_lora_requests(**args)                             # not on a GPU
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0
    monkeypatch.setattr(api._lib, "load", lambda: Library())
    L.loract_lora_requests(**args)
    assert reached == ["loract_lora_requests"]
    for kw in (dict(x=torch.zeros(8)), dict(x=torch.zeros(4, 9)), dict(x=torch.zeros(4, 8).bfloat16()), dict(a=torch.zeros(8, 2)), dict(a=torch.zeros(2, 8, 2)),
               dict(a=torch.zeros(3, 2, 8).transpose(1, 2)), dict(b=torch.zeros(3, 3, 6)), dict(b=torch.zeros(3, 2, 12)[:, :, ::2]), dict(ids=torch.zeros(4)),
               dict(ids=torch.zeros(5, dtype=torch.int32)), dict(ids=torch.zeros(8, dtype=torch.int32)[::2]), dict(scales=torch.zeros(4)),
               dict(scales=torch.zeros(3).double()), dict(residual=torch.zeros(4, 7)), dict(residual=torch.zeros(4, 6).bfloat16()), dict(out=torch.zeros(5, 6)),
               dict(out_dtype=torch.float64), dict(x=torch.zeros(4, 8).double(), a=torch.zeros(3, 8, 2).double(), b=torch.zeros(3, 2, 6).double())):
        with pytest.raises((ValueError, TypeError)):
            L.loract_lora_requests(**dict(args, **kw))
    assert len(reached) == 1
