"""What loract_adamw refuses is refused on the host, before anything is enqueued."""
import ctypes
import os
import struct
import subprocess

import pytest
import torch

import paper_2509_23472_amd as L
from paper_2509_23472_amd import _lib, api
from paper_2509_23472_amd._lib import LoractAdamwParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = -1, -3
P, G, M, V, E, C = (i << 40 for i in range(1, 7))


def test_parameter_structure(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    body = 'printf("%zu\\n", sizeof(loract_adamw_params));' + "".join('printf("%%zu\\n", offsetof(loract_adamw_params, %s));' % f[0]
                                                                      for f in LoractAdamwParams._fields_)
    src.write_text('#include "%s/include/loract.h"\n#include <stdio.h>\nint main(void) { %s return 0; }\n' % (ROOT, body))
    subprocess.run(["gcc", str(src), "-o", str(exe)], check=True)
    want = [int(v) for v in subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    assert [ctypes.sizeof(LoractAdamwParams)] + [getattr(LoractAdamwParams, f[0]).offset for f in LoractAdamwParams._fields_] == want
    values = [1.0, 2.0, 3.0, 4.0, 5.0, 6, 2 ** 64 - 7, 0, 1, 8]
    assert api._ADAMW_PARAMS.pack(*values)[:68] == bytes(LoractAdamwParams(*values))[:68]


def _call(p=(P,), g=(G,), n=(1000,), copy=None, m=M, v=V, e=E, lr_dev=None, step_dev=None, scale=None, count=None, **kw):
    base = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, seed=0, p_dtype=0, g_dtype=0, state_bits=8)
    base.update(kw)
    pack = lambda v: None if v is None else struct.pack("%dQ" % len(v), *v)
    sizes = None if n is None else struct.pack("%dq" % len(n), *n)
    return _lib.load().loract_adamw(pack(p), pack(g), pack(copy), sizes, len(n) if count is None else count, ctypes.byref(LoractAdamwParams(**base)),
                                    m, v, e, lr_dev, step_dev, scale, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(beta1=1.0)), (INVALID, dict(beta1=-0.1)), (INVALID, dict(beta2=1.0)), (INVALID, dict(beta2=NAN)), (INVALID, dict(eps=-1.0)),
    (INVALID, dict(eps=INF)), (INVALID, dict(weight_decay=-0.1)), (INVALID, dict(weight_decay=NAN)), (INVALID, dict(step=0)), (INVALID, dict(p_dtype=2)),
    (INVALID, dict(g_dtype=-1)), (INVALID, dict(state_bits=16)), (INVALID, dict(n=(-1,))), (INVALID, dict(p=(0,))), (INVALID, dict(g=(0,))),
    (INVALID, dict(m=None)), (INVALID, dict(v=None)), (INVALID, dict(e=None)), (INVALID, dict(m=M + 8)), (INVALID, dict(v=V + 4)), (INVALID, dict(e=E + 1)),
    (INVALID, dict(p=(P + 2,))), (INVALID, dict(g=(G + 1,))), (INVALID, dict(copy=(C + 1,))), (INVALID, dict(copy=(C,), p_dtype=1)),
    (INVALID, dict(scale=G + 2)), (INVALID, dict(p=None)), (INVALID, dict(g=None)), (INVALID, dict(count=-1)), (UNSUPPORTED, dict(n=((1 << 33) + 1,))),
    (UNSUPPORTED, dict(count=(1 << 24) + 1))])
def test_refusals(code, kw):
    assert _call(**kw) == code


def test_refused_rates():
    for lr in (-1.0, NAN, INF):
        base = LoractAdamwParams(lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, seed=0, p_dtype=0, g_dtype=0, state_bits=32)
        one = lambda v: struct.pack("Q", v)
        assert _lib.load().loract_adamw(one(P), one(G), None, one(5), 1, ctypes.byref(base), M, V, None, None, None, None, None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(p=(P, P), g=(G, G + 4000), n=(1000, 1000)),                                    # a tensor that is in the list twice
    dict(p=(P, P + 3996), g=(G, G + 4000), n=(1000, 1000)), dict(p=(P + 3996, P), g=(G, G + 4000), n=(1000, 1000)),
    dict(g=(P + 3996,)), dict(g=(P - 3996,)), dict(g=(M,)), dict(g=(V + 1020,)), dict(g=(E + 4,)), dict(m=P), dict(m=V), dict(m=V - 1008), dict(e=M + 1022),
    dict(copy=(P,)), dict(copy=(G,)), dict(copy=(M - 1998,)), dict(scale=P + 8), dict(lr_dev=M + 4), dict(step_dev=E), dict(scale=C + 4, copy=(C,))])
def test_outputs_that_share_memory(kw):
    assert _call(**kw) == INVALID


def test_nothing_to_do():
    assert _call(n=(), p=(), g=()) == 0 and _call(n=(0, 0), p=(0, 0), g=(0, 0), m=None, v=None) == 0


class _Tensors:
    def __init__(self, **kw):
        self.p = [torch.zeros(4), torch.zeros(300)]
        self.g = [torch.zeros(4), torch.zeros(300)]
        self.state = L.AdamwState([4, 300], 8, torch.device("cpu"))
        self.kw = dict(step=1, lr=1e-3)


def test_the_binding_wants_tensors_on_the_gpu():
    t = _Tensors()
    with pytest.raises(ValueError):
        L.loract_adamw(t.p, t.g, t.state, **t.kw)
    with pytest.raises(ValueError):
        L.loract_adamw_state(t.p)
    with pytest.raises(ValueError):
        L.loract_adamw_state([])
    with pytest.raises(ValueError):
        L.loract_adamw([], [], t.state, **t.kw)
    with pytest.raises(ValueError):
        L.AdamwState([4], 16, torch.device("cpu"))


@pytest.mark.parametrize("bad", [lambda t: t.p.pop(), lambda t: t.g.pop(), lambda t: t.p.__setitem__(1, torch.zeros(299)), lambda t: t.g.__setitem__(0, torch.zeros(5)),
                                 lambda t: t.p.__setitem__(1, torch.zeros(300, dtype=torch.bfloat16)), lambda t: t.g.__setitem__(1, torch.zeros(600)[::2]),
                                 lambda t: t.g.__setitem__(0, torch.zeros(4, dtype=torch.float64)), lambda t: setattr(t.state, "m", torch.zeros(768)),
                                 lambda t: setattr(t.state, "exps", t.state.exps[:1]), lambda t: t.kw.update(lr=torch.zeros(2)),
                                 lambda t: t.kw.update(step=torch.zeros(1)), lambda t: t.kw.update(grad_scale=1.0), lambda t: t.kw.update(copies=[t.p[0]]),
                                 lambda t: t.kw.update(copies=[torch.zeros(4, dtype=torch.bfloat16)])])
def test_the_binding_refuses(bad, monkeypatch):
    """As on a GPU: every tensor says that it lives on GPU 0."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    reached = []

    class Library:
        def loract_adamw(self, *args):
            reached.append(args)
            return 0
    monkeypatch.setattr(api._lib, "load", lambda: Library())
    t = _Tensors()
    L.loract_adamw(t.p, t.g, t.state, **t.kw)
    assert len(reached) == 1
    bad(t)
    with pytest.raises((ValueError, TypeError)):
        L.loract_adamw(t.p, t.g, t.state, **t.kw)
    assert len(reached) == 1


SPANS = r"""
#include "%s/paper_2509_23472_amd/csrc/spans.h"
#include <cstdio>
#include <random>
#include <vector>
// Every place of a gradient among the written intervals, in ascending, descending and mixed order, against all pairs.
int main() {
  std::mt19937 rng(5);
  auto pick = [&](int n) { return (int)(rng() %% (unsigned)n); };
  int met = 0, apart = 0;
  for (int round = 0; round < 3000; ++round) {
    const int n = 1 + pick(40), order = pick(3);
    std::vector<int> at(n);
    for (int i = 0; i < n; ++i) at[i] = i;
    if (order == 1) std::reverse(at.begin(), at.end());
    if (order == 2) std::shuffle(at.begin(), at.end(), rng);
    std::vector<void*> p(n), copy(n);
    std::vector<const void*> g(n);
    std::vector<int64_t> size(n);
    const uintptr_t p0 = 1 << 20, c0 = 1 << 24;
    for (int i = 0; i < n; ++i) {
      size[i] = pick(8) ? 1 + pick(30) : 0;
      p[i] = (void*)(p0 + at[i] * 400);
      copy[i] = pick(3) ? (void*)(c0 + at[i] * 400) : nullptr;
      g[i] = (const void*)((pick(2) ? p0 : c0) + at[i] * 400 + 200);
    }
    if (pick(2)) g[pick(n)] = (const void*)((pick(2) ? p0 : c0) + pick(n) * 400 + 4 * pick(100));
    if (pick(8) == 0) p[pick(n)] = p[pick(n)];               // (a tensor that is in the list twice)
    Span state[3] = {{1 << 28, (1 << 28) + 1000}, {1 << 29, (1 << 29) + 1000}, {7, 7}}, scalars[3] = {{0, 0}, {0, 0}, {0, 0}};
    if (pick(20) == 0) scalars[1] = {(uintptr_t)(1 << 29) + 996, (uintptr_t)(1 << 29) + 1004};
    if (pick(20) == 0) state[0] = {p0 + 100, p0 + 104};
    std::vector<Span> out, in;
    for (const Span& s : state) if (s.hi > s.lo) out.push_back(s);
    for (const Span& s : scalars) if (s.hi > s.lo) in.push_back(s);
    for (int i = 0; i < n; ++i) {
      if (!size[i]) continue;
      out.push_back({(uintptr_t)p[i], (uintptr_t)p[i] + size[i] * 4});
      if (copy[i]) out.push_back({(uintptr_t)copy[i], (uintptr_t)copy[i] + size[i] * 2});
      in.push_back({(uintptr_t)g[i], (uintptr_t)g[i] + size[i] * 4});
    }
    bool want = false;
    for (size_t i = 0; i < out.size(); ++i) {
      for (size_t j = 0; j < i; ++j) want |= out[i].lo < out[j].hi && out[j].lo < out[i].hi;
      for (const Span& s : in) want |= out[i].lo < s.hi && s.lo < out[i].hi;
    }
    if (adamw_meets(p.data(), g.data(), copy.data(), size.data(), n, 4, 4, state, scalars) != (int)want) return 1;
    (want ? met : apart)++;
  }
  return met > 300 && apart > 300 ? 0 : 2;
}
"""


def test_shared_memory_among_many_tensors_in_any_order(tmp_path):
    src, exe = tmp_path / "spans.cpp", tmp_path / "spans"
    src.write_text(SPANS % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
