"""Outputs that share memory with what a call reads are refused on the host, before anything is enqueued; csrc/overlap.h against a
count of bytes."""
import ctypes
import os
import subprocess

import pytest

from paper_2509_23472_amd import _lib
from paper_2509_23472_amd._lib import LoractLinearParams, LoractQkParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = -1
MB = 1 << 20


def _at(mb, off=0):
    """Addresses that nothing lives at, a megabyte apart: enough for every operand here."""
    return ctypes.c_void_p(mb * MB + off)


PROGRAM = r"""
#include "%s/paper_2509_23472_amd/csrc/overlap.h"
#include <cstdio>
#include <random>
#include <vector>
static std::vector<int> bytes(const Extent& e) {
  std::vector<int> hit(2048, 0);
  for (int64_t o = 0; o < e.outer; ++o)
    for (int64_t i = 0; i < e.inner; ++i)
      for (int64_t w = 0; w < e.width; ++w) hit[(size_t)((uintptr_t)e.at + o * e.outer_step + i * e.inner_step + w)]++;
  return hit;
}
int main() {
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() %% (unsigned)(hi - lo + 1)); };
  long met = 0, apart_in_range = 0, distinct = 0, wrong = 0;
  for (int trial = 0; trial < 100000; ++trial) {
    const int how = pick(0, 5);                     // steps in common, as of slices of one matrix
    int o[2] = {pick(-40, 120), pick(-40, 120)}, n[2] = {pick(-20, 40), pick(-20, 40)};
    if (how < 3) o[1] = o[0];
    if (how < 2) n[1] = n[0];
    if (how == 4) { o[1] = n[0]; n[1] = o[0]; }
    Extent e[2];
    for (int s = 0; s < 2; ++s) e[s] = Extent((const void*)(uintptr_t)(600 + pick(0, 300)), pick(1, 5), o[s], pick(1, 4), n[s], pick(1, 12));
    const std::vector<int> a = bytes(e[0]), b = bytes(e[1]);
    bool meet = false, own = true;
    int lo[2] = {2048, 2048}, hi[2] = {0, 0};
    for (int i = 0; i < 2048; ++i) {
      meet |= a[i] && b[i];
      own &= a[i] < 2;
      if (a[i]) { lo[0] = i < lo[0] ? i : lo[0]; hi[0] = i; }
      if (b[i]) { lo[1] = i < lo[1] ? i : lo[1]; hi[1] = i; }
    }
    met += meet;
    apart_in_range += !meet && lo[0] <= hi[1] && lo[1] <= hi[0];
    wrong += extents_meet(e[0], e[1]) != meet;
    if (extent_distinct(e[0])) { ++distinct; wrong += !own; }
    wrong += extents_same(e[0], e[1]) && a != b;
  }
  std::printf("%%ld %%ld %%ld %%ld\n", wrong, met, apart_in_range, distinct);
  const int64_t far = (int64_t)1 << 62;              // steps whose products pass 64 bits
  const Extent huge((const void*)4096, 1 << 30, far, 1, 0, 64), small((const void*)8192, 1 << 30, 64, 1, 0, 64);
  return extents_meet(huge, small) || extents_meet(huge, Extent()) ? 1 : 0;
}
"""


def test_extents_against_a_count_of_bytes(tmp_path):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(PROGRAM % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    wrong, met, apart, distinct = (int(v) for v in out)
    assert wrong == 0 and met > 10000 and apart > 10000 and distinct > 5000


def _linear(x=1, w=2, bias=3, t=4, b=5, r=6, y=7, z=8, ws=9, **kw):
    base = dict(m=64, n_in=96, n_out=96, ldx=96, ldw=96, ldr=96, ldy=96, ldz=96, ldp=96, dtype=1, out_dtype=1, w_layout=0, act=0, r_lora=4,
                lora_scale=1.0, p_drop=0.0, seed=0)
    base.update(kw)
    at = lambda v: v if isinstance(v, ctypes.c_void_p) else _at(v)
    return _lib.load().loract_linear(at(x), at(w), at(bias), at(t), at(b), at(r), ctypes.byref(LoractLinearParams(**base)), at(y), at(z), at(ws),
                                     1 << 40, None)


@pytest.mark.parametrize("kw", [
    dict(y=1), dict(y=2), dict(y=3), dict(y=4), dict(y=5), dict(y=8), dict(z=1), dict(z=2), dict(z=6), dict(z=4), dict(z=5), dict(z=3),
    dict(y=_at(1, 63 * 192)),                                            # the last row of X
    dict(y=_at(6, 192)),                                                 # the residual, a row further
    dict(y=6, ldr=100), dict(y=6, out_dtype=0),                          # the residual with other rows, or of another type
    dict(x=_at(7, 50), ldx=192, ldy=192), dict(x=_at(7, 191), ldx=192, ldy=192),     # slices of one matrix that share columns
    dict(w_layout=1, y=_at(2, 95 * 192 + 190))])
def test_linear_refuses_outputs_in_its_inputs(kw):
    assert _linear(**kw) == INVALID


def test_linear_refuses_outputs_in_its_workspace():
    split = dict(m=64, n_in=8192, ldx=8192, ldw=8192)                    # K is split: a workspace is used
    assert _linear(y=60, ws=60, z=40, w=20, **split) == INVALID and _linear(z=60, ws=60, y=40, w=20, **split) == INVALID


def _backward(dy=1, z=2, t=3, dp=4, db=5, d_b=6, ws=7, **kw):
    base = dict(m=64, n_in=1, n_out=96, ldy=96, ldz=96, ldp=96, dtype=1, out_dtype=1, w_layout=0, act=2, r_lora=4, lora_scale=1.0, p_drop=0.0, seed=0)
    base.update(kw)
    at = lambda v: v if isinstance(v, ctypes.c_void_p) else _at(v)
    return _lib.load().loract_linear_backward(at(dy), at(z), at(t), ctypes.byref(LoractLinearParams(**base)), at(dp), at(db), at(d_b), at(ws), 1 << 40, None)


@pytest.mark.parametrize("kw", [dict(dp=_at(1, 2)), dict(dp=1, ldp=97), dict(dp=_at(2, 192)), dict(dp=3), dict(dp=7), dict(db=1), dict(db=2), dict(db=4),
                                dict(db=6), dict(db=7), dict(d_b=1), dict(d_b=2), dict(d_b=3), dict(d_b=4), dict(d_b=7)])
def test_linear_backward_refuses_outputs_in_its_inputs(kw):
    assert _backward(**kw) == INVALID


def test_dropout_refuses_outputs_in_its_inputs():
    f = lambda x, r, y, ldy=8: _lib.load().loract_dropout(x, 8, r, 8, 4, 8, 0, 0.1, 0, y, ldy, None)
    assert f(_at(1), _at(2), _at(1, 4)) == INVALID and f(_at(1), _at(2), _at(2, 32)) == INVALID and f(_at(1), _at(2), _at(1), 9) == INVALID


D = 64


def _qk(token, head, out_token, out_head, **kw):
    base = dict(m=4, heads_q=2, heads_k=2, d=D, rot=D, interleaved=0, dtype=1, n_pos=8, eps=1e-6, q_token=token, q_head=head, k_token=token, k_head=head,
                qo_token=out_token, qo_head=out_head, ko_token=out_token, ko_head=out_head, dq_token=token, dq_head=head, dk_token=token, dk_head=head)
    base.update(kw)
    return LoractQkParams(**base)


def _qk_forward(p, q=1, k=2, qo=3, ko=4, table=5, gamma=6, pos=7):
    at = lambda v: v if isinstance(v, ctypes.c_void_p) else _at(v)
    return _lib.load().loract_qknorm_rope_forward(at(q), at(k), ctypes.byref(p), at(gamma), at(gamma), at(table), at(pos), at(qo), at(ko), None)


def _qk_backward(p, q=1, k=2, dqo=3, dko=4, dq=5, dk=6, gq=7, gk=8, ws=9, table=10):
    at = lambda v: v if isinstance(v, ctypes.c_void_p) else _at(v)
    return _lib.load().loract_qknorm_rope_backward(at(q), at(k), ctypes.byref(p), None, None, at(table), None, at(dqo), at(dko), at(dq), at(dk), at(gq), at(gk),
                                                   at(ws), 1 << 40, None)


def test_qknorm_rope_refuses_outputs_in_its_inputs():
    plain = _qk(2 * D, D, 2 * D, D)
    for kw in (dict(qo=2), dict(ko=1), dict(qo=4), dict(qo=5), dict(ko=6), dict(qo=7), dict(qo=_at(1, 2 * D)), dict(ko=_at(2, 2))):
        assert _qk_forward(plain, **kw) == INVALID, kw
    packed = _qk(6 * D, D, 6 * D, D)                                     # q, k and v of a token side by side
    assert _qk_forward(packed, q=1, k=_at(1, 4 * D), qo=_at(1, 4 * D), ko=1) == INVALID
    assert _qk_forward(packed, qo=3, ko=_at(3, 2 * D)) == INVALID        # the second head of q is the first of k
    for kw in (dict(dq=2), dict(dk=1), dict(dq=4), dict(dk=3), dict(dq=6), dict(dq=_at(3, 2)), dict(gq=1), dict(gk=6), dict(gq=8), dict(dq=9), dict(gq=9),
               dict(dq=10), dict(gk=10)):
        assert _qk_backward(plain, **kw) == INVALID, kw


@pytest.mark.parametrize("strides", [(D, D), (2 * D, D - 1), (D, 2 * D), (2 * D - 1, D), (0, D), (2 * D, 0)])
def test_qknorm_rope_refuses_outputs_whose_heads_meet(strides):
    assert _qk_forward(_qk(2 * D, D, *strides)) == INVALID
    assert _qk_backward(_qk(2 * D, D, *strides)) == INVALID
