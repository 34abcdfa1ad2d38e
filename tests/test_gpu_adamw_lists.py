"""AdamW over long lists of tensors, in every launch of a step and all pairs of types: each element of the parameters, copies and states against
the formulas in 64 bits, with the bounds of test_gpu_adamw.py."""
import numpy as np
import pytest
import torch

import paper_2509_23472_amd as L
import step_ref as ref
from test_gpu_adamw import HYPER, U32, _flat, _held, _make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _mixed(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def _halves(seed, step, count):
    """32 random bits for every element of the state: ref.halves for many."""
    golden = np.uint64(0x9E3779B97F4A7C15)
    start = np.uint64(ref.splitmix64(seed, step))
    words = _mixed(start + np.arange(1, count // 2 + 1, dtype=np.uint64) * golden)
    out = words.view(np.uint32).astype(np.int64)
    assert (out[:64] == ref.halves(seed, step, 64)).all() and out[-1] == ref.splitmix64(int(start), count // 2) >> 32
    return out


def _bytes(top):
    return np.array([ref.unit_byte(t) for t in top])


def _check_codes(codes, exps, want, off, bits, place, root):
    """codes and exps lie between what the two ends of want +- off give."""
    lo, hi = np.zeros((2, len(codes)))
    lo[place], hi[place] = np.maximum(np.abs(want) - off, 0), np.abs(want) + off
    lo, hi, bits, got = (x.reshape(-1, ref.BLOCK) for x in (lo, hi, bits, np.abs(codes)))
    exps = exps.astype(np.int64)
    assert (_bytes(lo.max(1)) <= exps).all() and (exps <= _bytes(hi.max(1))).all()
    unit = np.exp2(exps - 127.0)[:, None]
    least, most = (ref.rounded(x / unit, bits, 10, 3, -6) for x in (lo, hi))
    if root:
        least, most = (np.where(x > 0, np.maximum(y, 2.0 ** -9), y) for x, y in ((lo, least), (hi, most)))
    assert (got >= least).all() and (got <= most).all(), np.argwhere((got < least) | (got > most))[:4]


def _step_and_check(params, grads, state, sizes, step, seed, copies):
    place = ref.places(sizes)
    m0, v0 = _held(state, place)
    p0, g0 = _flat(params), _flat(grads)
    L.loract_adamw(params, grads, state, step=step, seed=seed, copies=copies, **HYPER)
    torch.cuda.synchronize()
    b1, b2 = HYPER["betas"]
    p, m, v, size = ref.adamw(p0, g0, m0, v0, step, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
    off_m = 4 * U32 * (b1 * np.abs(m0) + (1 - b1) * np.abs(g0))
    off_v = 5 * U32 * v
    den = np.sqrt(v) / np.sqrt(1 - b2 ** step) + HYPER["eps"]
    off_p = 14 * U32 * size + HYPER["lr"] / (1 - b1 ** step) * off_m / den
    words = _halves(seed, step, len(state.m))
    got = _flat(params)
    if params[0].dtype is F32:
        assert (np.abs(got - p) <= off_p).all(), np.argwhere(np.abs(got - p) > off_p)[:4]
    else:
        lo, hi = (ref.rounded(x, (words >> 20)[place], 12, 7, -126) for x in (np.maximum(np.abs(p) - off_p, 0), np.abs(p) + off_p))
        assert (np.abs(got) >= lo).all() and (np.abs(got) <= hi).all(), np.argwhere((np.abs(got) < lo) | (np.abs(got) > hi))[:4]
    if copies is not None:
        assert all(torch.equal(c, q.bfloat16()) for c, q in zip(copies, params))
    if state.bits == 32:
        got_m, got_v = _held(state, place)
        assert (np.abs(got_m - m) <= off_m).all() and (np.abs(got_v - v) <= off_v).all()
        return
    codes_m, codes_r, exps = state.m.double().cpu().numpy(), state.v.double().cpu().numpy(), state.exps.cpu().numpy()
    assert (np.sign(codes_m[place]) * np.sign(m) >= 0).all() and (codes_r >= 0).all()
    _check_codes(codes_m, exps[:, 0], m, off_m, words & 1023, place, False)
    _check_codes(codes_r, exps[:, 1], np.sqrt(v), 5 * U32 * np.sqrt(v), (words >> 10) & 1023, place, True)


# (a launch holds 98 tensors with copies, 122 without)
LISTS = {"333 small": [17 + i % 5 for i in range(333)], "one to a block and none": [256, 0, 257, 1] * 90, "of a chunk and more": [2048, 2049, 4095, 3, 0] * 41,
         "123": [300 + i for i in range(123)], "122": [31] * 122, "98": [2049] * 98, "99": [7] * 99, "long": [70000, 5, 131073, 2048]}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype,copy", [(F32, F32, True), (F32, BF, True), (F32, F32, False), (F32, BF, False), (BF, BF, False), (BF, F32, False)])
@pytest.mark.parametrize("sizes", LISTS.values(), ids=LISTS.keys())
def test_every_launch_of_a_list(sizes, p_dtype, g_dtype, copy, bits):
    params, grads = _make(sizes, p_dtype, g_dtype, len(sizes))
    state = L.loract_adamw_state(params, bits=bits)
    copies = [torch.full((n + 2,), 7.0, dtype=BF, device="cuda") for n in sizes] if copy else None
    inner = [c[1:n + 1] for c, n in zip(copies, sizes)] if copy else None
    for step in (1, 2, 700):
        _step_and_check(params, grads, state, sizes, step, 2 ** 63 + 5, inner)
        for g in grads:
            g.mul_(-0.7)
    assert copies is None or all(c[0] == 7 and c[-1] == 7 for c in copies)
