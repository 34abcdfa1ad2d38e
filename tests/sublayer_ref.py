"""Plain implementations of the sub-layer's operators in 64 bits on the CPU, and the bounds that their float32 counterparts keep.

Every bound is the effect of rounding: a sum of K float32 products strays by at most 6 sqrt(K) 2^-24 of the sum of their
magnitudes (six deviations of a random walk whose steps are roundings of partial sums), functions of one number by a few units of
float32, and what is stored by the unit roundoff of its type (2^-8 for bf16).
"""
from __future__ import annotations

import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # unit roundoff: half a step of 8 and of 24 significant bits
GOLDEN, C1, C2, ALL = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 2 ** 64 - 1


def splitmix64(seed, number):
    """Output `number` (from 1) of the generator started at `seed`."""
    z = (seed + number * GOLDEN) & ALL
    z = ((z ^ (z >> 30)) * C1) & ALL
    z = ((z ^ (z >> 27)) * C2) & ALL
    return z ^ (z >> 31)


def drop_factors(m, n, p, seed, rows=None):
    """What dropout multiplies every element with (the rows `rows` of an m x n matrix, or all of them)."""
    rows = np.arange(m) if rows is None else np.asarray(rows)
    if p == 0.0:
        return torch.ones(len(rows), n, dtype=torch.float64)
    thr = min(65535, math.floor(65536 * p + 0.5))
    per = -(-n // 4)
    number = rows.astype(np.uint64)[:, None] * np.uint64(per) + np.arange(1, per + 1, dtype=np.uint64)[None, :]
    z = np.uint64(seed & ALL) + number * np.uint64(GOLDEN)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(C1)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(C2)
    z ^= z >> np.uint64(31)
    assert int(z[-1, -1]) == splitmix64(seed, int(number[-1, -1]))
    fields = (z[..., None] >> np.array([0, 16, 32, 48], dtype=np.uint64)) & np.uint64(0xFFFF)
    keep = torch.from_numpy((fields.reshape(len(rows), per * 4)[:, :n] >= thr).astype(np.float64))
    return keep * (65536.0 / (65536 - thr))


def act(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def linear(x, w_nt, bias=None, t=None, b=None, scale=1.0, act_name="none", factors=None, residual=None):
    """(Y, P, bound of P's float32 error); all in float64, w_nt n_out x n_in."""
    p = x @ w_nt.t()
    mag = x.abs() @ w_nt.abs().t()
    terms = x.shape[1]
    if t is not None:
        p = p + scale * (t @ b)
        mag = mag + abs(scale) * (t.abs() @ b.abs())
        terms += t.shape[1]
    if bias is not None:
        p = p + bias
        mag = mag + bias.abs()
    y = act(act_name, p)
    if factors is not None:
        y = torch.where(factors == 0, torch.zeros_like(y), y * factors)
    if residual is not None:
        y = y + residual
    return y, p, (6 * math.sqrt(terms) + 4) * 2.0 ** -24 * mag


def linear_bound(y, p, p_err, out_dtype, factors=None, residual=None):
    """Bound of Y's error: P's, stretched by the activation (slopes up to 1.13), its own few roundings, the last one."""
    f = 1.0 if factors is None else factors
    err = f * (1.13 * p_err + 8 * 2.0 ** -24 * p.abs()) + 2.0 ** -23 * (y.abs() + (0 if residual is None else residual.abs()))
    return err + 1.01 * U[out_dtype] * (y.abs() + err) + 1e-37


def rotate(y, table_rows, interleaved, back=False):
    """Rot (or its transpose) of tokens x heads x d by the table's rows (tokens x 2 x rot / 2)."""
    half = table_rows.shape[2]
    c, s = table_rows[:, 0][:, None], table_rows[:, 1][:, None]
    if back:
        s = -s
    out = y.clone()
    ia = torch.arange(half) * 2 if interleaved else torch.arange(half)
    ib = ia + 1 if interleaved else ia + half
    out[..., ia] = y[..., ia] * c - y[..., ib] * s
    out[..., ib] = y[..., ia] * s + y[..., ib] * c
    return out


def qknorm(x, gamma, table, positions, eps, interleaved, dy=None):
    """Forward (y, bound) or, with dy, backward (dx, bound, dgamma, bound); bounds without the last rounding."""
    m, heads, d = x.shape
    gamma = torch.ones(d, dtype=torch.float64) if gamma is None else gamma
    pos = torch.arange(m) if positions is None else positions.long()
    live = (pos >= 0)[:, None, None]
    rows = table[pos.clamp(min=0)] if table is not None else torch.zeros(m, 2, 0, dtype=torch.float64)
    rms = (x.square().mean(-1, keepdim=True) + eps).sqrt()
    hat = x / rms
    few = (6 * math.sqrt(d) + 16) * 2.0 ** -24
    if dy is None:
        y = rotate(hat * gamma, rows, interleaved)
        mag = rotate_mag(hat * gamma, rows, interleaved)
        return torch.where(live, y, torch.zeros_like(y)), few * mag
    t = torch.where(live, rotate(dy, rows, interleaved, back=True), torch.zeros_like(dy))
    mag_t = torch.where(live, rotate_mag(dy, rows, interleaved), torch.zeros_like(dy))
    u = t * gamma
    dx = (u - hat * (u * hat).mean(-1, keepdim=True)) / rms
    dx_mag = (mag_t * gamma.abs() + hat.abs() * (mag_t * gamma.abs() * hat.abs()).mean(-1, keepdim=True)) / rms
    dg = (t * hat).sum((0, 1))
    dg_mag = (mag_t * hat.abs()).sum((0, 1))
    return dx, 2 * few * dx_mag, dg, (few + 6 * math.sqrt(m * heads) * 2.0 ** -24) * dg_mag


def rotate_mag(y, table_rows, interleaved):
    return rotate(y.abs(), torch.stack([table_rows[:, 0].abs(), -table_rows[:, 1].abs()], 1), interleaved).maximum(
        rotate(y.abs(), table_rows.abs(), interleaved))


def check(got, want, bound, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    bad = ~(off <= bound)
    bad &= ~((got == want) | (got.isnan() & want.isnan()))       # (equal infinities; NaN where it belongs)
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d off, first at %s: %r, should be %r within %.3g" % (
            what, int(bad.sum()), bad.numel(), at, float(got[at]), float(want[at]), float(torch.as_tensor(bound).expand_as(want)[at])))
