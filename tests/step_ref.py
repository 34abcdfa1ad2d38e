"""Plain implementations in 64 bits of what a step ends with and of the adapters of many requests."""
from __future__ import annotations

import numpy as np
import torch

from sublayer_ref import splitmix64

BLOCK = 256


def padded(n):
    return -(-n // BLOCK) * BLOCK


def places(sizes):
    """Where the elements of the tensors stand in the state."""
    at, out = 0, []
    for n in sizes:
        out.append(np.arange(n) + at)
        at += padded(n)
    return np.concatenate(out) if out else np.zeros(0, dtype=np.int64)


def halves(seed, step, count):
    """32 random bits for every element of the state."""
    start = splitmix64(seed, step)
    words = [splitmix64(start, i + 1) for i in range(count // 2)]
    return np.array(words, dtype=np.uint64).view(np.uint32).astype(np.int64)


def unit_byte(top):
    """The byte of the exponent that takes `top` to 320/3 or more and below 640/3."""
    if not top > 0:
        return 1
    power = int(np.floor(np.log2(top * 3 / 320)))
    while top / 2.0 ** power >= 640 / 3:
        power += 1
    while top / 2.0 ** power < 320 / 3:
        power -= 1
    return max(power, -126) + 127


def rounded(x, bits, count, digits, lowest):
    """|x| to `digits` digits after the point (2^(lowest - digits) apart below 2^lowest), up where the place between two
    neighbours plus (bits + 1/2) / 2^count is at least 1."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    low = np.maximum(np.frexp(np.maximum(x, 2.0 ** lowest))[1] - 1, lowest).astype(np.float64)
    gap = np.exp2(low - digits)
    return np.floor(x / gap + (bits + 0.5) / 2 ** count) * gap


def adamw(p, g, m, v, step, lr, betas, eps, decay):
    """(p, m, v, size of what p's last sum is made of) in 64 bits."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    move = lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps)
    return p * (1 - lr * decay) - move, m, v, np.abs(p) + np.abs(move)


def e4m3(codes):
    """The numbers that bytes stand for."""
    return torch.from_numpy(np.asarray(codes, dtype=np.uint8)).view(torch.float8_e4m3fn).double().numpy()


# ---------------------------------------------------------------------------------------------
# Log probabilities (torch, 64 bits, on the device of the logits).

def logprobs(x, targets, temperature=1.0):
    """(log p of all, entropy, logp of the targets); rows of nothing but -inf: -inf, 0, -inf."""
    z = x.double() / temperature
    top = z.max(1, keepdim=True)[0]
    none = top[:, 0] == -float("inf")
    low = z - torch.where(none[:, None], torch.zeros_like(top), top)
    log_p = low - torch.where(none[:, None], torch.zeros_like(top), low.exp().sum(1, keepdim=True).log())
    p = torch.where(none[:, None], torch.zeros_like(low), log_p.exp())
    entropy = -torch.where(p > 0, p * log_p, torch.zeros_like(p)).sum(1)
    if targets is None:
        return log_p, p, entropy, None
    at = targets.long().clamp(0, x.shape[1] - 1)
    logp = log_p.gather(1, at[:, None])[:, 0]
    logp = torch.where(targets < 0, torch.zeros_like(logp), logp)
    return log_p, p, entropy, torch.where(targets >= x.shape[1], torch.full_like(logp, float("nan")), logp)


def logprobs_grad(x, targets, d_logp, d_entropy, temperature=1.0):
    log_p, p, entropy, _ = logprobs(x, targets, temperature)
    grad, size = torch.zeros_like(p), torch.zeros_like(p)
    none = x.max(1)[0] == -float("inf")
    if d_logp is not None:
        g = torch.where((targets < 0) | none, torch.zeros_like(d_logp), d_logp).double()[:, None]
        hit = (torch.arange(x.shape[1], device=x.device) == targets[:, None]).double()
        grad += g * (hit - p)
        size += g.abs() * (hit + p)
    if d_entropy is not None:
        d = d_entropy.double()[:, None]
        grad -= torch.where(p > 0, d * p * (log_p + entropy[:, None]), torch.zeros_like(p))
        size += torch.where(p > 0, d.abs() * p * (log_p.abs() + entropy[:, None]), torch.zeros_like(p))
    if targets is not None:
        grad[targets >= x.shape[1]] = float("nan")
    return grad / temperature, size / temperature


def top(x, k):
    """Indices of the k largest, ties in the order of their indices; what is no number counts as -inf."""
    v = torch.where(x != x, torch.full_like(x, -float("inf")), x).float().cpu()
    return torch.sort(v, dim=1, descending=True, stable=True)[1][:, :k].int().to(x.device)


# ---------------------------------------------------------------------------------------------
# Adapters of many requests.

def lora_requests(x, a, b, ids, scales, residual):
    """(Y, bound without the output's rounding) in 64 bits: sums of K products stray by 6 sqrt(K) 2^-24 of their magnitudes, X A enters the second
    product with 16 bits (of bf16 operands)."""
    y = torch.zeros(x.shape[0], b.shape[2], dtype=torch.float64, device=x.device) if residual is None else residual.double().clone()
    off = y.abs() * 2.0 ** -24
    u, k, r = 2.0 ** -24, x.shape[1], a.shape[2]
    held = 2.0 ** -16 if x.dtype is torch.bfloat16 else u
    for i in range(a.shape[0]):
        rows = (ids == i).nonzero()[:, 0]
        s = 1.0 if scales is None else float(scales[i])
        xi, ai, bi = x[rows].double(), a[i].double(), b[i].double()
        t = xi @ ai
        y[rows] += s * (t @ bi)
        off_t = 6 * k ** 0.5 * u * (xi.abs() @ ai.abs()) + (held + 2 * u) * t.abs()
        off[rows] += abs(s) * (off_t @ bi.abs() + (6 * (2 * r) ** 0.5 + 4) * u * (t.abs() @ bi.abs()))
    y[ids >= a.shape[0]] = float("nan")
    return y, off
