"""Two pre-norm sub-layers of a LoRA fine-tuning step on the package's operators: Z = F(Norm(X)) + X (Section 3.3).

What is kept from the forward to the backward pass is the compressed activation (U, V) and the RMS vector; everything between them
is computed again from the reconstruction, as under gradient checkpointing, and dropout masks come again from their seed.

  mlp        F = dropout(W2 silu(W1 a + s (a A) B + b1) + b2)
  attention  the part before the attention product: packed queries, keys and values with their LoRA update, norms of queries
             and keys and the rotation by position

Run as a script it trains neither: it times one step of both on random bf16 data and prints what is kept.
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_23472_amd as L


@dataclass
class Lora:
    a: torch.Tensor          # n_in x r
    b: torch.Tensor          # r x n_out
    scale: float


@dataclass
class Mlp:
    gamma: torch.Tensor      # n floats
    w1: torch.Tensor         # ffn x n, frozen
    b1: torch.Tensor
    lora: Lora
    w2: torch.Tensor         # n x ffn, frozen
    b2: torch.Tensor
    p_drop: float
    eps: float = 1e-6


def _mlp_hidden(p: Mlp, a):
    """The LoRA product T = a A, the activated hidden layer and its pre-activation."""
    t = L.loract_linear(a, p.lora.a, w_transposed=True)
    h, z = L.loract_linear(a, p.w1, p.b1, lora_t=t, lora_b=p.lora.b, lora_scale=p.lora.scale, act="silu", save_preact=True)
    return t, h, z


def mlp_forward(p: Mlp, x, rank: int, seed: int):
    a, rms = L.loract_prenorm_forward(x, p.gamma, p.eps)
    kept = L.loract_compress(a, rank, seed=seed) + (rms, seed)
    _, h, _ = _mlp_hidden(p, a)
    return L.loract_linear(h, p.w2, p.b2, p_drop=p.p_drop, seed=seed, residual=x), kept


def mlp_backward(p: Mlp, kept, dy):
    """Gradients of x, the biases and the LoRA factors."""
    u, v, rms, seed = kept
    a = L.loract_reconstruct(u, v)
    t, _, z = _mlp_hidden(p, a)
    d2, db2, _ = L.loract_linear_backward(dy, p_drop=p.p_drop, seed=seed)
    dh = L.loract_linear(d2, p.w2, w_transposed=True)
    d1, db1, d_b = L.loract_linear_backward(dh, z, lora_t=t, lora_scale=p.lora.scale, act="silu", out=dh)
    d_a = L.loract_lora_grad(u, v, d1, p.lora.b, p.lora.scale)
    da = _input_grad(d1, p.w1, p.lora)
    dx = L.loract_prenorm_backward(a, rms, p.gamma, da)
    return dict(x=L.loract_dropout(dx, 0.0, 0, residual=dy, out=dx), b1=db1, b2=db2, a=d_a, b=d_b)


def _input_grad(dp, w, lora: Lora):
    """dP W + s (dP B^T) A^T: the forward's weights, multiplied from the other side."""
    return L.loract_linear(dp, w, w_transposed=True, lora_t=L.loract_linear(dp, lora.b), lora_b=lora.a.t().contiguous(), lora_scale=lora.scale)


@dataclass
class Attention:
    gamma: torch.Tensor
    wqkv: torch.Tensor       # (hq + 2 hk) d x n, frozen
    lora: Lora
    gamma_q: torch.Tensor    # d floats
    gamma_k: torch.Tensor
    table: torch.Tensor      # of loract_rope_table
    hq: int
    hk: int
    eps: float = 1e-6


def _qkv(p: Attention, a):
    t = L.loract_linear(a, p.lora.a, w_transposed=True)
    packed = L.loract_linear(a, p.wqkv, lora_t=t, lora_b=p.lora.b, lora_scale=p.lora.scale)
    return (t,) + _split(p, packed)


def _split(p: Attention, packed):
    """Queries, keys and values as they lie in the packed matrix (tokens x heads x d each)."""
    m, d = packed.shape[0], p.gamma_q.numel()
    edges = (0, p.hq * d, (p.hq + p.hk) * d, (p.hq + 2 * p.hk) * d)
    return tuple(packed[:, edges[i]:edges[i + 1]].view(m, -1, d) for i in range(3))


def attention_inputs(p: Attention, x, positions, rank: int, seed: int):
    """Queries and keys, normed and rotated, and values; and what the backward pass needs."""
    a, rms = L.loract_prenorm_forward(x, p.gamma, p.eps)
    kept = L.loract_compress(a, rank, seed=seed) + (rms, positions)
    _, q, k, v = _qkv(p, a)
    q, k = L.loract_qknorm_rope_forward(q, k, p.gamma_q, p.gamma_k, p.table, positions=positions, out=(q, k))
    return (q, k, v), kept


def attention_inputs_backward(p: Attention, kept, dq, dk, dv):
    """Gradients of x (without the residual's), of the LoRA factors and of the norms' gammas."""
    u, vt, rms, positions = kept
    a = L.loract_reconstruct(u, vt)
    t, q, k, _ = _qkv(p, a)
    packed = torch.empty((a.shape[0], (p.hq + 2 * p.hk) * p.gamma_q.numel()), dtype=a.dtype, device=a.device)
    gq, gk, gv = _split(p, packed)
    gv.copy_(dv)
    _, _, d_gq, d_gk = L.loract_qknorm_rope_backward(q, k, p.gamma_q, p.gamma_k, p.table, dq, dk, positions=positions, out=(gq, gk))
    _, _, d_b = L.loract_linear_backward(packed, lora_t=t, lora_scale=p.lora.scale, bias_grad=False, out=packed)
    d_a = L.loract_lora_grad(u, vt, packed, p.lora.b, p.lora.scale)
    dx = L.loract_prenorm_backward(a, rms, p.gamma, _input_grad(packed, p.wqkv, p.lora))
    return dict(x=dx, a=d_a, b=d_b, gamma_q=d_gq, gamma_k=d_gk)


def make_lora(n_in, n_out, r, dtype, gen):
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return Lora((rand(n_in, r) * n_in ** -0.5).to(dtype), (rand(r, n_out) * r ** -0.5).to(dtype), 0.5)


def make_mlp(n, ffn, r, dtype, gen, p_drop=0.1):
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return Mlp(1 + 0.1 * rand(n), (rand(ffn, n) * n ** -0.5).to(dtype), 0.1 * rand(ffn), make_lora(n, ffn, r, dtype, gen),
               (rand(n, ffn) * ffn ** -0.5).to(dtype), 0.1 * rand(n), p_drop)


def make_attention(n, hq, hk, d, r, n_pos, dtype, gen):
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    out = (hq + 2 * hk) * d
    return Attention(1 + 0.1 * rand(n), (rand(out, n) * n ** -0.5).to(dtype), make_lora(n, out, r, dtype, gen), 1 + 0.1 * rand(d),
                     1 + 0.1 * rand(d), L.loract_rope_table(n_pos, d), hq, hk)


def main():
    m, n, ffn, heads, d, r, rank = 8192, 4096, 11008, 32, 128, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    mlp = make_mlp(n, ffn, r, torch.bfloat16, gen)
    att = make_attention(n, heads, heads, d, r, 2048, torch.bfloat16, gen)
    x, dy = (torch.randn(m, n, generator=gen, device="cuda").bfloat16() for _ in range(2))
    positions = torch.arange(2048, dtype=torch.int32, device="cuda").repeat(m // 2048)

    def step():
        y, kept = mlp_forward(mlp, x, rank, 7)
        (q, k, v), kept_qkv = attention_inputs(att, y, positions, rank, 8)
        mlp_backward(mlp, kept, dy)
        attention_inputs_backward(att, kept_qkv, q, k, v)
        return sum(t.numel() * t.element_size() for t in kept[:3] + kept_qkv[:3])

    for _ in range(3):
        size = step()
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(10):
        step()
    stop.record()
    torch.cuda.synchronize()
    print("%d tokens x %d, MLP of %d and attention inputs of %d heads, LoRA rank %d, activations at rank %d: %.2f ms a step, %.1f MB kept "
          "(%.0f MB as they are)" % (m, n, ffn, heads, r, rank, start.elapsed_time(stop) / 10, size / 1e6, 2 * x.numel() * 2 / 1e6))


if __name__ == "__main__":
    main()
