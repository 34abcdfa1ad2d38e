"""A fine-tuning step from the loss to the update, and the adapters that it trains in serving, on the package's operators.

Several adapters (A, B) of one frozen projection from activations to a vocabulary's logits.  A training step of one of them:

  forward   logits = a W^T + s (a A) B; the activation is kept as its factors (U, V)
  loss      mean of -log p(target) over the tokens that have one, with the logits' gradient in the same call, in their place
  backward  the gradients of A (from the factors) and of B
  update    AdamW on float32 A and B, whose bf16 copies are the adapters' places in the pools that serving reads

Serving: one batch of requests of any adapters; the projection is shared, every token gets its own adapter's update, then its
next token's alternatives.

Run as a script it times a step and a batch on random data.
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass
from typing import List

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_23472_amd as L


@dataclass
class Adapter:
    a: torch.Tensor          # n x r floats
    b: torch.Tensor          # r x vocabulary floats
    state: L.AdamwState
    steps: int = 0


@dataclass
class Model:
    w: torch.Tensor          # vocabulary x n, frozen
    pool_a: torch.Tensor     # adapters x n x r
    pool_b: torch.Tensor     # adapters x r x vocabulary
    scales: torch.Tensor     # adapters floats
    adapters: List[Adapter]


def make_model(vocabulary, n, r, adapters, gen, bits=8, zero_b=True) -> Model:
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    w = (rand(vocabulary, n) * n ** -0.5).bfloat16()
    a, b = rand(adapters, n, r) * n ** -0.5, rand(adapters, r, vocabulary) * (0.0 if zero_b else r ** -0.5)
    made = [Adapter(a[i].clone(), b[i].clone(), L.loract_adamw_state([a[i], b[i]], bits=bits)) for i in range(adapters)]
    return Model(w, a.bfloat16(), b.bfloat16(), torch.full((adapters,), 0.5, device="cuda"), made)


def gradients(model: Model, index: int, x, targets, rank: int, seed: int):
    """(log probabilities of the targets, dA, dB) of the mean loss of adapter `index`."""
    a, b, scale = model.pool_a[index], model.pool_b[index], 0.5
    u, v = L.loract_compress(x, rank, seed=seed)
    t = L.loract_linear(x, a, w_transposed=True)
    logits = L.loract_linear(x, model.w, lora_t=t, lora_b=b, lora_scale=scale)
    live = targets >= 0
    weights = -live.float() / live.sum().clamp(min=1)
    logp, _, d_logits = L.loract_token_logprobs_grad(logits, targets, weights, out=logits)
    _, _, d_b = L.loract_linear_backward(d_logits, lora_t=t, lora_scale=scale, bias_grad=False, out=d_logits)
    d_a = L.loract_lora_grad(u, v, d_logits, b, scale)
    return logp, d_a, d_b


def train_step(model: Model, index: int, x, targets, rank: int = 64, lr: float = 1e-3, clip: float = 1.0):
    """One step of adapter `index`; returns the log probabilities before it.  Nothing here waits for the GPU."""
    it = model.adapters[index]
    it.steps += 1
    logp, d_a, d_b = gradients(model, index, x, targets, rank, it.steps)
    norm = torch.sqrt(d_a.square().sum() + d_b.square().sum())
    L.loract_adamw([it.a, it.b], [d_a, d_b], it.state, step=it.steps, lr=lr, weight_decay=0.0, seed=index, grad_scale=(clip / (norm + 1e-6)).clamp(max=1.0).view(1),
                   copies=[model.pool_a[index], model.pool_b[index]])
    return logp


def serve(model: Model, x, ids, top: int = 5) -> L.TokenLogprobs:
    """The alternatives of every token's next one, each under its own adapter (ids, negative for the bare projection)."""
    logits = L.loract_linear(x, model.w)
    L.loract_lora_requests(x, model.pool_a, model.pool_b, ids, model.scales, residual=logits, out=logits)
    return L.loract_token_logprobs(logits, top=top)


def main():
    m, n, vocabulary, r, count = 8192, 4096, 32000, 16, 8
    gen = torch.Generator(device="cuda").manual_seed(0)
    model = make_model(vocabulary, n, r, count, gen)
    x = torch.randn(m, n, generator=gen, device="cuda").bfloat16()
    targets = torch.randint(0, vocabulary, (m,), generator=gen, device="cuda")
    ids = (torch.arange(64, device="cuda") % count).int()

    def timed(f, reps):
        for _ in range(3):
            f()
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(reps):
            f()
        stop.record()
        torch.cuda.synchronize()
        return start.elapsed_time(stop) / reps

    step = timed(lambda: train_step(model, 0, x, targets, rank=128), 10)
    batch = timed(lambda: serve(model, x[:64], ids), 50)
    print("%d tokens x %d, vocabulary of %d, rank %d: %.2f ms a training step; %d tokens of %d adapters served in %.3f ms" %
          (m, n, vocabulary, r, step, ids.numel(), count, batch))


if __name__ == "__main__":
    main()
