"""The run of loss, update and serving of examples/adapters_train_and_serve.py against 64 bits.

Tolerances: the activations have rank 12 and are compressed at rank 16, so their factors give them back up to bf16.  A gradient passes through about a
dozen bf16 roundings (factors, T, logits, their gradient, A and B in bf16), 2^-8 each and independent: 2^-8 sqrt(12) = 1.4e-2 of its norm, and as much
again for their growth in the products.
"""
import os
import sys

import pytest
import torch

import paper_2509_23472_amd as L
import step_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
TOL = 2.8e-2


def _data(m, n, vocabulary, gen):
    x = torch.randn(m, 12, generator=gen, device="cuda") @ torch.randn(12, n, generator=gen, device="cuda")
    x = (x / x.square().mean(1, keepdim=True).sqrt()).bfloat16()
    targets = torch.randint(0, vocabulary, (m,), generator=gen, device="cuda")
    targets[::7] = -1
    return x, targets


@pytest.mark.parametrize("m,n,vocabulary,r", [(200, 128, 1000, 8), (1100, 256, 2049, 16)])
def test_gradients(m, n, vocabulary, r):
    import adapters_train_and_serve as ex
    gen = torch.Generator(device="cuda").manual_seed(1)
    model = ex.make_model(vocabulary, n, r, 3, gen, zero_b=False)
    x, targets = _data(m, n, vocabulary, gen)
    logp, d_a, d_b = ex.gradients(model, 1, x, targets, 16, 5)
    a, b = (t[1].double().requires_grad_() for t in (model.pool_a, model.pool_b))
    z = x.double() @ model.w.double().t() + 0.5 * (x.double() @ a) @ b
    want = torch.log_softmax(z, 1).gather(1, targets.clamp(min=0)[:, None])[:, 0] * (targets >= 0)
    (-want.sum() / (targets >= 0).sum()).backward()
    # a logit is off by 2^-8 of itself and T by as much of it
    assert ((logp - want.detach()).abs() <= 2 * 2.0 ** -7 * z.detach().abs().amax(1)).all()
    for got, leaf in ((d_a, a), (d_b, b)):
        assert (got.double() - leaf.grad).norm() <= TOL * leaf.grad.norm()


@pytest.mark.parametrize("bits", [8, 32])
def test_steps_then_serving(bits):
    import adapters_train_and_serve as ex
    gen = torch.Generator(device="cuda").manual_seed(2)
    model = ex.make_model(1000, 128, 8, 3, gen, bits=bits)
    x, targets = _data(256, 128, 1000, gen)
    before = [t.clone() for t in (model.pool_a, model.pool_b)]
    for step in range(3):
        for index in (0, 2):
            ex.train_step(model, index, x, (targets + index) % 1000, rank=16)
    for pool, old, name in ((model.pool_a, before[0], "a"), (model.pool_b, before[1], "b")):
        assert torch.equal(pool[1], old[1]) and torch.isfinite(pool).all()
        for index in (0, 2):
            assert not torch.equal(pool[index], old[index]) and torch.equal(pool[index], getattr(model.adapters[index], name).bfloat16())
    ids = torch.randint(-1, 3, (256,), generator=gen, device="cuda").int()
    got = ex.serve(model, x, ids, top=4)
    # the same logits one adapter at a time, and what serving made of them
    logits = L.loract_linear(x, model.w)
    want, off = ref.lora_requests(x, model.pool_a, model.pool_b, ids, model.scales, logits)
    L.loract_lora_requests(x, model.pool_a, model.pool_b, ids, model.scales, residual=logits, out=logits)
    assert ((logits.double() - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()
    again = L.loract_token_logprobs(logits, top=4)
    assert torch.equal(got.top_ids, again.top_ids) and torch.equal(got.top_logp, again.top_logp) and torch.equal(got.top_ids, ref.top(logits, 4))


def test_script_runs(capsys):
    import adapters_train_and_serve as ex
    ex.main()
    assert "training step" in capsys.readouterr().out
