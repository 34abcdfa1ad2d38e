"""The sub-layers of examples/prenorm_sublayers.py against autograd in 64 bits.

The activations have rank 12 and are compressed at rank 16, so that what the backward pass reconstructs is the activation up to the
rounding of its factors: 2^-8 for every bf16 number that is stored on the way.  A gradient passes through about a dozen of them
(factors, reconstruction, pre-activation, dP, dX, the norm's input and output), whose relative errors are independent: 2^-8 sqrt(12) = 1.4e-2
of its norm, with as much again for their growth in the products; float32 is bound by the compression's own tolerance, 1e-5, likewise.
"""
import os
import sys

import pytest
import torch

import sublayer_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
TOL = {torch.bfloat16: 2.8e-2, torch.float32: 1e-4}


def _close(got, want, dtype, what):
    err = ((got.double() - want).norm() / want.norm()).item()
    assert err <= TOL[dtype], (what, err)


def _activation(m, n, dtype, gen):
    """An input whose norm has rank 12: rows of one length."""
    x = torch.randn(m, 12, generator=gen, device="cuda") @ torch.randn(12, n, generator=gen, device="cuda")
    return (x / x.square().mean(1, keepdim=True).sqrt()).to(dtype)


def _norm(x, gamma, eps):
    return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gamma


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,ffn,r", [(200, 128, 320, 8), (1024, 256, 512, 16), (77, 136, 200, 3)])
def test_mlp(m, n, ffn, r, dtype):
    import prenorm_sublayers as ex
    gen = torch.Generator(device="cuda").manual_seed(1)
    p = ex.make_mlp(n, ffn, r, dtype, gen)
    x, dy = _activation(m, n, dtype, gen), torch.randn(m, n, generator=gen, device="cuda").to(dtype)
    y, kept = ex.mlp_forward(p, x, 16, 5)
    got = ex.mlp_backward(p, kept, dy)
    leaf = {k: v.double().requires_grad_() for k, v in dict(x=x, b1=p.b1, b2=p.b2, a=p.lora.a, b=p.lora.b).items()}
    a = _norm(leaf["x"], p.gamma.double(), p.eps)
    z = a @ p.w1.double().t() + p.lora.scale * (a @ leaf["a"]) @ leaf["b"] + leaf["b1"]
    drop = ref.drop_factors(m, n, p.p_drop, 5).cuda()
    want = ((z * torch.sigmoid(z)) @ p.w2.double().t() + leaf["b2"]) * drop + leaf["x"]
    _close(y, want.detach(), dtype, "y")
    want.backward(dy.double())
    for name, value in got.items():
        _close(value, leaf[name].grad, dtype, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,hq,hk,d,r", [(256, 128, 4, 2, 32, 8), (300, 192, 6, 1, 64, 5)])
def test_attention_inputs(m, n, hq, hk, d, r, dtype):
    import prenorm_sublayers as ex
    gen = torch.Generator(device="cuda").manual_seed(2)
    p = ex.make_attention(n, hq, hk, d, r, m, dtype, gen)
    x = _activation(m, n, dtype, gen)
    positions = torch.arange(m, dtype=torch.int32, device="cuda") % (m // 2)
    (q, k, v), kept = ex.attention_inputs(p, x, positions, 16, 6)
    dq, dk, dv = (torch.randn(t.shape, generator=gen, device="cuda").to(dtype) for t in (q, k, v))
    got = ex.attention_inputs_backward(p, kept, dq, dk, dv)
    leaf = {name: t.double().requires_grad_() for name, t in dict(x=x, a=p.lora.a, b=p.lora.b, gamma_q=p.gamma_q, gamma_k=p.gamma_k).items()}
    a = _norm(leaf["x"], p.gamma.double(), p.eps)
    packed = a @ p.wqkv.double().t() + p.lora.scale * (a @ leaf["a"]) @ leaf["b"]
    rows = p.table.double()[positions.long()]

    def rotated(t, gamma):
        t = _norm(t, gamma, p.eps)
        lo, hi, c, s = t[..., :d // 2], t[..., d // 2:], rows[:, 0][:, None], rows[:, 1][:, None]
        return torch.cat([lo * c - hi * s, lo * s + hi * c], -1)

    wq, wk, wv = (t.reshape(m, -1, d) for t in packed.split([hq * d, hk * d, hk * d], 1))
    wq, wk = rotated(wq, leaf["gamma_q"]), rotated(wk, leaf["gamma_k"])
    for have, want, name in ((q, wq, "q"), (k, wk, "k"), (v, wv, "v")):
        _close(have, want.detach(), dtype, name)
    torch.autograd.backward([wq, wk, wv], [dq.double(), dk.double(), dv.double()])
    for name, value in got.items():
        _close(value, leaf[name].grad, dtype, name)
