"""Activations and their slopes over the range of their arguments, through every form of the linear map, against 64 bits.

A matrix of inputs whose first column is z, times weights whose first column is one and whose others are zero: P = z exactly, so that
what is off is the activation's alone.  Bounds in units of 2^-24, relative: silu 8 (exp 3, reciprocal 2, three roundings); gelu 16 (the
same, Phi's polynomial 6 and two more roundings) and z^2 / 2, by which its exponent is rounded.
"""
import math

import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu

# (n_in, n_out, tokens at a time): few outputs; few outputs with K split; few tokens, both layouts; tiles; tiles with K split
FORMS = {"few_outputs": (64, 8, 8192, "nt"), "few_outputs_split": (2048, 8, 256, "nt"), "few_tokens": (64, 40, 16, "nt"),
         "few_tokens_as_it_lies": (64, 64, 16, "nn"), "tiles": (64, 40, 8192, "nt"), "tiles_split": (1024, 40, 512, "nt"),
         "tiles_as_they_lie": (64, 40, 8192, "nn")}


def _ends():
    """8192 values, dense where exp(-z) passes out of the range of float32 and where sigmoid becomes 1."""
    z = torch.cat([torch.linspace(-110.0, -80.0, 4096), torch.linspace(80.0, 110.0, 2048), torch.linspace(-80.0, 80.0, 2048)])
    return z.float()


def _act(name, z):
    """ref.act, with gelu's left tail by erfc: 1 + erf(z / sqrt(2)) has no digits left of it below z = -8, in 64 bits either."""
    return 0.5 * z * torch.special.erfc(-z / math.sqrt(2)) if name == "gelu" else ref.act(name, z)


def _forward(z, form, act, dtype=torch.float32, out_dtype=None):
    import paper_2509_23472_amd as L
    n_in, n_out, at_once, layout = FORMS.get(form) or LARGE[form]
    z = z[:256] if at_once < 64 else z
    w = torch.zeros(n_out, n_in, dtype=dtype, device="cuda")
    w[:, 0] = 1.0
    if layout == "nn":
        w = w.t().contiguous()
    parts = []
    for part in z.split(at_once):
        x = torch.zeros(len(part), n_in, dtype=dtype, device="cuda")
        x[:, 0] = part.cuda()
        parts.append(L.loract_linear(x, w, act=act, w_transposed=layout == "nn", out_dtype=out_dtype))
    return z, torch.cat(parts)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_float32_activations_at_the_ends_of_the_range(act, form):
    z = _ends()
    if FORMS[form][2] < 64:
        z = z[::32]
    z, y = _forward(z, form, act)
    assert torch.isfinite(y).all()
    want = _act(act, z.double())[:, None].expand(y.shape)
    # (1e-36: results below the smallest normal number may be zero, and so may be the sigmoid that is multiplied with z)
    rel = 2.0 ** -24 * (16 + z.double().square() / 2 if act == "gelu" else torch.full_like(z.double(), 8.0))
    ref.check(y, want, (rel * want[:, 0].abs())[:, None] + 1e-36, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("r", [0, 8])
def test_float32_slopes_at_the_ends_of_the_range(act, r):
    import paper_2509_23472_amd as L
    z = _ends().view(1024, 8).contiguous()
    t = torch.ones(1024, r, device="cuda") if r else None
    dp, db, d_b = L.loract_linear_backward(torch.ones(1024, 8, device="cuda"), z.cuda(), act=act, lora_t=t)
    want = ref.slope(act, z.double())
    assert torch.isfinite(dp).all() and torch.isfinite(db).all() and (d_b is None or torch.isfinite(d_b).all())
    # a slope is a sum of terms up to 1 + |z| in size, each a few roundings; silu's left tail is s (1 + z (1 - s)) without cancellation
    bound = 16 * 2.0 ** -24 * (1 + z.double().abs())
    if act == "silu":
        bound = torch.where(z < -2, 16 * 2.0 ** -24 * want.abs() + 1e-36, bound)
    ref.check(dp, want, bound, act)


@pytest.mark.parametrize("form", ["few_outputs", "tiles", "tiles_split"])
def test_float32_gelu_near_zero_and_above(form):
    """In units of 2^-24: Phi = 1/2 + z r rounded (Phi) and multiplied with z (Phi), z r half of a unit by r's rounding and a quarter by
    its polynomial; above sqrt(2), 1 less a tail of at most 0.08 that is up to 16 units off itself."""
    z = torch.cat([torch.linspace(-1.0, 1.0, 4096), torch.linspace(1.0, 20.0, 2048), torch.logspace(-12, 0, 2048)])
    z, y = _forward(z, form, "gelu")
    z = z.double()
    phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    bound = z.abs() * (2 * phi + torch.where(z > math.sqrt(2), 1.25, 0.75)) * 2.0 ** -24
    ref.check(y, (z * phi)[:, None].expand(y.shape), bound[:, None], "gelu")


# tiles of bf16 operands: 128 x 128 whole and with K split, and 256 x 256
LARGE = {"large": (64, 200, 4096, "nt"), "large_as_it_lies": (64, 200, 4096, "nn"), "large_split": (2048, 128, 512, "nt"),
         "large_256": (64, 256, 65536, "nt")}


@pytest.mark.parametrize("form", list(FORMS) + list(LARGE))
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_float32_results_of_bf16_operands(act, form):
    """What follows the product of bf16 operands is rounded no earlier than its result is."""
    z = torch.unique(torch.cat([_ends(), torch.linspace(-20.0, 20.0, 4096)]).bfloat16())
    at_once = (FORMS.get(form) or LARGE[form])[2]
    z = z.float()
    z = z[::16] if at_once < 64 else z.repeat(1 + at_once // len(z))[:max(at_once, len(z))]
    z, y = _forward(z, form, act, torch.bfloat16, torch.float32)
    assert y.dtype == torch.float32
    want = _act(act, z.double())[:, None].expand(y.shape)
    rel = 2.0 ** -24 * (16 + z.double().square() / 2 if act == "gelu" else torch.full_like(z.double(), 8.0))
    ref.check(y, want, (rel * want[:, 0].abs())[:, None] + 1e-36, act)
