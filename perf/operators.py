"""The sub-layer operators that are timed, each through the public entry points of the package.

What a LoRA fine-tuning program runs around a compressed activation, in training and in serving:

  linear    loract_linear: Y = R + D(act(X W^T + bias + s T B)); with the weights as they lie for the
            other direction it is the input gradient of the backward pass
  backward  loract_linear_backward: dP = act'(Z) D(dY), the bias gradient and the gradient of B
  dropout   loract_dropout: dropout whose mask is never stored, optionally added to a residual
  qk        loract_qknorm_rope_forward and, in training, loract_qknorm_rope_backward: RMS norm of every
            head of queries and keys and the rotation by position

The dropout mask is a function of (seed, row, column): the 16-bit field col % 4 of the splitmix64 output
number row * ceil(n / 4) + col / 4 + 1 of the seed, kept where it is at least round(65536 p).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------
# Cases.

def listed():
    return [
        # Attention output projection of a LLaMA-7B layer, 4 x 2048 tokens: LoRA update, dropout, residual.
        dict(name="attention_out", kind="linear", dtype="bf16", m=8192, n_in=4096, n_out=4096, layout="nt", act="none",
             bias=False, r=16, p=0.1, residual=True, keep=False),
        # MLP up-projection of the same layer with its activation; the pre-activation is kept for backward.
        dict(name="mlp_up", kind="linear", dtype="bf16", m=8192, n_in=4096, n_out=11008, layout="nt", act="silu",
             bias=True, r=16, p=0.0, residual=False, keep=True),
        # Its input gradient: the same weights, multiplied from the other side, added to the residual's gradient.
        dict(name="mlp_input_grad", kind="linear", dtype="bf16", m=8192, n_in=11008, n_out=4096, layout="nn", act="none",
             bias=False, r=16, p=0.0, residual=True, keep=False),
        # The LoRA down-projection T = X A of an attention input: a product with 16 columns.
        dict(name="lora_down", kind="linear", dtype="bf16", m=8192, n_in=4096, n_out=16, layout="nn", act="none",
             bias=False, r=0, p=0.0, residual=False, keep=False),
        # One token at a time in serving: the weights are read once for one row.
        dict(name="one_token", kind="linear", dtype="bf16", m=1, n_in=4096, n_out=11008, layout="nt", act="silu",
             bias=True, r=16, p=0.0, residual=False, keep=False),
        # Single precision, sizes that are no multiples of anything.
        dict(name="fp32_ragged", kind="linear", dtype="f32", m=3001, n_in=1030, n_out=770, layout="nt", act="gelu",
             bias=True, r=12, p=0.1, residual=True, keep=True),
        # Backward of the MLP up-projection's epilogue with the gradients of the bias and of LoRA's B.
        dict(name="mlp_up_backward", kind="backward", dtype="bf16", m=8192, n=11008, act="silu", r=16, p=0.0, bias=True),
        # The same for a ViT-B attention output of 64 images with dropout, in single precision.
        dict(name="vit_backward", kind="backward", dtype="f32", m=12608, n=768, act="gelu", r=8, p=0.1, bias=True),
        # Residual dropout of a LLaMA-7B sub-layer.
        dict(name="residual_dropout", kind="dropout", dtype="bf16", m=8192, n=4096, p=0.1, residual=True),
        # One image of 197 tokens: all latency.
        dict(name="one_image_dropout", kind="dropout", dtype="f32", m=197, n=768, p=0.05, residual=False),
        # Queries and keys of 4 x 2048 tokens as they lie in the packed projection, forward and backward.
        dict(name="qk_step", kind="qk", dtype="bf16", batch=4, seq=2048, hq=32, hk=8, d=128, rot=128, interleaved=False,
             grad=True, pad=0),
        # One new token for each of 4 sequences far into a long context.
        dict(name="qk_decode", kind="qk", dtype="bf16", batch=4, seq=1, hq=32, hk=8, d=128, rot=128, interleaved=False,
             grad=False, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, unit):
    """Log-uniform; mostly a multiple of `unit`, sometimes of 8, sometimes whatever it is."""
    v = _log(rng, lo, hi)
    how = rng.random()
    step = unit if how < 0.55 else (8 if how < 0.75 else 1)
    return max(lo, min(hi, v // step * step))


def draw(rng):
    kind = rng.choice(["linear"] * 5 + ["backward"] * 2 + ["dropout", "qk", "qk"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "linear":
        m = rng.choice([_log(rng, 1, 16), _log(rng, 16, 256), _size(rng, 256, 16384, 64), _size(rng, 256, 16384, 64)])
        n_in = _size(rng, 64, 11008, 64)
        n_out = _size(rng, 8, 64, 8) if rng.random() < 0.2 else _size(rng, 64, 11008, 64)
        top = 2 * 8192 * 4096 * 11008 // (1 if dtype == "bf16" else 8)
        m = max(1, min(m, top // (2 * n_in * n_out)))
        return dict(kind=kind, dtype=dtype, m=m, n_in=n_in, n_out=n_out, layout=rng.choice(["nt", "nt", "nn"]),
                    act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.5,
                    r=rng.choice([0, 0, 4, 8, 16, 16, 33, 64]), p=rng.choice([0.0, 0.0, 0.1, 0.37]),
                    residual=rng.random() < 0.5, keep=rng.random() < 0.4)
    if kind == "backward":
        n = _size(rng, 64, 11008, 64)
        return dict(kind=kind, dtype=dtype, m=min(_size(rng, 1, 16384, 64), 8192 * 11008 // n), n=n,
                    act=rng.choice(["none", "relu", "gelu", "silu"]), r=rng.choice([0, 0, 4, 8, 16, 16, 33, 64]),
                    p=rng.choice([0.0, 0.0, 0.1, 0.37]), bias=rng.random() < 0.7)
    if kind == "dropout":
        n = _size(rng, 64, 4096, 64)
        return dict(kind=kind, dtype=dtype, m=min(_size(rng, 1, 65536, 64), 8192 * 11008 // n), n=n,
                    p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5)
    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    hk = rng.choice([1, 2, 4, 8, 12])
    hq = hk * rng.choice([1, 1, 2, 4])
    grad = rng.random() < 0.6
    batch = _log(rng, 1, 16)
    seq = _log(rng, 1, 4096) if grad else rng.choice([1, _log(rng, 1, 4096)])
    batch = max(1, min(batch, 2 * 8192 * 40 * 128 // (seq * (hq + hk) * d)))
    seq = min(seq, 2 * 8192 * 40 * 128 // ((hq + hk) * d))
    return dict(kind=kind, dtype=dtype, batch=batch, seq=seq, hq=hq, hk=hk, d=d, rot=rng.choice([d, d, d, d // 2]),
                interleaved=rng.random() < 0.3, grad=grad, pad=rng.choice([0, 0, seq // 5]))


def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "linear":
        m, n_in, n_out, r = case["m"], case["n_in"], case["n_out"], case["r"]
        out = m * n_out * b
        return {"bytes": (m * n_in + n_in * n_out + (m + n_out) * r) * b + out * (1 + case["residual"] + case["keep"]) +
                         (4 * n_out if case["bias"] else 0),
                "flops": 2 * m * n_out * (n_in + r)}
    if case["kind"] == "backward":
        m, n, r = case["m"], case["n"], case["r"]
        return {"bytes": m * n * b * (2 + (case["act"] != "none")) + m * r * b + 4 * n * (r + case["bias"]),
                "flops": m * n * (2 * r + 10)}
    if case["kind"] == "dropout":
        return {"bytes": case["m"] * case["n"] * b * (2 + case["residual"]), "flops": 2 * case["m"] * case["n"]}
    m, heads = case["batch"] * case["seq"], case["hq"] + case["hk"]
    size = m * heads * case["d"]
    rows = case["batch"] if case["seq"] == 1 else case["seq"]
    return {"bytes": size * b * (5 if case["grad"] else 2) + 4 * (m + rows * case["rot"]),
            "flops": size * (24 if case["grad"] else 8)}


# ---------------------------------------------------------------------------------------------
# Inputs.

def _positions(case):
    """Positions of the tokens: every sequence starts at 0, its padding has none (-1); a decoding step stands far in."""
    seq, batch, pad = case["seq"], case["batch"], case["pad"]
    if seq == 1:
        return torch.tensor([65535 - 977 * i for i in range(batch)], dtype=torch.int32)
    one = torch.arange(seq, dtype=torch.int32)
    rows = one.repeat(batch, 1)
    if pad:
        rows[:, seq - pad:] = -1
    return rows.reshape(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).to(dt)

    s = dict(case=case, seed=(0x5851F42D4C957F2D * (seed + 1)) & (2 ** 64 - 1))
    if case["kind"] == "linear":
        m, n_in, n_out, r = case["m"], case["n_in"], case["n_out"], case["r"]
        s["x"] = normal(m, n_in)
        shape = (n_out, n_in) if case["layout"] == "nt" else (n_in, n_out)
        s["w"] = normal(*shape, scale=n_in ** -0.5)
        s["bias"] = torch.randn(n_out, generator=gen, device="cuda") * 0.1 if case["bias"] else None
        s["t"] = normal(m, r) if r else None
        s["b"] = normal(r, n_out, scale=r ** -0.5) if r else None
        s["res"] = normal(m, n_out) if case["residual"] else None
        s["scale"] = 0.5
    elif case["kind"] == "backward":
        m, n, r = case["m"], case["n"], case["r"]
        s["dy"] = normal(m, n)
        s["z"] = normal(m, n, scale=1.5) if case["act"] != "none" else None
        s["t"] = normal(m, r) if r else None
        s["scale"] = 0.5
    elif case["kind"] == "dropout":
        s["x"] = normal(case["m"], case["n"])
        s["res"] = normal(case["m"], case["n"]) if case["residual"] else None
    else:
        m, hq, hk, d, rot = case["batch"] * case["seq"], case["hq"], case["hk"], case["d"], case["rot"]
        qkv = normal(m, (hq + 2 * hk) * d)
        s["q"] = qkv[:, :hq * d].view(m, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hk) * d].view(m, hk, d)
        s["gq"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")
        s["gk"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")
        s["pos"] = _positions(case).cuda()
        n_pos = 65536 if case["seq"] == 1 else case["seq"]
        angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2.0 / rot)
        s["table"] = torch.stack([angle.cos(), angle.sin()], dim=1).float().cuda()
        if case["grad"]:
            s["dq"] = normal(m, hq, d)
            s["dk"] = normal(m, hk, d)
    return s


# ---------------------------------------------------------------------------------------------
# One pass.

def run(s):
    case = s["case"]
    return _run_own(s, case) if own else _PLAIN[case["kind"]](s, case)


def _run_own(s, case):
    import paper_2509_23472_amd as L
    if case["kind"] == "linear":
        return L.loract_linear(s["x"], s["w"], s["bias"], w_transposed=case["layout"] == "nn", lora_t=s["t"], lora_b=s["b"],
                               lora_scale=s["scale"], act=case["act"], p_drop=case["p"], seed=s["seed"], residual=s["res"],
                               save_preact=case["keep"])
    if case["kind"] == "backward":
        out = L.loract_linear_backward(s["dy"], s["z"], lora_t=s["t"], lora_scale=s["scale"], act=case["act"],
                                       p_drop=case["p"], seed=s["seed"], bias_grad=case["bias"])
        return [o for o in out if o is not None]
    if case["kind"] == "dropout":
        return L.loract_dropout(s["x"], case["p"], s["seed"], residual=s["res"])
    rope = dict(positions=s["pos"], eps=EPS, interleaved=case["interleaved"])
    out = list(L.loract_qknorm_rope_forward(s["q"], s["k"], s["gq"], s["gk"], s["table"], **rope))
    if case["grad"]:
        out += list(L.loract_qknorm_rope_backward(s["q"], s["k"], s["gq"], s["gk"], s["table"], s["dq"], s["dk"], **rope))
    return out


def _logical_shift(x, bits):
    return (x >> bits) & ((1 << (64 - bits)) - 1)


def _signed(v):
    return v - (1 << 64) if v >= 1 << 63 else v


def _plain_mask(seed, m, n, p):
    """The kept elements (m x n truth values) and the factor they are multiplied with; 64-bit integers wrap."""
    thr = min(65535, int(round(p * 65536)))
    groups = (n + 3) // 4
    z = torch.arange(1, m * groups + 1, device="cuda", dtype=torch.int64) * _signed(0x9E3779B97F4A7C15) + _signed(seed)
    z = (z ^ _logical_shift(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _logical_shift(z, 27)) * _signed(0x94D049BB133111EB)
    z = z ^ _logical_shift(z, 31)
    fields = torch.stack([_logical_shift(z, 16 * i) & 0xFFFF if i else z & 0xFFFF for i in range(4)], dim=-1)
    return fields.view(m, groups * 4)[:, :n] >= thr, 65536.0 / (65536 - thr)


def _plain_dropout(v, seed, p):
    if p == 0.0:
        return v
    keep, factor = _plain_mask(seed, v.shape[0], v.shape[1], p)
    return torch.where(keep, v * factor, torch.zeros_like(v))


def _plain_linear(s, case):
    dt = DT[case["dtype"]]
    w = s["w"].float()
    z = s["x"].float() @ (w.t() if case["layout"] == "nt" else w)
    if s["t"] is not None:
        z = z + s["scale"] * (s["t"].float() @ s["b"].float())
    if s["bias"] is not None:
        z = z + s["bias"]
    y = z
    if case["act"] == "relu":
        y = torch.where(z < 0, torch.zeros_like(z), z)
    elif case["act"] == "gelu":
        y = 0.5 * z * (1.0 + torch.erf(z * 0.7071067811865476))
    elif case["act"] == "silu":
        y = z / (1.0 + torch.exp(-z))
    y = _plain_dropout(y, s["seed"], case["p"])
    if s["res"] is not None:
        y = y + s["res"].float()
    return (y.to(dt), z.to(dt)) if case["keep"] else y.to(dt)


def _plain_backward(s, case):
    g = _plain_dropout(s["dy"].float(), s["seed"], case["p"])
    if case["act"] != "none":
        z = s["z"].float()
        if case["act"] == "relu":
            g = torch.where(z > 0, g, torch.zeros_like(g))
        elif case["act"] == "gelu":
            g = g * (0.5 * (1.0 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327)
        else:
            sig = 1.0 / (1.0 + torch.exp(-z))
            g = g * (sig * (1.0 + z * (1.0 - sig)))
    out = [g.to(DT[case["dtype"]])]
    if case["bias"]:
        out.append(g.sum(0))
    if s["t"] is not None:
        out.append(s["scale"] * (s["t"].float().t() @ g))
    return out


def _plain_dropout_case(s, case):
    y = _plain_dropout(s["x"].float(), s["seed"], case["p"])
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(DT[case["dtype"]])


def _rotate(y, cos, sin, rot, interleaved):
    """Rotates the pairs of the first `rot` elements of every head; cos and sin are tokens x 1 x rot / 2."""
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([ra, rb], dim=-1).flatten(-2) if interleaved else torch.cat([ra, rb], dim=-1)
    return torch.cat([turned, y[..., rot:]], dim=-1)


def _plain_qk(s, case):
    dt, rot, inter = DT[case["dtype"]], case["rot"], case["interleaved"]
    live = (s["pos"] >= 0)[:, None, None]
    rows = s["table"][s["pos"].clamp(min=0).long()]
    cos, sin = rows[:, 0][:, None, :], rows[:, 1][:, None, :]
    fwd, grads, gammas = [], [], []
    for x, gamma, dy in ((s["q"], s["gq"], s.get("dq")), (s["k"], s["gk"], s.get("dk"))):
        x = x.float()
        inv = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        hat = x * inv
        y = _rotate(hat * gamma, cos, sin, rot, inter)
        fwd.append(torch.where(live, y, torch.zeros_like(y)).to(dt))
        if case["grad"]:
            t = _rotate(dy.float(), cos, -sin, rot, inter)
            t = torch.where(live, t, torch.zeros_like(t))
            gammas.append((t * hat).sum((0, 1)))
            t = t * gamma
            grads.append(((t - hat * (t * hat).mean(-1, keepdim=True)) * inv).to(dt))
    return fwd + grads + gammas


_PLAIN = {"linear": _plain_linear, "backward": _plain_backward, "dropout": _plain_dropout_case, "qk": _plain_qk}


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits.

def _exact_factor(seed, m, n, p):
    """What dropout multiplies every element with (m x n): 0 or 1 / (1 - p), p in steps of 2^-16."""
    if p == 0.0:
        return torch.ones((), dtype=torch.float64, device="cuda")
    thr = min(65535, int(round(p * 65536)))
    per_row = -(-n // 4)
    with np.errstate(over="ignore"):
        state = np.uint64(seed) + np.arange(1, m * per_row + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15)
        state ^= state >> np.uint64(30)
        state *= np.uint64(0xBF58476D1CE4E5B9)
        state ^= state >> np.uint64(27)
        state *= np.uint64(0x94D049BB133111EB)
        state ^= state >> np.uint64(31)
    fields = state.astype("<u8").view("<u2").reshape(m, per_row * 4)[:, :n]
    return torch.from_numpy(fields >= thr).cuda().double() * (65536.0 / (65536 - thr))


def _exact_act(name, z):
    if name == "relu":
        return z * (z > 0)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_act_slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    sig = torch.sigmoid(z)
    return sig + z * sig * torch.sigmoid(-z)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        w = s["w"].double()
        if case["layout"] == "nt":
            w = w.t().contiguous()
        z = torch.mm(s["x"].double(), w)
        if case["r"]:
            z += torch.mm(s["t"].double(), s["b"].double()) * s["scale"]
        if case["bias"]:
            z += s["bias"].double()
        y = _exact_act(case["act"], z) * _exact_factor(s["seed"], case["m"], case["n_out"], case["p"])
        if case["residual"]:
            y = y + s["res"].double()
        return (y, z) if case["keep"] else y
    if case["kind"] == "backward":
        g = s["dy"].double() * _exact_factor(s["seed"], case["m"], case["n"], case["p"])
        if case["act"] != "none":
            g = g * _exact_act_slope(case["act"], s["z"].double())
        out = [g]
        if case["bias"]:
            out.append(torch.mm(torch.ones(1, case["m"], dtype=torch.float64, device="cuda"), g)[0])
        if case["r"]:
            out.append(torch.mm(s["t"].double().t().contiguous(), g) * s["scale"])
        return out
    if case["kind"] == "dropout":
        y = s["x"].double() * _exact_factor(s["seed"], case["m"], case["n"], case["p"])
        return y + s["res"].double() if case["residual"] else y
    # Rotations as complex products: (a + ib) e^{i angle}; the transpose of a rotation is the conjugate's product.
    pos = s["pos"].long()
    live = (pos >= 0).double()
    rows = s["table"].double()[pos.clamp(min=0)]
    turn = torch.complex(rows[:, 0], rows[:, 1])[:, None, :]
    half, rot = case["rot"] // 2, case["rot"]

    def turned(v, by):
        out = v.clone()
        if case["interleaved"]:
            c = torch.view_as_complex(v[..., :rot].reshape(*v.shape[:2], half, 2).contiguous()) * by
            out[..., :rot] = torch.view_as_real(c).flatten(-2)
        else:
            c = torch.complex(v[..., :half].contiguous(), v[..., half:rot].contiguous()) * by
            out[..., :half], out[..., half:rot] = c.real, c.imag
        return out * live[:, None, None]

    fwd, grads, gammas = [], [], []
    for name, gamma in (("q", s["gq"].double()), ("k", s["gk"].double())):
        x = s[name].double()
        rms = (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        fwd.append(turned(x / rms * gamma, turn))
        if case["grad"]:
            t = turned(s["d" + name].double(), turn.conj())
            gammas.append((t * (x / rms)).sum((0, 1)))
            inner = (t * gamma * x).mean(-1, keepdim=True) / rms.square()
            grads.append((t * gamma - x * inner) / rms)
    return fwd + grads + gammas
