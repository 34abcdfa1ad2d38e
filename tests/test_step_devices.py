"""Operands of loss, update and requests that live on different GPUs, or on one that is not the current one, are refused before the library is called."""
import pytest
import torch

import paper_2509_23472_amd as L
from paper_2509_23472_amd import api


def _calls():
    """name -> (operands by name, call)."""
    f = lambda *s: torch.zeros(*s)
    logits = dict(logits=f(4, 8), targets=torch.zeros(4, dtype=torch.int64), stats=f(3, 4), d_logp=f(4), d_entropy=f(4), out=f(4, 8))
    requests = dict(x=f(4, 8), a=f(3, 8, 2), b=f(3, 2, 6), ids=torch.zeros(4, dtype=torch.int32), scales=f(3), residual=f(4, 6), out=f(4, 6))
    state = L.AdamwState([4, 6], 8, torch.device("cpu"))
    adamw = dict(p=f(4), p2=f(6), g=f(4), g2=f(6), c=f(4).bfloat16(), c2=f(6).bfloat16(), m=state.m, v=state.v, exps=state.exps, lr=f(1), step=torch.zeros(1, dtype=torch.int64),
                 scale=f(1))
    return {
        "forward": ({k: logits[k] for k in ("logits", "targets")}, lambda o: L.loract_token_logprobs(o["logits"], o["targets"], top=2)),
        "backward": (logits, lambda o: L.loract_token_logprobs_backward(o["logits"], o["targets"], o["stats"], o["d_logp"], o["d_entropy"], out=o["out"])),
        "grad": ({k: v for k, v in logits.items() if k != "stats"},
                 lambda o: L.loract_token_logprobs_grad(o["logits"], o["targets"], o["d_logp"], o["d_entropy"], out=o["out"])),
        "requests": (requests, lambda o: L.loract_lora_requests(o["x"], o["a"], o["b"], o["ids"], o["scales"], residual=o["residual"], out=o["out"])),
        "adamw": (adamw, lambda o: L.loract_adamw([o["p"], o["p2"]], [o["g"], o["g2"]], state, step=o["step"], lr=o["lr"], grad_scale=o["scale"],
                                                  copies=[o["c"], o["c2"]]))}


class _Library:
    def __init__(self):
        self.reached = []

    def __getattr__(self, name):
        return lambda *args: self.reached.append(name) or 0


def _setup(monkeypatch, current, elsewhere=()):
    away = {id(t) for t in elsewhere}
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 1 if id(self) in away else 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    lib = _Library()
    monkeypatch.setattr(api._lib, "load", lambda: lib)
    return lib


@pytest.mark.parametrize("name,operand", [(n, o) for n, (operands, _) in _calls().items() for o in operands])
def test_an_operand_elsewhere(name, operand, monkeypatch):
    operands, call = _calls()[name]
    lib = _setup(monkeypatch, 0, [operands[operand]])
    with pytest.raises(ValueError):
        call(operands)
    assert lib.reached == []


@pytest.mark.parametrize("name", list(_calls()))
def test_the_current_gpu(name, monkeypatch):
    operands, call = _calls()[name]
    lib = _setup(monkeypatch, 0)
    call(operands)
    assert len(lib.reached) == 1
    lib = _setup(monkeypatch, 1)
    with pytest.raises(ValueError, match="not the current one"):
        call(operands)
    assert lib.reached == []
