"""The sub-layer's binding refuses operands that live on different GPUs, or on one that is not the current one, before the library is called."""
import pytest
import torch

import paper_2509_23472_amd as L
from paper_2509_23472_amd import api


class On:
    """A tensor that says it lives on that GPU."""

    def __init__(self, tensor, device):
        self._tensor, self._device = tensor, device

    def __getattr__(self, name):
        return getattr(self._tensor, name)

    def get_device(self):
        return self._device


class NoLibrary:
    def __getattr__(self, name):
        raise AssertionError("the library was called: " + name)


def _calls(d):
    """Every entry point with all operands on GPU 0 but the one that `d` names."""
    at = lambda name, *shape, dtype=torch.float32: On(torch.zeros(*shape, dtype=dtype), 1 if name == d else 0)
    return {
        "dropout": lambda: L.loract_dropout(at("x", 4, 8), 0.1, 0, residual=at("residual", 4, 8), out=at("out", 4, 8)),
        "linear": lambda: L.loract_linear(at("x", 4, 8), at("w", 6, 8), at("bias", 6), lora_t=at("lora_t", 4, 2), lora_b=at("lora_b", 2, 6),
                                          residual=at("residual", 4, 6), out=at("out", 4, 6)),
        "backward": lambda: L.loract_linear_backward(at("dy", 4, 6), at("z", 4, 6), act="silu", lora_t=at("lora_t", 4, 2), out=at("out", 4, 6)),
        "forward qk": lambda: L.loract_qknorm_rope_forward(at("q", 4, 2, 8), at("k", 4, 2, 8), at("gamma_q", 8), at("gamma_k", 8), at("table", 4, 2, 4),
                                                           positions=at("positions", 4, dtype=torch.int32), out=(at("out", 4, 2, 8), at("out_k", 4, 2, 8))),
        "backward qk": lambda: L.loract_qknorm_rope_backward(at("q", 4, 2, 8), at("k", 4, 2, 8), at("gamma_q", 8), at("gamma_k", 8), at("table", 4, 2, 4),
                                                             at("dq", 4, 2, 8), at("dk", 4, 2, 8), out=(at("out", 4, 2, 8), at("out_k", 4, 2, 8)))}


OPERANDS = {"dropout": ["x", "residual", "out"], "linear": ["x", "w", "bias", "lora_t", "lora_b", "residual", "out"],
            "backward": ["dy", "z", "lora_t", "out"], "forward qk": ["q", "k", "gamma_q", "gamma_k", "table", "positions", "out", "out_k"],
            "backward qk": ["q", "k", "gamma_q", "gamma_k", "table", "dq", "dk", "out", "out_k"]}


@pytest.mark.parametrize("call,operand", [(c, o) for c, names in OPERANDS.items() for o in names])
def test_operands_on_different_gpus(call, operand, monkeypatch):
    monkeypatch.setattr(api._lib, "load", lambda: NoLibrary())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError):
        _calls(operand)[call]()


@pytest.mark.parametrize("call", ["dropout", "forward qk"])
def test_operands_on_a_gpu_that_is_not_the_current_one(call, monkeypatch):
    class Names:
        def __getattr__(self, name):
            return lambda *args: pytest.fail("the library was called: " + name)
    monkeypatch.setattr(api._lib, "load", lambda: Names())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    with pytest.raises(ValueError, match="not the current one"):
        _calls(None)[call]()


def test_enqueue_asks_for_the_current_gpu(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="not the current one"):
        api._enqueue(lambda *args: pytest.fail("the library was called"), (), None, b"", 0, "call")
