"""The microscaled calls marshalled in C++ against marshalling in Python: the same bits, the same refusals."""
import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding


class _Counted:
    """The module, and which of its calls were made and which were left to Python."""

    def __init__(self, module):
        self.module, self.made, self.left = module, [], []

    def __getattr__(self, name):
        def call(*args):
            got = getattr(self.module, name)(*args)
            (self.made if got else self.left).append(name)
            return got

        return call


def _calls(device, N=70, din=100, dout=60, k=8):
    gen = torch.Generator(device=device).manual_seed(3)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=device)
    t = {"X": randn(N, din), "dH": randn(N, dout), "dXs": randn(N, k), "bias": randn(dout),
         "sp_index": torch.arange(k, device=device).repeat(N, 1).mul(7).to(torch.uint8)}
    for bits in (8, 4):
        t[f"c{bits}"], t[f"s{bits}"] = (x.zero_() for x in maxk.mx_empty(N, din, bits, device))
    t["wc"], t["ws"] = (x.random_(100, 130, generator=gen) for x in maxk.mx_empty(dout, din, 4, device))
    t["out"], t["Y"], t["dW"], t["db"], t["dX"] = (torch.zeros(*s, device=device) for s in ((N, din), (N, dout), (dout, din), (dout,), (N, din)))
    calls = {
        "quantize 8": lambda: maxk.maxk_mx_quantize(t["X"], t["c8"], t["s8"]),
        "quantize 4": lambda: maxk.maxk_mx_quantize(t["X"], t["c4"], t["s4"]),
        "dequantize": lambda: maxk.maxk_mx_dequantize(t["c8"], t["s8"], t["out"]),
        "linear": lambda: maxk.maxk_mx_linear(t["c4"], t["s4"], t["wc"], t["ws"], t["Y"], t["bias"]),
        "linear without bias": lambda: maxk.maxk_mx_linear(t["c4"], t["s4"], t["wc"], t["ws"], t["Y"]),
        "weight_grad": lambda: maxk.maxk_mx_weight_grad(t["c8"], t["s8"], t["dH"], t["dW"], t["db"]),
        "weight_grad_cbsr": lambda: maxk.maxk_mx_weight_grad_cbsr(t["c4"], t["s4"], t["dXs"], t["sp_index"], t["dW"]),
        "input_grad": lambda: maxk.maxk_mx_input_grad(t["dH"], t["wc"], t["ws"], t["dX"]),
        "input_grad_cbsr": lambda: maxk.maxk_mx_input_grad_cbsr(t["dXs"], t["sp_index"], t["wc"], t["ws"], t["dX"]),
    }
    return t, calls


def test_host_tensors_are_refused_alike(monkeypatch):
    binding.load_library()
    for name, call in _calls("cpu")[1].items():
        got = []
        for fast in (binding._FAST, None):
            monkeypatch.setattr(binding, "_FAST", fast)
            with pytest.raises(maxk.MaxKError) as e:
                call()
            got.append(str(e.value))
            monkeypatch.undo()
        assert got[0] == got[1], name


@pytest.mark.gpu
def test_calls_give_the_same_bits(monkeypatch):
    binding.load_library()
    results = []
    for fast in (True, False):
        t, calls = _calls("cuda")
        counted = _Counted(binding._FAST)
        monkeypatch.setattr(binding, "_FAST", counted if fast else None)
        for call in calls.values():
            call()
        monkeypatch.undo()
        torch.cuda.synchronize()
        assert (len(counted.made), len(counted.left)) == ((len(calls), 0) if fast else (0, 0))
        results.append([x.clone() for x in t.values()])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_what_does_not_fit_is_left_to_python_and_named(monkeypatch):
    binding.load_library()
    t, _ = _calls("cuda")
    counted = _Counted(binding._FAST)
    monkeypatch.setattr(binding, "_FAST", counted)
    refused = [
        lambda: maxk.maxk_mx_quantize(t["X"].double(), t["c8"], t["s8"]),
        lambda: maxk.maxk_mx_quantize(t["X"], t["c8"][:-1], t["s8"]),
        lambda: maxk.maxk_mx_quantize(t["X"].t(), *maxk.mx_empty(100, 70, 8)),
        lambda: maxk.maxk_mx_dequantize(t["c8"], t["s4"].int(), t["out"]),
        lambda: maxk.maxk_mx_linear(t["c8"], t["s8"], t["wc"], t["ws"], t["Y"]),
        lambda: maxk.maxk_mx_linear(t["c4"], t["s4"], t["wc"], t["ws"], t["Y"], t["bias"][:-1]),
        lambda: maxk.maxk_mx_linear(t["c4"], t["s4"], t["wc"], t["ws"], t["Y"][:, :-1]),
        lambda: maxk.maxk_mx_weight_grad(t["c8"], t["s8"], t["dH"][:, :-1].contiguous(), t["dW"]),
        lambda: maxk.maxk_mx_weight_grad(t["c8"], t["s8"], t["dH"], t["dW"], t["db"], torch.empty(4, dtype=torch.uint8, device="cuda")),
        lambda: maxk.maxk_mx_weight_grad_cbsr(t["c8"], t["s8"], t["dXs"], t["sp_index"].long(), t["dW"]),
        lambda: maxk.maxk_mx_weight_grad_cbsr(t["c8"], t["s8"], t["dXs"], t["sp_index"], t["dW"].half()),
        lambda: maxk.maxk_mx_input_grad(t["dH"], t["wc"][:-1], t["ws"][:-1], t["dX"]),
        lambda: maxk.maxk_mx_input_grad_cbsr(t["dXs"], t["sp_index"], t["wc"], t["ws"][:-1], t["dX"]),
        lambda: maxk.maxk_mx_input_grad_cbsr(t["dXs"].bfloat16(), t["sp_index"], t["wc"], t["ws"], t["dX"]),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(maxk.MaxKError):
            call()
            pytest.fail(f"call {i} was made")
    monkeypatch.undo()
    assert not counted.made
