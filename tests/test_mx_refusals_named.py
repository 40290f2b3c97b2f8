"""Each refusal of the microscaled calls' Python side by its own message: tensors are taken for device tensors, so that nothing else can refuse them."""
import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding


class _Made(Exception):
    pass


class _Library:
    """Every call has been made; the workspace query alone answers."""

    def __getattr__(self, name):
        def call(*args):
            if name == "maxk_mx_weight_grad_workspace":
                return 64
            raise _Made(name)

        return call


@pytest.fixture(autouse=True)
def host_tensors_pass(monkeypatch):
    def dev(t, dtype, what):
        if not t.is_contiguous() or t.dtype != dtype:
            raise maxk.MaxKError(f"{what}: expected a contiguous device tensor of {dtype}")
        return t.data_ptr()

    monkeypatch.setattr(binding, "_FAST", None)
    monkeypatch.setattr(binding, "_dev", dev)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "load_library", _Library)


N, DIN, DOUT, K = 4, 40, 8, 2
F32, U8 = torch.float32, torch.uint8
X, dH, dXs, dW = (torch.zeros(*s) for s in ((N, DIN), (N, DOUT), (N, K), (DOUT, DIN)))
c8, c4, s = torch.zeros(N, 64, dtype=torch.int8), torch.zeros(N, 32, dtype=U8), torch.zeros(N, 2, dtype=U8)
w4, ws, idx = torch.zeros(DOUT, 32, dtype=U8), torch.zeros(DOUT, 2, dtype=U8), torch.zeros(N, K, dtype=U8)
b = torch.zeros(DOUT)

GOOD = {
    "quantize": lambda X=X, c=c8, s=s: maxk.maxk_mx_quantize(X, c, s),
    "dequantize": lambda c=c4, s=s, X=X: maxk.maxk_mx_dequantize(c, s, X),
    "linear": lambda c=c4, s=s, w=w4, ws=ws, Y=dH, b=b: maxk.maxk_mx_linear(c, s, w, ws, Y, b),
    "weight_grad": lambda c=c8, s=s, G=dH, dW=dW, db=b, room=None: maxk.maxk_mx_weight_grad(c, s, G, dW, db, room),
    "weight_grad_cbsr": lambda c=c4, s=s, G=dXs, idx=idx, dW=dW, db=b, room=None: maxk.maxk_mx_weight_grad_cbsr(c, s, G, idx, dW, db, room),
    "input_grad": lambda G=dH, w=w4, ws=ws, dX=X: maxk.maxk_mx_input_grad(G, w, ws, dX),
    "input_grad_cbsr": lambda G=dXs, idx=idx, w=w4, ws=ws, dX=X: maxk.maxk_mx_input_grad_cbsr(G, idx, w, ws, dX),
}

FIT, TYPE, MATRIX, INDEX, DENSE = r"do not fit \[", "expected float32, bfloat16 or float16", "expected a matrix", r"sp_index must be \[N, k\]", "expected a contiguous device tensor"
REFUSED = [
    ("quantize", dict(c=c8.float()), "codes must be int8 .8 bits. or uint8"), ("quantize", dict(c=c8[:, :40]), FIT), ("quantize", dict(s=s[:3]), FIT),
    ("quantize", dict(X=X[0]), MATRIX), ("quantize", dict(X=X[:3]), FIT), ("quantize", dict(X=X.double()), TYPE), ("quantize", dict(s=s.int()), DENSE),
    ("quantize", dict(X=X.t().contiguous().t()), DENSE),
    ("dequantize", dict(c=c4[:, :31]), FIT), ("dequantize", dict(X=torch.zeros(N, 65)), FIT), ("dequantize", dict(X=X.int()), TYPE), ("dequantize", dict(s=s.to(torch.int8)), DENSE),
    ("linear", dict(c=c8), "X: codes must be uint8 .4 bits."), ("linear", dict(w=torch.zeros(DOUT, 64, dtype=torch.int8)), "W: codes must be uint8 .4 bits."),
    ("linear", dict(w=w4[:, :16], ws=ws[:, :1]), "blocks do not match"), ("linear", dict(Y=torch.zeros(N, 9)), f"W: .*{FIT}"), ("linear", dict(Y=torch.zeros(5, DOUT)), f"X: .*{FIT}"),
    ("linear", dict(b=torch.zeros(9)), r"bias must be \[dout\]"), ("linear", dict(b=torch.zeros(1, DOUT)), r"bias must be \[dout\]"), ("linear", dict(b=b.half()), DENSE),
    ("linear", dict(Y=dH.double()), TYPE), ("linear", dict(Y=dH[0]), MATRIX),
    ("weight_grad", dict(G=dH[:3]), FIT), ("weight_grad", dict(G=dH[:, :7].contiguous()), r"dW / db must be \[dout, din\]"), ("weight_grad", dict(dW=dW.t()), FIT),
    ("weight_grad", dict(db=torch.zeros(7)), r"dW / db must be"), ("weight_grad", dict(G=dH.long()), TYPE), ("weight_grad", dict(dW=dW.half()), DENSE), ("weight_grad", dict(db=b.half()), DENSE),
    ("weight_grad", dict(room=torch.zeros(64)), DENSE), ("weight_grad", dict(c=c8.short()), "codes must be int8"), ("weight_grad", dict(G=dH[0]), MATRIX),
    ("weight_grad_cbsr", dict(idx=idx[:, :1]), INDEX), ("weight_grad_cbsr", dict(idx=idx.long()), INDEX), ("weight_grad_cbsr", dict(G=dXs[:3], idx=idx[:3]), FIT),
    ("weight_grad_cbsr", dict(G=dXs.half()), DENSE), ("weight_grad_cbsr", dict(db=torch.zeros(7)), r"dW / db must be"), ("weight_grad_cbsr", dict(dW=dW[0]), MATRIX),
    ("input_grad", dict(dX=X[:3]), r"dX must be \[N, din\]"), ("input_grad", dict(G=dH[:, :7]), FIT), ("input_grad", dict(w=w4[:7], ws=ws[:7]), FIT), ("input_grad", dict(ws=ws[:, :1]), FIT),
    ("input_grad", dict(w=torch.zeros(DOUT, 64, dtype=torch.int8)), "W: codes must be uint8"), ("input_grad", dict(G=dH.double()), TYPE), ("input_grad", dict(dX=X.double()), TYPE),
    ("input_grad_cbsr", dict(idx=idx[:3]), INDEX), ("input_grad_cbsr", dict(dX=X[:3]), r"dX must be \[N, din\]"), ("input_grad_cbsr", dict(ws=ws[:, :1]), FIT),
    ("input_grad_cbsr", dict(G=dXs.bfloat16()), DENSE), ("input_grad_cbsr", dict(w=w4[0]), MATRIX), ("input_grad_cbsr", dict(dX=X.int()), TYPE),
]


@pytest.mark.parametrize("name", GOOD)
def test_what_fits_is_made(name):
    with pytest.raises(_Made, match=f"maxk_mx_{name}$"):
        GOOD[name]()


@pytest.mark.parametrize("at", range(len(REFUSED)))
def test_what_does_not_fit_is_named(at):
    name, changed, message = REFUSED[at]
    with pytest.raises(maxk.MaxKError, match=message):
        GOOD[name](**changed)
