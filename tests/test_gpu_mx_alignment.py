"""Operands of the microscaled calls that begin one element into their memory: the same values, through accesses that need no more than an element's alignment."""
import pytest
import torch

import paper_2312_08656_amd as maxk
from test_gpu_mx import TYPES
from test_gpu_mx_instances import close, gradients, random_stored

pytestmark = pytest.mark.gpu

N, DIN, DOUT = 3001, 256, 128


def shifted(t, fill=None):
    """A copy of t one element into its memory, and the element before it and those behind it, which must stay."""
    room = torch.full((t.numel() + 65,), 9, dtype=t.dtype, device="cuda")
    view = room[1:1 + t.numel()].view(t.shape)
    view.copy_(t) if fill is None else view.fill_(fill)
    return view, room


def untouched(view, room):
    return bool((room[:1] == 9).all()) and bool((room[1 + view.numel():] == 9).all())


@pytest.mark.parametrize("kind", TYPES)
def test_product(kind):
    gen = torch.Generator(device="cuda").manual_seed(1)
    xc, xs, X = random_stored(gen, N, DIN, 4)
    wc, ws, W = random_stored(gen, DOUT, DIN, 4)
    bias = torch.randn(DOUT, generator=gen, device="cuda")
    Y, room = shifted(torch.empty(N, DOUT, dtype=TYPES[kind], device="cuda"), float("nan"))
    maxk.maxk_mx_linear(xc, shifted(xs)[0], wc, shifted(ws)[0], Y, shifted(bias)[0])
    close(Y, X @ W.t().contiguous() + bias.double(), X.abs() @ W.t().abs().contiguous() + bias.double().abs(), DIN + 1, kind)
    assert untouched(Y, room)


@pytest.mark.parametrize("bits", [8, 4])
def test_gradients(bits):
    gen = torch.Generator(device="cuda").manual_seed(2 + bits)
    codes, scales, X = random_stored(gen, N, DIN, bits)
    wc, ws, W = random_stored(gen, DOUT, DIN, 4)
    scales, ws = shifted(scales)[0], shifted(ws)[0]
    for what, given, dH in gradients(gen, N, DOUT, [13, 50]):
        given = [shifted(t)[0] for t in given]
        cbsr = len(given) == 2
        (dW, dW_room), (db, db_room) = shifted(torch.empty(DOUT, DIN, device="cuda"), float("nan")), shifted(torch.empty(DOUT, device="cuda"), float("nan"))
        (maxk.maxk_mx_weight_grad_cbsr if cbsr else maxk.maxk_mx_weight_grad)(codes, scales, *given, dW, db)
        close(dW, dH.t().contiguous() @ X, dH.abs().t().contiguous() @ X.abs(), N)
        close(db, dH.sum(0), dH.abs().sum(0), N)
        for kind, dtype in TYPES.items():
            dX, dX_room = shifted(torch.empty(N, DIN, dtype=dtype, device="cuda"), float("nan"))
            (maxk.maxk_mx_input_grad_cbsr if cbsr else maxk.maxk_mx_input_grad)(*given, wc, ws, dX)
            close(dX, dH @ W, dH.abs() @ W.abs(), DOUT, kind)
            assert untouched(dX, dX_room)
        assert untouched(dW, dW_room) and untouched(db, db_room)


def test_a_workspace_within_another():
    gen = torch.Generator(device="cuda").manual_seed(5)
    codes, scales, X = random_stored(gen, N, DIN, 8)
    dH = torch.randn(N, DOUT, generator=gen, device="cuda")
    need = maxk.mx_weight_grad_workspace(N, DIN, DOUT)
    room = torch.full((need + 32,), 9, dtype=torch.uint8, device="cuda")
    dW, again = torch.empty(DOUT, DIN, device="cuda"), torch.empty(DOUT, DIN, device="cuda")
    maxk.maxk_mx_weight_grad(codes, scales, dH, dW)
    maxk.maxk_mx_weight_grad(codes, scales, dH, again, None, room[16:16 + need])
    assert torch.equal(dW, again) and bool((room[:16] == 9).all()) and bool((room[16 + need:] == 9).all())
    for bad in (room[1:1 + need], room[16:15 + need]):
        with pytest.raises(maxk.MaxKError):
            maxk.maxk_mx_weight_grad(codes, scales, dH, again, None, bad)
