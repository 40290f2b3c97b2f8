"""The microscaled operators at row counts that send a workgroup round its loop several times, in every form that a call can take: each kind of
gradient and column index, whole and broken 16-byte rows, few and many kept columns, both formats.  Whole outputs against 64-bit sums on the device."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk
from test_gpu_mx import LAST, TYPES


def random_stored(gen, rows, din, bits, device="cuda"):
    """Any codes (zeros past din), scales over ten powers of two; and what they stand for, in 64 bits."""
    codes, scales = maxk.mx_empty(rows, din, bits, device)
    nb = scales.shape[1]
    scales.copy_(torch.randint(118, 128, scales.shape, generator=gen, device=device))
    if bits == 8:
        whole = torch.randint(-127, 128, (rows, nb * 32), generator=gen, device=device)
        whole[:, din:] = 0
        codes.copy_(whole)
        whole = whole.double() / 64
    else:
        nibbles = torch.randint(0, 16, (rows, nb * 32), generator=gen, device=device)
        nibbles[:, din:] = 0
        codes.copy_(nibbles[:, 0::2] + 16 * nibbles[:, 1::2])
        whole = torch.tensor([*mx.SIZES, *-mx.SIZES], dtype=torch.float64, device=device)[nibbles]
    unit = torch.exp2(scales.double() - 127)
    return codes, scales, (whole.reshape(rows, nb, 32) * unit.unsqueeze(2)).reshape(rows, -1)[:, :din].contiguous()


@pytest.mark.parametrize("bits", [8, 4])
def test_what_random_codes_stand_for(bits):
    codes, scales, values = random_stored(torch.Generator().manual_seed(1), 50, 100, bits, "cpu")
    np.testing.assert_array_equal(values.numpy(), mx.values(codes.numpy(), scales.numpy(), 100))


def close(got, want, terms, n_terms, kind="f32"):
    """The bound of the smaller tests: 8 + sqrt(n_terms) units of 2^-24 of the sum of |terms|, and one rounding to the type."""
    rel, tiny = LAST[kind]
    worst = (got.double() - want).abs() / ((8 + n_terms ** 0.5) * 2.0 ** -24 * terms + 1.001 * rel * want.abs() + tiny + 1e-37)
    assert got.shape == want.shape and bool((worst <= 1).all()), float(worst.nan_to_num(nan=float("inf")).max())  # (NaN is not <= 1)


def gradients(gen, N, dout, ks):
    """(what it is, the call's tensors, the dense matrix in 64 bits): dense in each type, CBSR of each k with each index that holds its columns."""
    size = 1e-3 * torch.exp(torch.randn(N, 1, generator=gen, device="cuda"))
    for kind, dtype in TYPES.items():
        dH = (torch.randn(N, dout, generator=gen, device="cuda") * size).to(dtype)
        yield kind, (dH,), dH.double()
    for k in ks:
        columns = torch.rand(N, dout, generator=gen, device="cuda").topk(k, dim=1).indices.sort(dim=1).values
        dXs = torch.randn(N, k, generator=gen, device="cuda") * size
        dense = torch.zeros(N, dout, dtype=torch.float64, device="cuda").scatter_(1, columns, dXs.double())
        for index in (torch.uint8, torch.int16, torch.int32):
            if index != torch.uint8 or dout <= 256:
                yield f"k={k} {index}", (dXs, columns.to(index)), dense


# widths of dH on both sides of what one tile, group or chunk holds; odd ones make rows that are not whole 16-byte pieces.  Rows: two tiles of 32 for each of up to 512
# workgroups are a round where dH is narrow, 256 of one tile where it is wide
@pytest.mark.gpu
@pytest.mark.parametrize("N,din,dout", [(100003, 100, 64), (100003, 128, 61), (50021, 300, 64), (50021, 260, 61), (100003, 100, 128), (100003, 90, 101), (50021, 256, 128),
                                        (50021, 255, 125), (50021, 128, 256), (50021, 127, 253), (50021, 256, 256), (50021, 200, 253), (30011, 256, 384), (30011, 131, 301),
                                        (30011, 256, 512), (30011, 300, 509), (30011, 256, 600), (30011, 301, 611)])
def test_input_gradients_of_several_rounds(N, din, dout):
    gen = torch.Generator(device="cuda").manual_seed(N + din + dout)
    codes, scales, W = random_stored(gen, dout, din, 4)
    for what, given, dH in gradients(gen, N, dout, [k for k in (13, 50, 100) if k <= dout]):
        want, terms = dH @ W, dH.abs() @ W.abs()
        for kind in ("f32", "bf16", "f16") if what == "f32" else ("f32",):
            dX = torch.full((N, din), float("nan"), dtype=TYPES[kind], device="cuda")
            (maxk.maxk_mx_input_grad_cbsr if len(given) == 2 else maxk.maxk_mx_input_grad)(*given, codes, scales, dX)
            close(dX, want, terms, dout, kind)


# tiles of dW of 64 x 64, 128 x 128 and 256 x 128 by width, with and without columns to spare
@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("N,din,dout", [(100003, 64, 64), (100003, 40, 61), (3001, 100, 100), (3001, 128, 128), (70001, 100, 100), (70001, 128, 128), (70001, 127, 101),
                                        (50021, 256, 256), (50021, 270, 200), (50021, 100, 253), (50021, 384, 384), (50021, 200, 301), (20011, 256, 512), (9001, 300, 516)])
def test_weight_gradients_of_several_rounds(N, din, dout, bits):
    gen = torch.Generator(device="cuda").manual_seed(N + din + dout + bits)
    codes, scales, X = random_stored(gen, N, din, bits)
    for what, given, dH in gradients(gen, N, dout, [k for k in (13, 50, 90) if k <= dout]):
        dW, db = torch.full((dout, din), float("nan"), device="cuda"), torch.full((dout,), float("nan"), device="cuda")
        (maxk.maxk_mx_weight_grad_cbsr if len(given) == 2 else maxk.maxk_mx_weight_grad)(codes, scales, *given, dW, db)
        close(dW, dH.t().contiguous() @ X, dH.abs().t().contiguous() @ X.abs(), N)
        close(db, dH.sum(0), dH.abs().sum(0), N)


# a product's widths in by what registers hold of a row (128, 256, 512, 1024 and more columns), its rows past and within L2, X past the Infinity Cache in the last two
@pytest.mark.gpu
@pytest.mark.parametrize("N,din,dout", [(200003, 100, 47), (200003, 128, 100), (200003, 100, 256), (200003, 200, 300), (9001, 200, 64), (200003, 256, 256), (100003, 500, 47),
                                        (100003, 512, 384), (100003, 300, 500), (9001, 512, 256), (100003, 1000, 100), (100003, 700, 320), (9001, 1024, 64), (50021, 1100, 100),
                                        (520003, 1024, 64), (520003, 1000, 47)])
def test_products_of_several_steps(N, din, dout):
    gen = torch.Generator(device="cuda").manual_seed(N + din + dout)
    xc, xs, X = random_stored(gen, N, din, 4)
    wc, ws, W = random_stored(gen, dout, din, 4)
    bias = torch.randn(dout, generator=gen, device="cuda")
    want, terms = X @ W.t().contiguous() + bias.double(), X.abs_() @ W.t().abs().contiguous() + bias.double().abs()
    for kind in ("f32", "bf16", "f16"):
        Y = torch.full((N, dout), float("nan"), dtype=TYPES[kind], device="cuda")
        maxk.maxk_mx_linear(xc, xs, wc, ws, Y, bias)
        close(Y, want, terms, din + 1, kind)


# rows of X of whole blocks, of whole 16-byte pieces and of neither, in each type and format: more than the units that a workgroup has under way
@pytest.mark.gpu
@pytest.mark.parametrize("din", [256, 100, 104, 99])
@pytest.mark.parametrize("bits", [8, 4])
def test_storage_of_many_rows(bits, din):
    gen = torch.Generator(device="cuda").manual_seed(din + bits)
    N = 20011
    for kind, dtype in TYPES.items():
        X = (torch.randn(N, din, generator=gen, device="cuda") * torch.exp(torch.randn(N, 1, generator=gen, device="cuda"))).to(dtype)
        want_codes, want_scales = mx.quantize(X.float().cpu().numpy(), bits)
        codes, scales = maxk.mx_empty(N, din, bits)
        maxk.maxk_mx_quantize(X, codes, scales)
        assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
        back = torch.full((N, din), float("nan"), dtype=dtype, device="cuda")
        maxk.maxk_mx_dequantize(codes, scales, back)
        want = torch.from_numpy(mx.values(want_codes, want_scales, din))
        assert torch.equal(back.cpu(), (want.float() if kind == "bf16" else want).to(dtype))
