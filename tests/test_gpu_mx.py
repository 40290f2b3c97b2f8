"""Microscaled storage, the 4-bit product and the gradients from it on the GPU, against plain 64-bit NumPy."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# one rounding to the type at the end: half a unit in the last place of a normal result, and of a subnormal fp16 one
LAST = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def check(got, want, terms, n_terms, kind="f32"):
    """fp32 sums of n_terms exact products in any order stray by at most (n_terms - 1) 2^-24 of the sum of |terms|, and by far less as
    rounding errors do not line up: 8 + sqrt(n_terms) units are allowed."""
    rel, tiny = LAST[kind]
    bound = (8 + np.sqrt(n_terms)) * 2.0 ** -24 * terms + 1.001 * rel * np.abs(want) + tiny + 1e-37
    worst = np.abs(got - want) / bound
    assert got.shape == want.shape and (worst <= 1).all(), f"worst error over bound {np.nanmax(worst)}, NaN: {np.isnan(got).sum()}"


def stored(X, bits):
    codes, scales = mx.quantize(X, bits)
    return codes, scales, dev(codes), dev(scales)


# ------------------------------------------------------------------ storage

SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (7, 64), (64, 100), (33, 256), (130, 257), (1000, 384), (2, 1433), (513, 48), (1, 4096)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_storage_is_exact(bits, kind):
    rng = np.random.default_rng(11)
    for N, din in SHAPES:
        X = dev(mx.features(rng, N, din, spread=0.5 if kind == "f16" else 3.0)).to(TYPES[kind])
        want_codes, want_scales = mx.quantize(X.float().cpu().numpy(), bits)
        codes, scales = maxk.mx_empty(N, din, bits)
        codes.fill_(77), scales.fill_(77)
        maxk.maxk_mx_quantize(X, codes, scales)
        np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)
        np.testing.assert_array_equal(codes.cpu().numpy(), want_codes)
        values = mx.values(want_codes, want_scales, din)
        for back in TYPES.values():
            out = torch.full((N, din), float("nan"), dtype=back, device="cuda")
            maxk.maxk_mx_dequantize(codes, scales, out)
            want = torch.from_numpy(values).to(back) if back != torch.bfloat16 else torch.from_numpy(values).float().to(back)
            assert torch.equal(out.cpu(), want), (N, din, back)


@pytest.mark.parametrize("bits", [8, 4])
def test_storage_of_every_exponent_and_of_non_finite_values(bits):
    rng = np.random.default_rng(12)
    rows = []
    for e in range(0, 256):
        pattern = (rng.integers(0, 2, 32).astype(np.uint32) << 31) | (rng.integers(max(e - 9, 0), e + 1, 32).astype(np.uint32) << 23) | \
            rng.integers(0, 1 << 23, 32).astype(np.uint32)
        rows.append(pattern.view(np.float32))
    # values on and next to the halfway points of the formats
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5], np.float32)
    rows.append(np.concatenate([grid, np.nextafter(grid, 0), np.nextafter(grid, 9), -grid]).astype(np.float32))
    rows.append(np.array([x for m in range(16) for x in ((m + 0.5) / 64, -(m + 64.5) / 64)], np.float32))
    rows += [np.zeros(32, np.float32), np.full(32, -0.0, np.float32)]
    for bad in (np.inf, -np.inf, np.nan):
        row = rng.standard_normal(32).astype(np.float32)
        row[17] = bad
        rows.append(row)
    X = np.stack(rows)
    want_codes, want_scales = mx.quantize(X, bits)
    codes, scales = maxk.mx_empty(len(rows), 32, bits)
    maxk.maxk_mx_quantize(dev(X), codes, scales)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)
    np.testing.assert_array_equal(codes.cpu().numpy(), want_codes)
    out = torch.empty(len(rows), 32, device="cuda")
    maxk.maxk_mx_dequantize(codes, scales, out)
    np.testing.assert_array_equal(out.cpu().numpy().astype(np.float64), mx.values(want_codes, want_scales, 32))


def test_storage_of_unaligned_rows():
    # a matrix that starts one element into its memory
    rng = np.random.default_rng(13)
    for kind, bits, din in (("f32", 8, 256), ("bf16", 4, 256), ("f16", 8, 64), ("f32", 4, 64)):
        X = dev(mx.features(rng, 40, din, 0.5)).to(TYPES[kind])
        shifted = torch.empty(40 * din + 1, dtype=X.dtype, device="cuda")[1:].view(40, din)
        shifted.copy_(X)
        a, b = maxk.mx_empty(40, din, bits), maxk.mx_empty(40, din, bits)
        maxk.maxk_mx_quantize(X, *a)
        maxk.maxk_mx_quantize(shifted, *b)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        maxk.maxk_mx_dequantize(*a, X)
        maxk.maxk_mx_dequantize(*a, shifted)
        assert torch.equal(X, shifted)


# ------------------------------------------------------------------ the product


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,din,dout", [(1, 1, 1), (1, 256, 256), (2, 32, 7), (15, 33, 17), (16, 128, 64), (17, 100, 47), (64, 64, 100), (100, 160, 256),
                                        (300, 256, 384), (1000, 384, 130), (33, 1000, 65), (40, 1433, 300), (5, 4100, 16), (4099, 96, 48)])
def test_linear(N, din, dout, kind):
    rng = np.random.default_rng(N + din + dout)
    x_codes, x_scales, xc, xs = stored(mx.features(rng, N, din), 4)
    w_codes, w_scales, wc, ws = stored(mx.features(rng, dout, din, 0.3) / np.sqrt(din), 4)
    X, W = mx.values(x_codes, x_scales, din), mx.values(w_codes, w_scales, din)
    for bias in (None, rng.standard_normal(dout).astype(np.float32)):
        Y = torch.full((N, dout), float("nan"), dtype=TYPES[kind], device="cuda")
        maxk.maxk_mx_linear(xc, xs, wc, ws, Y, None if bias is None else dev(bias))
        b = 0.0 if bias is None else bias.astype(np.float64)
        check(host(Y), X @ W.T + b, np.abs(X) @ np.abs(W).T + np.abs(b), din + 1, kind)


def test_linear_of_extreme_scales():
    # operands whose product is representable although one of them is near either end of the scale; a NaN block stays in its row
    rng = np.random.default_rng(21)
    X = mx.features(rng, 24, 128, 0.3)
    W = mx.features(rng, 32, 128, 0.3)
    for up, down in ((100, -100), (-110, 105), (120, -126), (0, -120)):
        x_codes, x_scales, xc, xs = stored(np.ldexp(X, up), 4)
        w_codes, w_scales, wc, ws = stored(np.ldexp(W, down), 4)
        Y = torch.empty(24, 32, device="cuda")
        maxk.maxk_mx_linear(xc, xs, wc, ws, Y)
        A, B = mx.values(x_codes, x_scales, 128), mx.values(w_codes, w_scales, 128)
        check(host(Y), A @ B.T, np.abs(A) @ np.abs(B).T, 128)
    X[5, 40] = np.nan
    x_codes, x_scales, xc, xs = stored(X, 4)
    w_codes, w_scales, wc, ws = stored(W, 4)
    Y = torch.empty(24, 32, device="cuda")
    maxk.maxk_mx_linear(xc, xs, wc, ws, Y)
    bad = np.isnan(host(Y))
    assert bad[5].all() and not np.delete(bad, 5, axis=0).any()


# ------------------------------------------------------------------ gradients

GRADS = [  # N, din, dout, k (0: dense)
    (1, 1, 1, 0), (1, 256, 256, 32), (3, 33, 17, 5), (31, 64, 64, 8), (33, 100, 47, 0), (64, 128, 130, 13), (100, 384, 384, 96), (257, 160, 256, 32),
    (1000, 256, 300, 0), (2500, 100, 100, 13), (5000, 40, 70, 70), (4097, 300, 20, 1), (70000, 64, 64, 16), (40, 1433, 513, 128), (20, 2000, 40, 0),
]


def gradient(rng, N, dout, k, kind, index=np.int32):
    """(device tensors of the call, the dense matrix they stand for)."""
    size = 1e-3 * np.exp(rng.standard_normal((N, 1)))
    if k:
        dXs = (rng.standard_normal((N, k)) * size).astype(np.float32)
        cols = mx.columns(rng, N, dout, k)
        return (dev(dXs), dev(cols.astype(index))), mx.scatter(dXs, cols, dout)
    dH = dev((rng.standard_normal((N, dout)) * size).astype(np.float32)).to(TYPES[kind])
    return (dH,), host(dH)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,din,dout,k", GRADS)
def test_weight_grad(N, din, dout, k, kind, bits):
    if k and kind != "f32":
        pytest.skip("a CBSR gradient is fp32")
    rng = np.random.default_rng(N + din + dout + k + bits)
    codes, scales, c, s = stored(mx.features(rng, N, din), bits)
    X = mx.values(codes, scales, din)
    for index in (np.uint8, np.int16, np.int32) if k else (None,):
        if index == np.uint8 and dout > 256:
            continue
        given, dH = gradient(rng, N, dout, k, kind, index)
        dW = torch.full((dout, din), float("nan"), device="cuda")
        db = torch.full((dout,), float("nan"), device="cuda")
        call = maxk.maxk_mx_weight_grad_cbsr if k else maxk.maxk_mx_weight_grad
        call(c, s, *given, dW, db)
        check(host(dW), dH.T @ X, np.abs(dH).T @ np.abs(X), N)
        check(host(db), dH.sum(axis=0), np.abs(dH).sum(axis=0), N)
        again = torch.empty_like(dW)
        room = torch.empty(maxk.mx_weight_grad_workspace(N, din, dout), dtype=torch.uint8, device="cuda").fill_(255)  # NaN in fp32
        call(c, s, *given, again, None, room)
        assert torch.equal(again, dW)  # the same bits, whatever the workspace held


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,din,dout,k", GRADS)
def test_input_grad(N, din, dout, k, kind):
    rng = np.random.default_rng(N + din + dout + k)
    codes, scales, c, s = stored(mx.features(rng, dout, din, 0.3) / np.sqrt(din), 4)
    W = mx.values(codes, scales, din)
    for index in (np.uint8, np.int16, np.int32) if k else (None,):
        if index == np.uint8 and dout > 256:
            continue
        given, dH = gradient(rng, N, dout, k, kind, index)
        for out in ("f32", kind):
            dX = torch.full((N, din), float("nan"), dtype=TYPES[out], device="cuda")
            (maxk.maxk_mx_input_grad_cbsr if k else maxk.maxk_mx_input_grad)(*given, c, s, dX)
            check(host(dX), dH @ W, np.abs(dH) @ np.abs(W), k or dout, out)


def test_gradients_of_exact_sums_are_exact():
    # whole numbers whose sums stay below 2^24: every order gives the same, and nothing of a 24-bit value may be lost
    rng = np.random.default_rng(31)
    N, din, dout = 37, 64, 96
    X = rng.integers(-1, 2, (N, din)).astype(np.float32)
    for k in (0, 1):
        dH = np.zeros((N, dout), np.float32)
        cols = rng.integers(0, dout, (N, 1))
        np.put_along_axis(dH, cols, rng.integers(-2 ** 18, 2 ** 18, (N, 1)).astype(np.float32), axis=1)
        for bits in (8, 4):
            codes, scales, c, s = stored(X, bits)
            np.testing.assert_array_equal(mx.values(codes, scales, din), X)
            dW, db = torch.empty(dout, din, device="cuda"), torch.empty(dout, device="cuda")
            if k:
                maxk.maxk_mx_weight_grad_cbsr(c, s, dev(np.take_along_axis(dH, cols, 1)), dev(cols.astype(np.uint8)), dW, db)
            else:
                maxk.maxk_mx_weight_grad(c, s, dev(dH), dW, db)
            np.testing.assert_array_equal(host(dW), dH.T.astype(np.float64) @ X)
            np.testing.assert_array_equal(host(db), dH.sum(axis=0, dtype=np.float64))


def test_no_rows():
    dW, db = torch.full((5, 40), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda")
    for bits in (8, 4):
        codes, scales = maxk.mx_empty(0, 40, bits)
        maxk.maxk_mx_quantize(torch.empty(0, 40, device="cuda"), codes, scales)
        maxk.maxk_mx_dequantize(codes, scales, torch.empty(0, 40, device="cuda"))
        dW.fill_(3.0), db.fill_(3.0)
        maxk.maxk_mx_weight_grad(codes, scales, torch.empty(0, 5, device="cuda"), dW, db)
        assert not dW.any() and not db.any()
        dW.fill_(3.0), db.fill_(3.0)
        maxk.maxk_mx_weight_grad_cbsr(codes, scales, torch.empty(0, 2, device="cuda"), torch.empty(0, 2, dtype=torch.uint8, device="cuda"), dW, db)
        assert not dW.any() and not db.any()
    w = maxk.mx_empty(5, 40, 4)
    maxk.maxk_mx_linear(codes, scales, *w, torch.empty(0, 5, device="cuda"))
    maxk.maxk_mx_input_grad(torch.empty(0, 5, device="cuda"), *w, torch.empty(0, 40, device="cuda"))


def test_outputs_end_where_they_end():
    # rows and columns around every tile edge: what lies behind an output stays
    rng = np.random.default_rng(41)
    for N, din, dout in ((1, 33, 5), (17, 100, 65), (129, 130, 129), (300, 257, 31)):
        codes, scales, c, s = stored(mx.features(rng, N, din), 4)
        w = stored(mx.features(rng, dout, din, 0.3), 4)[2:]
        dH = dev(rng.standard_normal((N, dout)).astype(np.float32))

        def guarded(rows, cols, dtype=torch.float32):
            room = torch.full((rows * cols + 4096,), 7.0, device="cuda").to(dtype)
            return room, room[:rows * cols].view(rows, cols)

        for (room, out), call in ((guarded(N, dout), lambda Y: maxk.maxk_mx_linear(c, s, *w, Y)),
                                  (guarded(N, dout, torch.bfloat16), lambda Y: maxk.maxk_mx_linear(c, s, *w, Y)),
                                  (guarded(dout, din), lambda dW: maxk.maxk_mx_weight_grad(c, s, dH, dW)),
                                  (guarded(N, din), lambda dX: maxk.maxk_mx_input_grad(dH, *w, dX)),
                                  (guarded(N, din, torch.float16), lambda dX: maxk.maxk_mx_input_grad(dH, *w, dX)),
                                  (guarded(N, din), lambda X: maxk.maxk_mx_dequantize(c, s, X))):
            call(out)
            assert bool((room[out.numel():] == 7).all())
        room = torch.full((c.numel() + 4096,), 7, dtype=torch.uint8, device="cuda")
        marks = torch.full((s.numel() + 4096,), 7, dtype=torch.uint8, device="cuda")
        maxk.maxk_mx_quantize(dev(mx.features(rng, N, din)), room[:c.numel()].view(c.shape), marks[:s.numel()].view(s.shape))
        assert bool((room[c.numel():] == 7).all()) and bool((marks[s.numel():] == 7).all())


def test_offsets_past_32_bits():
    # 2.2 billion elements: rows at either end and around 2^31 and 2^32 bytes
    N, din = 4_300_000, 512
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    gen = torch.Generator(device="cuda").manual_seed(5)
    X = torch.randn(N, din, generator=gen, device="cuda").to(torch.bfloat16)
    pick = torch.tensor([0, 1, 2 ** 20 - 1, 2 ** 21, 2 ** 21 + 1, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, N - 2, N - 1], device="cuda")
    few = X[pick].contiguous()
    w = maxk.mx_empty(256, din, 4)
    maxk.maxk_mx_quantize(torch.randn(256, din, generator=gen, device="cuda"), *w)
    for bits in (8, 4):
        big, small = maxk.mx_empty(N, din, bits), maxk.mx_empty(10, din, bits)
        maxk.maxk_mx_quantize(X, *big)
        maxk.maxk_mx_quantize(few, *small)
        assert torch.equal(big[0][pick], small[0]) and torch.equal(big[1][pick], small[1])
        X2, few2 = torch.empty_like(X), torch.empty_like(few)
        maxk.maxk_mx_dequantize(*big, X2)
        maxk.maxk_mx_dequantize(*small, few2)
        assert torch.equal(X2[pick], few2)
        del X2
    Y, fewY = torch.empty(N, 256, device="cuda"), torch.empty(10, 256, device="cuda")
    maxk.maxk_mx_linear(*big, *w, Y)
    maxk.maxk_mx_linear(*small, *w, fewY)
    torch.testing.assert_close(Y[pick], fewY, rtol=1e-5, atol=1e-4)
    maxk.maxk_mx_input_grad(Y, *w, X)
    maxk.maxk_mx_input_grad(fewY, *w, few)
    torch.testing.assert_close(X[pick].float(), few.float(), rtol=1e-2, atol=1e-2)
    # rows of zeros everywhere but at the picks: the weight gradient is that of the picks
    kept = Y[pick].clone()
    Y.zero_()
    Y[pick] = kept
    dW, fewdW = torch.empty(256, din, device="cuda"), torch.empty(256, din, device="cuda")
    maxk.maxk_mx_weight_grad(*big, Y, dW)
    maxk.maxk_mx_weight_grad(*small, kept, fewdW)
    torch.testing.assert_close(dW, fewdW, rtol=1e-4, atol=1e-3 * float(fewdW.abs().max()))


def test_other_streams_and_graph_replays():
    rng = np.random.default_rng(51)
    N, din, dout, k = 3000, 96, 80, 8
    X = dev(mx.features(rng, N, din))
    (dXs, cols), _ = gradient(rng, N, dout, k, "f32", np.uint8)
    w = maxk.mx_empty(dout, din, 4)
    maxk.maxk_mx_quantize(dev(mx.features(rng, dout, din, 0.3)), *w)
    stored8, stored4 = maxk.mx_empty(N, din, 8), maxk.mx_empty(N, din, 4)
    outs = [torch.empty(N, dout, device="cuda"), torch.empty(dout, din, device="cuda"), torch.empty(dout, device="cuda"), torch.empty(N, din, device="cuda"),
            torch.empty(N, din, device="cuda")]
    room = torch.empty(maxk.mx_weight_grad_workspace(N, din, dout), dtype=torch.uint8, device="cuda")

    def step():
        maxk.maxk_mx_quantize(X, *stored8)
        maxk.maxk_mx_quantize(X, *stored4)
        maxk.maxk_mx_linear(*stored4, *w, outs[0])
        maxk.maxk_mx_weight_grad_cbsr(*stored8, dXs, cols, outs[1], outs[2], room)
        maxk.maxk_mx_input_grad_cbsr(dXs, cols, *w, outs[3])
        maxk.maxk_mx_dequantize(*stored8, outs[4])

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for t in outs:
        t.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        X.mul_(-2.0)  # other inputs each time, and eager work in between
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs + [room.view(torch.float32)]:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), replay


def test_differences_of_a_loss():
    # a loss L = sum(C * (X W^T)): moving one entry of W by h moves it by h dW[o,i], one of X by h dX[n,i]
    rng = np.random.default_rng(61)
    N, din, dout = 50, 64, 40
    X, W = rng.integers(-2, 3, (N, din)).astype(np.float32), rng.integers(-2, 3, (dout, din)).astype(np.float32)
    C = rng.integers(-8, 9, (N, dout)).astype(np.float32)
    x, w = stored(X, 4)[2:], stored(W, 4)[2:]

    def loss(X, W):
        Y = torch.empty(N, dout, device="cuda")
        maxk.maxk_mx_linear(*stored(X, 4)[2:], *stored(W, 4)[2:], Y)
        return float((Y.double() * dev(C)).sum())

    dW, dX = torch.empty(dout, din, device="cuda"), torch.empty(N, din, device="cuda")
    maxk.maxk_mx_weight_grad(*x, dev(C), dW)
    maxk.maxk_mx_input_grad(dev(C), *w, dX)
    base = loss(X, W)
    for _ in range(6):
        for A, grad, which in ((X, dX, 0), (W, dW, 1)):
            r, c = rng.integers(A.shape[0]), rng.integers(A.shape[1])
            B = A.copy()
            B[r, c] += 1 if B[r, c] < 2 else -1  # a value that the format holds
            moved = loss(B, W) if which == 0 else loss(X, B)
            assert moved - base == (B[r, c] - A[r, c]) * float(grad[r, c])  # whole numbers: exact
