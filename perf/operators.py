"""The measured work: the linear half of a MaxK-GNN layer on microscaled storage, as a training or serving program calls it.

A layer is ``Y = A * MaxK_k(X W^T + b)``.  Full-batch training keeps X [N, din] for the weight gradient, so it is stored in blocks of 32
columns with one power-of-two scale a block: 8-bit integers (MX8) or 4-bit floating point (MX4, E2M1), which also carries the product.
The gradient that comes back from the aggregation is a CBSR (k values and columns a row) or, where nothing was cut, a dense matrix.

``path`` says which call a pass is:

* ``store``   X into codes and scales, and back to X's type (a checkpoint written and read);
* ``linear``  Y = X^ W^^T + b of MX4 operands;
* ``wgrad``   dW = dH^T X^ and db = column sums of dH, from a checkpoint of 8 or 4 bits;
* ``igrad``   dX = dH W^ of MX4 weights.

Layouts: codes are int8 [N, 32 nb] (MX8) or uint8 [N, 16 nb] (MX4, the even column in the low half byte), scales uint8 [N, nb], with
nb = ceil(din / 32) and zeros in the columns past din.
"""
from __future__ import annotations

import math

import torch

own = False

_FIELDS = ("name", "path", "N", "din", "dout", "k", "bits", "value")


def _case(*values):
    # k: kept columns a row of the gradient (0: a dense gradient); value: type of X and the restored X, of Y, of a dense dH, of dX
    return dict(zip(_FIELDS, values))


def listed():
    return [
        # a checkpoint of a thousand nodes: launches are all there is
        _case("tiny_store8", "store", 1024, 64, 0, 0, 8, "f32"),
        # hidden width 100: a last block of four columns, rows that are not whole 16-byte units in any format
        _case("ragged_store4", "store", 40013, 100, 0, 0, 4, "f32"),
        # the largest checkpoint of a mixed-precision run: hidden width 384 on 717 thousand nodes
        _case("wide_store8_bf16", "store", 716847, 384, 0, 0, 8, "bf16"),
        # serving: one node's features through a layer
        _case("one_row_linear", "linear", 1, 256, 256, 0, 4, "f32"),
        # input features of width 100 to a last layer of 47 classes
        _case("ragged_linear", "linear", 40013, 100, 47, 0, 4, "f32"),
        # inference on the largest graph
        _case("large_linear", "linear", 2449029, 256, 256, 0, 4, "f32"),
        # training steps: a thousand nodes; the headline graph at the k the paper recommends; a layer that nothing was cut in,
        # 16-bit gradients, from a 4-bit checkpoint
        _case("tiny_wgrad_k8", "wgrad", 1024, 64, 64, 8, 8, "f32"),
        _case("dense_wgrad_k32", "wgrad", 232965, 256, 256, 32, 8, "f32"),
        _case("wide_wgrad_bf16", "wgrad", 716847, 384, 384, 0, 4, "bf16"),
        # gradients of the inputs: ragged widths and odd k, the headline graph, and a dense fp32 gradient on a citation graph
        _case("ragged_igrad_k13", "igrad", 40013, 100, 100, 13, 4, "f32"),
        _case("dense_igrad_k32", "igrad", 232965, 256, 256, 32, 4, "f32"),
        _case("sparse_mid_igrad", "igrad", 169343, 256, 256, 0, 4, "f32"),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 2.4 million rows, widths 16 to 1024 in and 16 to 512 out, any k, each type."""
    while True:
        path = rng.choice(["store", "linear", "wgrad", "wgrad", "igrad"])
        N = int(round(math.exp(rng.uniform(0.0, math.log(2449029)))))
        if path == "store":
            N = max(N, 33)
        din = rng.choice([64, 100, 128, 256, 256, 384, 512, rng.randint(16, 1024), rng.randint(16, 1024)])
        dout = 0 if path == "store" else rng.choice([64, 128, 256, 256, 384, rng.randint(16, 512), rng.randint(16, 512)])
        k = 0
        if path in ("wgrad", "igrad") and rng.random() < 0.6:
            k = rng.choice([8, 16, 32, 32, 64, 96, rng.randint(1, 128)])
            if k > dout // 2:
                continue
        bits = 4 if path in ("linear", "igrad") else rng.choice([8, 8, 4])
        value = "f32" if k else rng.choice(["f32", "f32", "bf16", "f16"])
        if N * (din + max(dout, din)) > 2449029 * 512 or N * din * max(dout, 1) > 2449029 * 256 * 256:
            continue
        case = _case("", path, N, din, dout, k, bits, value)
        del case["name"]
        return case


# ------------------------------------------------------------------ inputs

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _features(N, din, seed):
    """Hidden features: N(0,1) with a spread from row to row (degrees) and from column to column, a few rows of zeros."""
    gen = _generator(seed)
    X = torch.randn(N, din, generator=gen, device="cuda")
    X *= torch.exp(0.5 * torch.randn(N, 1, generator=gen, device="cuda"))
    X *= torch.exp(0.3 * torch.randn(1, din, generator=gen, device="cuda"))
    if N > 64:
        X[torch.randint(N, (max(1, N // 200),), generator=gen, device="cuda")] = 0.0
    return X


def _weights(dout, din, seed):
    gen = _generator(seed)
    return (torch.rand(dout, din, generator=gen, device="cuda") * 2.0 - 1.0) / math.sqrt(din)


def _gradient(N, width, seed):
    """Gradients: small, their size spread over the rows."""
    gen = _generator(seed)
    return torch.randn(N, width, generator=gen, device="cuda") * (1e-3 * torch.exp(torch.randn(N, 1, generator=gen, device="cuda")))


def _kept(N, dout, k, seed):
    """k distinct ascending columns a row."""
    gen = _generator(seed)
    index = torch.empty(N, k, dtype=torch.uint8 if dout <= 256 else torch.int16, device="cuda")
    for i in range(0, N, 1 << 19):
        rows = min(1 << 19, N - i)
        keys = torch.rand(rows, dout, generator=gen, device="cuda")
        index[i:i + rows] = keys.topk(k, dim=1).indices.sort(dim=1).values.to(index.dtype)
    return index


def _blocks(X):
    """X as [N, nb, 32], zeros past its last column."""
    N, din = X.shape
    nb = (din + 31) // 32
    if din != nb * 32:
        X = torch.nn.functional.pad(X, (0, nb * 32 - din))
    return X.reshape(N, nb, 32)


def _times_power(x, e):
    """x * 2^e for whole e, in two steps so that neither power leaves the fp32 range."""
    half = torch.div(e, 2, rounding_mode="floor")
    return x * torch.exp2(half.float()) * torch.exp2((e - half).float())


def _quantise(X, bits):
    """(multiples q of the block's unit, exponent byte s): the value is q 2^(s-133) (8 bits) or q 2^(s-127) (4 bits)."""
    B = _blocks(X.float())
    amax = B.abs().amax(dim=2, keepdim=True)
    field = torch.where(amax > 0, (torch.frexp(amax).exponent.int() + 126).clamp_min(0), torch.zeros_like(amax, dtype=torch.int32))
    if bits == 8:
        q = torch.round(_times_power(B, 133 - field)).clamp_(-127.0, 127.0)
        return q, field.squeeze(2)
    field = (field - 2).clamp_min(0)
    y = _times_power(B, 127 - field)
    a = y.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), y), field.squeeze(2)


def _encode(X, bits):
    """Codes and scales as the calls take them."""
    N, parts = X.shape[0], []
    for i in range(0, N, 1 << 19):
        q, s = _quantise(X[i:i + (1 << 19)], bits)
        q = q.reshape(q.shape[0], -1)
        if bits == 8:
            codes = q.to(torch.int8)
        else:
            grid = torch.tensor(_E2M1, device="cuda")
            code = torch.searchsorted(grid, q.abs()).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
            codes = code[:, 0::2] | (code[:, 1::2] << 4)
        parts.append((codes, s.to(torch.uint8)))
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def prepare(case, seed):
    path, N, din, dout, k, bits = (case[f] for f in ("path", "N", "din", "dout", "k", "bits"))
    dtype = _DTYPE[case["value"]]
    state = {"case": case}
    if path == "store":
        state["X"] = _features(N, din, seed * 5 + 1).to(dtype)
        nb = (din + 31) // 32
        state["codes"] = torch.empty(N, nb * (32 if bits == 8 else 16), dtype=torch.int8 if bits == 8 else torch.uint8, device="cuda")
        state["scales"] = torch.empty(N, nb, dtype=torch.uint8, device="cuda")
        state["restored"] = torch.empty(N, din, dtype=dtype, device="cuda")
    if path in ("linear", "wgrad"):
        state["codes"], state["scales"] = _encode(_features(N, din, seed * 5 + 1), bits)
    if path in ("linear", "igrad"):
        state["W_codes"], state["W_scales"] = _encode(_weights(dout, din, seed * 5 + 2), 4)
    if path == "linear":
        state["bias"] = 0.1 * torch.randn(dout, generator=_generator(seed * 5 + 3), device="cuda")
        state["Y"] = torch.empty(N, dout, dtype=dtype, device="cuda")
    if path in ("wgrad", "igrad"):
        if k:
            state["dXs"] = _gradient(N, k, seed * 5 + 3)
            state["sp_index"] = _kept(N, dout, k, seed * 5 + 4)
        else:
            state["dH"] = _gradient(N, dout, seed * 5 + 3).to(dtype)
    if path == "wgrad":
        state["dW"] = torch.empty(dout, din, device="cuda")
        state["db"] = torch.empty(dout, device="cuda")
    if path == "igrad":
        state["dX"] = torch.empty(N, din, dtype=dtype, device="cuda")
    torch.cuda.empty_cache()
    return state


# ------------------------------------------------------------------ one pass


def _decode(codes, scales, bits, din):
    """fp32 values [N, din] of codes and scales."""
    N, nb = scales.shape
    if bits == 8:
        q = codes.float()
    else:
        grid = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
        q = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], dim=2)
    unit = torch.exp2(scales.float() - (133.0 if bits == 8 else 127.0))
    return (q.reshape(N, nb, 32) * unit.unsqueeze(2)).reshape(N, nb * 32)[:, :din]


def _dense_gradient(state):
    case = state["case"]
    if not case["k"]:
        return state["dH"].float()
    columns = state["sp_index"].long()
    dH = torch.zeros(case["N"], case["dout"], device="cuda")
    return dH.scatter_(1, columns, state["dXs"])


def _run_plain(state):
    case = state["case"]
    path, N, din, bits, dtype = case["path"], case["N"], case["din"], case["bits"], _DTYPE[case["value"]]
    if path == "store":
        q, field = _quantise(state["X"], bits)
        X = _times_power(q, field.unsqueeze(2) - (133 if bits == 8 else 127)).reshape(N, -1)[:, :din]
        return {"X": X.to(dtype), "scales": field.to(torch.uint8)}
    if path == "linear":
        X = _decode(state["codes"], state["scales"], 4, din)
        W = _decode(state["W_codes"], state["W_scales"], 4, din)
        return {"Y": (torch.mm(X, W.t()) + state["bias"]).to(dtype)}
    dH = _dense_gradient(state)
    if path == "wgrad":
        X = _decode(state["codes"], state["scales"], bits, din)
        return {"dW": torch.mm(dH.t(), X), "db": dH.sum(dim=0)}
    return {"dX": torch.mm(dH, _decode(state["W_codes"], state["W_scales"], 4, din)).to(dtype)}


def _run_own(state):
    import paper_2312_08656_amd as maxk

    case = state["case"]
    path, k = case["path"], case["k"]
    if path == "store":
        maxk.maxk_mx_quantize(state["X"], state["codes"], state["scales"])
        maxk.maxk_mx_dequantize(state["codes"], state["scales"], state["restored"])
        return {"X": state["restored"], "scales": state["scales"]}
    if path == "linear":
        maxk.maxk_mx_linear(state["codes"], state["scales"], state["W_codes"], state["W_scales"], state["Y"], bias=state["bias"])
        return {"Y": state["Y"]}
    if path == "wgrad":
        if k:
            maxk.maxk_mx_weight_grad_cbsr(state["codes"], state["scales"], state["dXs"], state["sp_index"], state["dW"], state["db"])
        else:
            maxk.maxk_mx_weight_grad(state["codes"], state["scales"], state["dH"], state["dW"], state["db"])
        return {"dW": state["dW"], "db": state["db"]}
    if k:
        maxk.maxk_mx_input_grad_cbsr(state["dXs"], state["sp_index"], state["W_codes"], state["W_scales"], state["dX"])
    else:
        maxk.maxk_mx_input_grad(state["dH"], state["W_codes"], state["W_scales"], state["dX"])
    return {"dX": state["dX"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once, each output written once; products of kept columns only."""
    path, N, din, dout, k, bits = (case[f] for f in ("path", "N", "din", "dout", "k", "bits"))
    vb = 4 if case["value"] == "f32" else 2
    nb = (din + 31) // 32
    code = 33 if bits == 8 else 17  # bytes of a block and its scale
    gradient = N * k * (4 + (1 if dout <= 256 else 2)) if k else N * dout * vb
    if path == "store":
        return {"bytes": 2 * N * din * vb + 2 * N * nb * code, "flops": 2 * N * din}
    if path == "linear":
        return {"bytes": (N + dout) * nb * 17 + 4 * dout + N * dout * vb, "flops": 2 * N * din * dout}
    if path == "wgrad":
        return {"bytes": N * nb * code + gradient + 4 * dout * (din + 1), "flops": 2 * N * (k or dout) * din}
    return {"bytes": dout * nb * 17 + gradient + N * din * vb, "flops": 2 * N * (k or dout) * din}


# ------------------------------------------------------------------ the definition in 64 bits


def _exact_values(codes, scales, bits, din):
    """What stored codes stand for, one code at a time from the format's table."""
    if bits == 8:
        whole = codes.double() / 64.0
    else:
        table = []
        for pattern in range(16):
            exponent, last = (pattern >> 1) & 3, pattern & 1
            size = 0.5 * last if exponent == 0 else (1.0 + 0.5 * last) * 2.0 ** (exponent - 1)
            table.append(-size if pattern & 8 else size)
        table = torch.tensor(table, dtype=torch.float64, device=codes.device)
        whole = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
        whole[:, 0::2] = table[(codes % 16).long()]
        whole[:, 1::2] = table[torch.div(codes, 16, rounding_mode="floor").long()]
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=codes.device), scales.double() - 127.0)
    return (whole * power.repeat_interleave(32, dim=1))[:, :din]


def _exact_stored(X, bits):
    """Nearest stored values of X, block by block, ties to the even code."""
    N, din = X.shape
    values = torch.empty(N, din, dtype=torch.float64, device=X.device)
    scales = torch.empty(N, (din + 31) // 32, dtype=torch.uint8, device=X.device)
    sizes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=X.device)
    for b in range(0, din, 32):
        part = X[:, b:b + 32].double()
        top = part.abs().max(dim=1).values
        exponent = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
        exponent = torch.where(top > 0, exponent, torch.full_like(top, -200.0)) - (0.0 if bits == 8 else 2.0)
        exponent = exponent.clamp(min=-127.0)
        unit = torch.pow(2.0, exponent).unsqueeze(1)
        if bits == 8:
            values[:, b:b + 32] = torch.round(part / unit * 64.0).clamp(-127, 127) / 64.0 * unit
        else:
            ratio = (part / unit).abs().clamp(max=6.0)
            upper = torch.searchsorted(sizes, ratio.contiguous()).clamp(max=7)
            lower = (upper - 1).clamp(min=0)
            below, above = ratio - sizes[lower], sizes[upper] - ratio
            code = torch.where((below < above) | ((below == above) & (lower % 2 == 0)), lower, upper)
            values[:, b:b + 32] = sizes[code] * torch.sign(part) * unit
        scales[:, b // 32] = (exponent + 127.0).to(torch.uint8)
    return values, scales


def exact(case, seed):
    state = prepare(case, seed)
    path, N, din, dout, k, bits = (case[f] for f in ("path", "N", "din", "dout", "k", "bits"))
    if path == "store":
        values, scales = _exact_stored(state["X"], bits)
        return {"X": values, "scales": scales}
    if path == "linear":
        Y = _exact_values(state["codes"], state["scales"], 4, din) @ _exact_values(state["W_codes"], state["W_scales"], 4, din).t().contiguous()
        return {"Y": Y + state["bias"].double()}
    if k:
        dH = torch.zeros(N * dout, dtype=torch.float64, device="cuda")
        at = torch.arange(N, device="cuda").unsqueeze(1) * dout + state["sp_index"].long()
        dH[at.reshape(-1)] = state["dXs"].double().reshape(-1)
        dH = dH.reshape(N, dout)
    else:
        dH = state["dH"].double()
    if path == "wgrad":
        return {"dW": dH.t().contiguous() @ _exact_values(state["codes"], state["scales"], bits, din), "db": dH.sum(dim=0)}
    return {"dX": dH @ _exact_values(state["W_codes"], state["W_scales"], 4, din)}
