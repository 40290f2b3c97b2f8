"""The measured work: both ends of a classifier, as a training or serving program calls them.

In front of a layer stands a root-mean-square norm with the residual's addition, whose output the layer keeps in 8 or 4 bits; behind the last
one stand the product with its weights, the classes' log probabilities and the loss that teaches them.

``path`` says which call a pass is:

* ``norm``       H = X + residual, Y = H r gamma with r = 1 / sqrt(mean of H^2 + eps), Y in its type or as codes and scales, read back;
* ``norm_step``  the same and its gradients: dX from dY and the gradient that arrives at H, dgamma;
* ``score``      of each row of logits the log probability of a given class, the entropy and the k likeliest classes;
* ``learn``      log probabilities and entropies, and the logits' gradient of their weighted sum;
* ``distill``    the divergence of softmax(logits / T) from a teacher's softmax over the k logits a row that it passed on, and its gradient;
* ``matvec``     Y = X W^T + b of a few rows with W in 4 bits.

Layouts: MX8 codes are int8 [N, 32 nb], MX4 codes uint8 [N, 16 nb] (the even column in the low half byte), scales uint8 [N, nb], with nb = ceil(width / 32)
and zeros in the columns past the last.
"""
from __future__ import annotations

import math

import torch

own = False

_FIELDS = ("name", "path", "N", "width", "k", "out", "bits", "value", "residual", "temperature")


def _case(*values):
    # width: classes, hidden width or input width; k: alternatives or the teacher's entries a row; out: rows of W; bits: of Y, 0: in its type;
    # value: type of X, the logits, H, Y and their gradients
    return dict(zip(_FIELDS, values))


def listed():
    return [
        # serving: one node's or one token's hidden features before its product
        _case("one_row_norm4", "norm", 1, 4096, 0, 0, 4, "bf16", True, 1.0),
        # full-batch training at hidden width 384 on 717 thousand nodes: the checkpoint that the weight gradient reads
        _case("wide_norm8", "norm", 716847, 384, 0, 0, 8, "bf16", True, 1.0),
        # hidden width 100, rows that are not whole 16-byte pieces in 16 bits
        _case("ragged_norm_step", "norm_step", 40013, 100, 0, 0, 0, "f16", True, 1.0),
        # a training step of the headline graph at hidden width 256
        _case("dense_norm_step", "norm_step", 232965, 256, 0, 0, 0, "f32", True, 1.0),
        # serving: one row of logits over a vocabulary, with the likeliest classes
        _case("one_row_score", "score", 1, 131072, 20, 0, 0, "bf16", False, 1.0),
        # inference on the largest graph, 47 classes
        _case("classes_score", "score", 2449029, 47, 5, 0, 0, "f32", False, 1.0),
        # a training step on a thousand nodes of 41 classes, and one over a vocabulary
        _case("tiny_learn", "learn", 1024, 41, 0, 0, 0, "f32", False, 1.0),
        _case("wide_learn", "learn", 4096, 131072, 0, 0, 0, "bf16", False, 1.0),
        # a student of a classifier with a thousand classes, an odd vocabulary with rows that start anywhere
        _case("classes_distill", "distill", 169343, 1000, 16, 0, 0, "f32", False, 4.0),
        _case("ragged_distill", "distill", 2011, 50021, 50, 0, 0, "bf16", False, 2.0),
        # serving: one row through the weights of a vocabulary; sixteen rows through a square layer
        _case("one_row_matvec", "matvec", 1, 4096, 0, 100003, 4, "bf16", False, 1.0),
        _case("batch_matvec", "matvec", 16, 8192, 0, 8192, 4, "f32", False, 1.0),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 2.4 million rows, widths 16 to 8192, 2 to 131072 classes, up to 64 alternatives, each type."""
    spread = lambda low, high: int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))  # noqa: E731
    while True:
        path = rng.choice(["norm", "norm_step", "score", "learn", "distill", "matvec"])
        value = rng.choice(["f32", "bf16", "f16"])
        if path in ("norm", "norm_step"):
            N, width = spread(1, 2449029), rng.choice([64, 100, 256, 256, 384, 1024, spread(16, 8192), spread(16, 8192), spread(16, 8192)])
            bits = rng.choice([8, 8, 4, 0]) if path == "norm" else 0
            if N * width > 716847 * 384:
                continue
            case = _case("", path, N, width, 0, 0, bits, value, rng.random() < 0.75, 1.0)
        elif path == "matvec":
            N, width, out = rng.choice([1, 1, 1, 2, 3, rng.randint(4, 16)]), spread(64, 16384), spread(16, 131072)
            if width * out > 4096 * 100003:
                continue
            case = _case("", path, N, width, 0, out, 4, value, False, 1.0)
        else:
            N, width = spread(1, 2449029), rng.choice([41, 47, 1000, spread(2, 131072), spread(2, 131072), spread(2, 131072) | 1])
            k = 0 if path == "learn" else min(width, rng.choice([1, 5, 20, 50, rng.randint(1, 64)]))
            if N * width > (2449029 * 47 if path == "score" else 4096 * 131072 // 4):
                continue
            case = _case("", path, N, width, k, 0, 0, value, False, rng.choice([1.0, 2.0, 4.0]) if path == "distill" else 1.0)
        del case["name"]
        return case


# ------------------------------------------------------------------ inputs

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_EPS = 1e-6


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _features(N, width, seed):
    """Hidden features: N(0,1) with a spread from row to row and from column to column, a few rows of zeros."""
    gen = _generator(seed)
    X = torch.randn(N, width, generator=gen, device="cuda")
    X *= torch.exp(0.5 * torch.randn(N, 1, generator=gen, device="cuda"))
    X *= torch.exp(0.3 * torch.randn(1, width, generator=gen, device="cuda"))
    if N > 64:
        X[torch.randint(N, (max(1, N // 200),), generator=gen, device="cuda")] = 0.0
    return X


def _gradient(N, width, seed):
    """Gradients: small, their size spread over the rows."""
    gen = _generator(seed)
    return torch.randn(N, width, generator=gen, device="cuda") * (1e-3 * torch.exp(torch.randn(N, 1, generator=gen, device="cuda")))


def _logits(N, V, labels, dtype, seed):
    """Logits as a trained model has them: a spread of 2, the given class ahead in most rows, the last classes of a wide row masked out."""
    gen = _generator(seed)
    X = torch.empty(N, V, dtype=dtype, device="cuda")
    rows = max(1, (1 << 28) // V)
    for i in range(0, N, rows):
        part = 2.0 * torch.randn(min(rows, N - i), V, generator=gen, device="cuda")
        ahead = 4.0 + 4.0 * torch.randn(part.shape[0], 1, generator=gen, device="cuda")
        part.scatter_add_(1, labels[i:i + rows].clamp_min(0).unsqueeze(1), ahead)
        if V > 256:
            part[:, V - V // 200:] = -math.inf
        X[i:i + rows] = part.to(dtype)
    return X


def _labels(N, V, seed):
    """Given classes, none (-1) in a few rows."""
    gen = _generator(seed)
    labels = torch.randint(V - (V // 200 if V > 256 else 0), (N,), generator=gen, device="cuda")
    return torch.where(torch.rand(N, generator=gen, device="cuda") < 0.02, torch.full_like(labels, -1), labels) if N > 64 else labels


def _teacher(logits, k, seed):
    """The k largest logits a row of a teacher that agrees with the student by and large, and their classes."""
    gen = _generator(seed)
    N, V = logits.shape
    data = torch.empty(N, k, dtype=logits.dtype, device="cuda")
    index = torch.empty(N, k, dtype=torch.uint8 if V <= 256 else torch.int32, device="cuda")
    rows = max(1, (1 << 28) // V)
    for i in range(0, N, rows):
        part = logits[i:i + rows].float()
        part += torch.randn(part.shape, generator=gen, device="cuda")
        top = part.topk(k, dim=1)
        data[i:i + rows] = top.values.to(logits.dtype)
        index[i:i + rows] = top.indices.to(index.dtype)
    return data, index


def _blocks(X):
    """X as [N, nb, 32], zeros past its last column."""
    N, width = X.shape
    nb = (width + 31) // 32
    if width != nb * 32:
        X = torch.nn.functional.pad(X, (0, nb * 32 - width))
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
        return torch.round(_times_power(B, 133 - field)).clamp_(-127.0, 127.0), field
    field = (field - 2).clamp_min(0)
    y = _times_power(B, 127 - field)
    a = y.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), y), field


def _encode4(X):
    """4-bit codes and scales as the calls take them."""
    N = X.shape[0]
    grid, parts, rows = torch.tensor(_E2M1, device="cuda"), [], max(1, (1 << 27) // X.shape[1])
    for i in range(0, N, rows):
        q, s = _quantise(X[i:i + rows], 4)
        q = q.reshape(q.shape[0], -1)
        code = torch.searchsorted(grid, q.abs()).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
        parts.append((code[:, 0::2] | (code[:, 1::2] << 4), s.squeeze(2).to(torch.uint8)))
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def prepare(case, seed):
    path, N, width, k, bits = (case[f] for f in ("path", "N", "width", "k", "bits"))
    dtype = _DTYPE[case["value"]]
    state = {"case": case}
    new = lambda *shape, dtype=dtype: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if path in ("norm", "norm_step"):
        state["X"] = _features(N, width, seed * 7 + 1).to(dtype)
        state["gamma"] = 1.0 + 0.3 * torch.randn(width, generator=_generator(seed * 7 + 2), device="cuda")
        state["residual"] = state["H"] = None
        if case["residual"]:
            state["residual"], state["H"] = _features(N, width, seed * 7 + 3).to(dtype), new(N, width)
        if bits:
            nb = (width + 31) // 32
            state["codes"] = new(N, nb * (32 if bits == 8 else 16), dtype=torch.int8 if bits == 8 else torch.uint8)
            state["scales"] = new(N, nb, dtype=torch.uint8)
            state["restored"] = new(N, width, dtype=torch.bfloat16)  # holds either format's values exactly
        else:
            state["Y"] = new(N, width)
    if path == "norm_step":
        state["dY"] = _gradient(N, width, seed * 7 + 4).to(dtype)
        state["dH"] = _gradient(N, width, seed * 7 + 5).to(dtype) if case["residual"] else None
        state["rstd"], state["dX"], state["dgamma"] = new(N, dtype=torch.float32), new(N, width), new(width, dtype=torch.float32)
    if path in ("score", "learn", "distill"):
        state["labels"] = _labels(N, width, seed * 7 + 1)
        state["logits"] = _logits(N, width, state["labels"], dtype, seed * 7 + 2)
    if path in ("score", "learn"):
        state["logprob"], state["entropy"] = new(N, dtype=torch.float32), new(N, dtype=torch.float32)
    if path == "score":
        state["top_data"], state["top_index"] = new(N, k, dtype=torch.float32), new(N, k, dtype=torch.int32)
    if path == "learn":
        # the gradient of a mean over the rows: advantages, and a small bonus for entropy
        state["dlogprob"] = torch.randn(N, generator=_generator(seed * 7 + 3), device="cuda") / N
        state["dentropy"] = torch.full((N,), -0.01 / N, device="cuda")
        state["dlogits"] = new(N, width)
    if path == "distill":
        state["teacher"], state["classes"] = _teacher(state["logits"], k, seed * 7 + 4)
        state["dloss"] = torch.rand(N, generator=_generator(seed * 7 + 5), device="cuda") / N
        state["loss"], state["dlogits"] = new(N, dtype=torch.float32), new(N, width)
    if path == "matvec":
        gen = _generator(seed * 7 + 2)
        state["X"] = _features(N, width, seed * 7 + 1).to(dtype)
        state["W_codes"], state["W_scales"] = _encode4((torch.rand(case["out"], width, generator=gen, device="cuda") * 2.0 - 1.0) / math.sqrt(width))
        state["bias"] = 0.1 * torch.randn(case["out"], generator=gen, device="cuda")
        state["Y"] = new(N, case["out"])
    torch.cuda.empty_cache()
    return state


# ------------------------------------------------------------------ one pass


def _decode4(codes, scales, width):
    """fp32 values [N, width] of 4-bit codes and scales."""
    N, nb = scales.shape
    grid = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    q = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], dim=2)
    return (q.reshape(N, nb, 32) * torch.exp2(scales.float() - 127.0).unsqueeze(2)).reshape(N, nb * 32)[:, :width]


def _norm_plain(state):
    """(H in its type, r, Y in fp32); the mean of squares in 64 bits, as Y may be rounded to few bits."""
    H = state["X"] if state["residual"] is None else (state["X"].float() + state["residual"].float()).to(state["X"].dtype)
    r = torch.rsqrt(H.double().square().mean(dim=1, keepdim=True) + _EPS).float()
    return H, r, H.float() * r * state["gamma"]


def _log_softmax(x):
    """(log p, p) of rows in fp32."""
    d = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(d)
    S = e.sum(dim=1, keepdim=True)
    return d - torch.log(S), e / S


def _given(values, labels):
    """values[n, labels[n]], 0 where no class is given."""
    got = values.gather(1, labels.clamp_min(0).unsqueeze(1)).squeeze(1)
    return torch.where(labels >= 0, got, torch.zeros_like(got))


def _surprise(logp, p):
    """p log p, 0 where p is."""
    return torch.where(p > 0, p * logp, torch.zeros_like(p))


def _likeliest(logits, k):
    """Columns of the k largest values a row, the lowest column first among equals: the largest of whole numbers that hold value and column."""
    bits = (logits.float() + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    keys = (order << 32) + (0xFFFFFFFF - torch.arange(logits.shape[1], device=logits.device))
    return 0xFFFFFFFF - (keys.topk(k, dim=1).values & 0xFFFFFFFF)


def _run_plain(state):
    case = state["case"]
    path, width, bits, dtype = case["path"], case["width"], case["bits"], _DTYPE[case["value"]]
    if path == "norm":
        H, _, Y = _norm_plain(state)
        if bits:
            q, field = _quantise(Y, bits)
            Y = _times_power(q, field - (133 if bits == 8 else 127)).reshape(H.shape[0], -1)[:, :width].to(torch.bfloat16)
        out = {"Y": Y if bits else Y.to(dtype)}
        return out if state["residual"] is None else {**out, "H": H}
    if path == "norm_step":
        H, r, Y = _norm_plain(state)
        dY, x = state["dY"].float(), H.float() * r
        g = dY * state["gamma"]
        dX = r * (g - x * (g * x).mean(dim=1, keepdim=True))
        if state["dH"] is not None:
            dX = dX + state["dH"].float()
        return {"Y": Y.to(dtype), "H": H, "dX": dX.to(dtype), "dgamma": (dY * x).sum(dim=0)}
    if path == "matvec":
        W = _decode4(state["W_codes"], state["W_scales"], width)
        return {"Y": (torch.mm(state["X"].float(), W.t()) + state["bias"]).to(dtype)}
    x = state["logits"].float()
    if path == "distill":
        T = case["temperature"]
        logp, p = _log_softmax(x / T)
        logq, q = _log_softmax(state["teacher"].float() / T)
        columns = state["classes"].long()
        loss = torch.where(q > 0, q * (logq - logp.gather(1, columns)), torch.zeros_like(q)).sum(dim=1)
        d = p.scatter_add_(1, columns, -q) * (state["dloss"].unsqueeze(1) / T)
        return {"loss": loss, "dlogits": d.to(dtype)}
    logp, p = _log_softmax(x)
    logprob, entropy = _given(logp, state["labels"]), -_surprise(logp, p).sum(dim=1)
    if path == "score":
        index = _likeliest(state["logits"], case["k"])
        return {"logprob": logprob, "entropy": entropy, "top_data": logp.gather(1, index), "top_index": index.to(torch.int32)}
    g = torch.where(state["labels"] >= 0, state["dlogprob"], torch.zeros_like(logprob)).unsqueeze(1)
    d = -g * p - state["dentropy"].unsqueeze(1) * (_surprise(logp, p) + p * entropy.unsqueeze(1))
    d.scatter_add_(1, state["labels"].clamp_min(0).unsqueeze(1), g)
    return {"logprob": logprob, "entropy": entropy, "dlogits": d.to(dtype)}


def _run_own(state):
    import paper_2312_08656_amd as maxk

    case = state["case"]
    path = case["path"]
    if path == "norm":
        if case["bits"]:
            maxk.maxk_rms_norm(state["X"], state["gamma"], codes=state["codes"], scales=state["scales"], residual=state["residual"], H=state["H"], eps=_EPS)
            maxk.maxk_mx_dequantize(state["codes"], state["scales"], state["restored"])
        else:
            maxk.maxk_rms_norm(state["X"], state["gamma"], state["Y"], residual=state["residual"], H=state["H"], eps=_EPS)
        out = {"Y": state["restored"] if case["bits"] else state["Y"]}
        return out if state["residual"] is None else {**out, "H": state["H"]}
    if path == "norm_step":
        H = state["X"] if state["residual"] is None else state["H"]
        maxk.maxk_rms_norm(state["X"], state["gamma"], state["Y"], residual=state["residual"], H=state["H"], rstd=state["rstd"], eps=_EPS)
        maxk.maxk_rms_norm_grad(state["dY"], H, state["gamma"], state["rstd"], state["dX"], state["dgamma"], dH=state["dH"])
        return {"Y": state["Y"], "H": H, "dX": state["dX"], "dgamma": state["dgamma"]}
    if path == "matvec":
        maxk.maxk_mx_matvec(state["X"], state["W_codes"], state["W_scales"], state["Y"], bias=state["bias"])
        return {"Y": state["Y"]}
    if path == "distill":
        maxk.maxk_distill_grad(state["logits"], state["teacher"], state["classes"], state["dloss"], state["dlogits"], temperature=case["temperature"],
                               loss=state["loss"])
        return {"loss": state["loss"], "dlogits": state["dlogits"]}
    if path == "score":
        maxk.maxk_logprobs(state["logits"], state["labels"], state["logprob"], state["entropy"], state["top_data"], state["top_index"])
        return {f: state[f] for f in ("logprob", "entropy", "top_data", "top_index")}
    maxk.maxk_logprobs_grad(state["logits"], state["dlogits"], state["labels"], state["dlogprob"], state["dentropy"], logprob=state["logprob"],
                            entropy=state["entropy"])
    return {f: state[f] for f in ("logprob", "entropy", "dlogits")}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Each input read once, each output written once."""
    path, N, width, k, out, bits = (case[f] for f in ("path", "N", "width", "k", "out", "bits"))
    vb = 4 if case["value"] == "f32" else 2
    nb = (width + 31) // 32
    if path in ("norm", "norm_step"):
        streams = 3 if case["residual"] else 1  # X; the residual and H
        moved = N * width * vb * streams + 4 * width
        if path == "norm":
            moved += 2 * N * nb * (33 if bits == 8 else 17) + 2 * N * width if bits else N * width * vb
            return {"bytes": moved, "flops": 6 * N * width}
        moved += N * width * vb * (3 if case["residual"] else 2) + N * width * vb + 4 * width  # dY, dH, dX; Y; H and r stay on the way
        return {"bytes": moved, "flops": 16 * N * width}
    if path == "matvec":
        return {"bytes": out * nb * 17 + 4 * out + N * (width + out) * vb, "flops": 2 * N * width * out}
    if path == "score":
        return {"bytes": N * width * vb + N * (16 + 8 * k), "flops": 6 * N * width}
    if path == "learn":
        return {"bytes": 2 * N * width * vb + 24 * N, "flops": 12 * N * width}
    return {"bytes": 2 * N * width * vb + N * k * (vb + (1 if width <= 256 else 4)) + 8 * N, "flops": 10 * N * width}


# ------------------------------------------------------------------ the definition in 64 bits


def _exact_values4(codes, scales, width):
    """What stored 4-bit codes stand for, one code at a time from the format's table."""
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
    return (whole * power.repeat_interleave(32, dim=1))[:, :width]


def _exact_stored(X, bits):
    """Nearest stored values of X [N, width], block by block, ties to the even code."""
    values = torch.empty_like(X)
    sizes = torch.tensor(_E2M1, dtype=torch.float64, device=X.device)
    for b in range(0, X.shape[1], 32):
        part = X[:, b:b + 32]
        top = part.abs().max(dim=1).values
        exponent = torch.frexp(top).exponent.double() - 1.0
        exponent = (torch.where(top > 0, exponent, torch.full_like(top, -200.0)) - (0.0 if bits == 8 else 2.0)).clamp(min=-127.0)
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
    return values


def _exact_rows(state, i, rows):
    """One slice of the rows of a softmax path."""
    case = state["case"]
    path, T = case["path"], case["temperature"]
    x = state["logits"][i:i + rows].double() / T
    lse = torch.logsumexp(x, dim=1, keepdim=True)
    logp, p = x - lse, torch.exp(x - lse)
    if path == "distill":
        t, columns = state["teacher"][i:i + rows].double() / T, state["classes"][i:i + rows].long()
        logq = t - torch.logsumexp(t, dim=1, keepdim=True)
        q = torch.exp(logq)
        loss = torch.nan_to_num(q * (logq - logp.gather(1, columns)), nan=0.0).sum(dim=1)
        return {"loss": loss, "dlogits": state["dloss"][i:i + rows].double().unsqueeze(1) / T * p.scatter_add(1, columns, -q)}
    y = state["labels"][i:i + rows]
    has = y >= 0
    at = y.clamp_min(0).unsqueeze(1)
    logprob = torch.where(has, logp.gather(1, at).squeeze(1), 0.0)
    plogp = torch.nan_to_num(p * logp, nan=0.0)
    entropy = -plogp.sum(dim=1)
    if path == "score":
        index = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["k"]]
        return {"logprob": logprob, "entropy": entropy, "top_data": logp.gather(1, index), "top_index": index.to(torch.int32)}
    g = torch.where(has, state["dlogprob"][i:i + rows].double(), 0.0).unsqueeze(1)
    d = -p * g - state["dentropy"][i:i + rows].double().unsqueeze(1) * (plogp + p * entropy.unsqueeze(1))
    return {"logprob": logprob, "entropy": entropy, "dlogits": d.scatter_add(1, at, g)}


def exact(case, seed):
    state = prepare(case, seed)
    path, N, width, bits = (case[f] for f in ("path", "N", "width", "bits"))
    if path in ("norm", "norm_step"):
        H = state["X"].double() if state["residual"] is None else (state["X"].double() + state["residual"].double()).to(state["X"].dtype).double()
        r = (H.pow(2).sum(dim=1, keepdim=True) / width + _EPS).pow(-0.5)
        Y = H * r * state["gamma"].double()
        out = {"Y": _exact_stored(Y, bits) if bits else Y}
        if path == "norm" and state["residual"] is None:
            return out
        out["H"] = H
        if path == "norm_step":
            dY, gamma = state["dY"].double(), state["gamma"].double()
            inner = (dY * gamma * H).sum(dim=1, keepdim=True)
            out["dX"] = dY * gamma * r - H * inner * r.pow(3) / width
            if state["dH"] is not None:
                out["dX"] += state["dH"].double()
            out["dgamma"] = (dY * H * r).sum(dim=0)
        return out
    if path == "matvec":
        W = state["W_codes"].shape[0]
        rows = max(1, (1 << 27) // width)
        parts = [state["X"].double() @ _exact_values4(state["W_codes"][i:i + rows], state["W_scales"][i:i + rows], width).t().contiguous()
                 for i in range(0, W, rows)]
        return {"Y": torch.cat(parts, dim=1) + state["bias"].double()}
    rows = max(1, (1 << 26) // width)
    parts = [_exact_rows(state, i, rows) for i in range(0, N, rows)]
    return {f: torch.cat([p[f] for p in parts]) for f in parts[0]}
