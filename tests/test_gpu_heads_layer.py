"""Both ends of a classifier as they are used together: under autograd, captured into graphs, on other streams, from either marshalling, and the example."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest
import torch

import heads_common as hc
import mx_common as mx
import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _graph(N, gen):
    degree = torch.randint(0, 12, (N,), generator=gen, device="cuda")
    rowptr = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    rowptr[1:] = torch.cumsum(degree, 0)
    nnz = int(rowptr[-1])
    col = torch.randint(N, (nnz,), generator=gen, device="cuda").to(torch.int32)
    return maxk.maxk_graph_create(rowptr, col, torch.randn(nnz, generator=gen, device="cuda"))


def _norm64(X, residual, gamma):
    H = X if residual is None else X + residual
    return H * torch.rsqrt((H * H).mean(1, keepdim=True) + EPS) * gamma, H


@pytest.mark.parametrize("residual", [True, False])
def test_residual_norm_under_autograd(residual):
    gen = torch.Generator(device="cuda").manual_seed(1)
    N, dim = 50, 72
    X, R = (torch.randn(N, dim, generator=gen, device="cuda", requires_grad=True) for _ in range(2))
    gamma = torch.randn(dim, generator=gen, device="cuda", requires_grad=True)
    a, b = (torch.randn(N, dim, generator=gen, device="cuda") for _ in range(2))
    inputs = [X, gamma] + ([R] if residual else [])
    doubles = [t.detach().double().cpu().requires_grad_(True) for t in (X, gamma, R)]
    y, h = _norm64(doubles[0], doubles[2] if residual else None, doubles[1])
    for use in ("Y", "H", "both") if residual else ("Y",):
        out = maxk.maxk_residual_norm(X, gamma, R if residual else None, EPS)
        Y, H = out if residual else (out, None)
        got = (Y * a).sum() * (use != "H") + ((H * b).sum() if use != "Y" else 0.0)
        want = (y * a.double().cpu()).sum() * (use != "H") + ((h * b.double().cpu()).sum() if use != "Y" else 0.0)
        grads = torch.autograd.grad(got, inputs, allow_unused=True)
        refs = torch.autograd.grad(want, doubles[:2] + ([doubles[2]] if residual else []), retain_graph=True, allow_unused=True)
        for g, r in zip(grads, refs):
            assert (g is None or r is None) and use == "H" or torch.allclose(g.double().cpu(), r, rtol=1e-5, atol=1e-5)  # fp32 sums of 72 and 50 terms of size 1
    # the gradient that a sum leaves is expanded; rows that are not contiguous; gamma alone
    Y = maxk.maxk_residual_norm(X.detach().t().contiguous().t(), gamma)
    (g,) = torch.autograd.grad(Y.sum(), gamma)
    r = _norm64(X.detach().double(), None, torch.ones(dim, dtype=torch.float64, device="cuda"))[0].sum(0)
    assert torch.allclose(g.double(), r, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("bits", [8, 4])
def test_norm_layer(bits, with_bias):
    """The norm and the layer one by one give the same bits, and so do their gradients."""
    gen = torch.Generator(device="cuda").manual_seed(bits)
    N, din, dout, k = 300, 100, 64, 8
    graph = _graph(N, gen)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    X, R, gamma, W, b = (t.requires_grad_(True) for t in (randn(N, din), randn(N, din), 1 + 0.3 * randn(din), randn(dout, din) / 10, randn(dout)))
    b = b if with_bias else None
    dOut, dH = randn(N, dout), randn(N, din)
    leaves = [t for t in (X, R, gamma, W, b) if t is not None]
    out, H = maxk.maxk_norm_layer(X, R, gamma, W, b, graph, k, bits, EPS)
    grads = torch.autograd.grad([out, H], leaves, [dOut, dH])
    Y, H2 = maxk.maxk_residual_norm(X, gamma, R, EPS)
    out2 = maxk.maxk_layer(Y, W, b, graph, k, bits)
    want = torch.autograd.grad([out2, H2], leaves, [dOut, dH])
    assert torch.equal(out, out2) and torch.equal(H, H2)
    assert all(torch.equal(g, w) for g, w in zip(grads, want))
    # without a residual; H alone; no gradient of some
    alone = maxk.maxk_norm_layer(X, None, gamma, W, b, graph, k, bits, EPS)
    assert torch.equal(alone, maxk.maxk_layer(maxk.maxk_residual_norm(X, gamma, None, EPS), W, b, graph, k, bits))
    _, H = maxk.maxk_norm_layer(X, R, gamma, W, b, graph, k, bits, EPS)
    g = torch.autograd.grad(H, leaves, dH, allow_unused=True)
    assert torch.equal(g[0], dH) and torch.equal(g[1], dH) and all((t == 0).all() for t in g[2:])
    out, _ = maxk.maxk_norm_layer(X.detach(), R.detach(), gamma.detach(), W, None, graph, k, bits, EPS)
    assert torch.equal(torch.autograd.grad(out, W, dOut)[0], torch.autograd.grad(maxk.maxk_layer(Y.detach(), W, None, graph, k, bits), W, dOut)[0])
    with torch.no_grad():
        assert torch.equal(maxk.maxk_norm_layer(X, R, gamma, W, b, graph, k, bits, EPS)[0], out2)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        assert maxk.maxk_norm_layer(X.bfloat16(), R.bfloat16(), gamma, W, b, graph, k, bits, EPS)[0].dtype == torch.float32
    for bad in (lambda: maxk.maxk_norm_layer(X, R, gamma, W, b, graph, k, 16), lambda: maxk.maxk_norm_layer(X, R[:, 1:], gamma, W, b, graph, k),
                lambda: maxk.maxk_norm_layer(X.half(), R.half(), gamma, W, b, graph, k), lambda: maxk.maxk_norm_layer(X, R, gamma[1:], W, b, graph, k)):
        with pytest.raises(maxk.MaxKError):
            bad()
    graph.destroy()


def test_second_derivatives_are_refused():
    X = torch.randn(6, 8, device="cuda", requires_grad=True)
    gamma = torch.ones(8, device="cuda")
    labels = torch.zeros(6, dtype=torch.int64, device="cuda")
    top = (torch.randn(6, 2, device="cuda"), torch.zeros(6, 2, dtype=torch.uint8, device="cuda"))
    for f in (lambda: maxk.maxk_residual_norm(X, gamma), lambda: maxk.maxk_class_logprobs(X, labels)[0], lambda: maxk.maxk_distill_loss(X, *top)):
        (g,) = torch.autograd.grad((f() ** 2).sum(), X, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
def test_logprobs_and_distillation_under_autograd(dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    N, V, k = 40, 120, 6
    x = (3 * torch.randn(N, V, generator=gen, device="cuda")).to(dtype).requires_grad_(True)
    labels = torch.randint(V, (N,), generator=gen, device="cuda")
    labels[3] = -1
    logprob, entropy = maxk.maxk_class_logprobs(x, labels)
    (g,) = torch.autograd.grad(-logprob.mean() + 0.1 * entropy.sum(), x)  # (an expanded gradient, and one of a broadcast scalar)
    *_, R = hc.logprobs(x, labels)
    want, bound = hc.logprobs_grad(R, labels, torch.full((N,), -1 / N), torch.full((N,), 0.1))
    hc.close(g, want, bound + 1e-8, dtype)
    assert g.dtype == dtype
    (g,) = torch.autograd.grad(maxk.maxk_class_logprobs(x, None).sum(), x)
    hc.close(g, *hc.logprobs_grad(R, None, None, torch.ones(N)), dtype)
    (g,) = torch.autograd.grad(maxk.maxk_class_logprobs(x.t().contiguous().t(), labels)[0].sum(), x)
    hc.close(g, *hc.logprobs_grad(R, labels, torch.ones(N), None), dtype)
    # a teacher's likeliest classes as maxk_topk_cbsr and as maxk_logprobs leave them
    teacher = torch.randn(N, V, generator=gen, device="cuda")
    data, index = torch.empty(N, k, device="cuda"), torch.empty(N, k, dtype=torch.uint8, device="cuda")
    maxk.maxk_topk_cbsr(teacher, k, data, index)
    logp, columns = torch.empty(N, k, device="cuda"), torch.empty(N, k, dtype=torch.int32, device="cuda")
    maxk.maxk_logprobs(teacher, top_data=logp, top_index=columns)
    assert torch.equal(columns.sort(dim=1).values.to(torch.uint8), index)
    for pair in ((data, index), (logp, columns)):
        loss = maxk.maxk_distill_loss(x, *pair, 2.0)
        want, bound, dx, dx_bound = hc.distill(x, *pair, 2.0, torch.full((N,), 1 / N))
        hc.close(loss, want, bound)
        (g,) = torch.autograd.grad(loss.mean(), x)
        hc.close(g, dx, dx_bound, dtype)


def _chain(t):
    """A residual norm stored in 4 bits, the product with 4-bit weights of its 32-bit form, log probabilities, alternatives, and both losses' gradients."""
    maxk.maxk_rms_norm(t["X"], t["gamma"], t["Y"], t["codes"], t["scales"], t["R"], t["H"], t["rstd"], EPS)
    maxk.maxk_mx_matvec(t["Y"], t["wc"], t["ws"], t["logits"], t["bias"])
    maxk.maxk_logprobs(t["logits"], t["labels"], t["logprob"], t["entropy"], t["data"], t["index"], workspace=t["room"])
    maxk.maxk_logprobs_grad(t["logits"], t["dlogits"], t["labels"], t["g"], t["u"], workspace=t["room"])
    maxk.maxk_distill_grad(t["logits"], t["data"], t["index"], t["g"], t["dlogits2"], 2.0, t["loss"], workspace=t["room"])
    maxk.maxk_rms_norm_grad(t["dY"], t["H"], t["gamma"], t["rstd"], t["dX"], t["dgamma"], dH=t["R"], workspace=t["room2"])


def _state(N, dim, V, k, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    t = {"X": randn(N, dim), "R": randn(N, dim), "gamma": 1 + 0.3 * randn(dim), "dY": randn(N, dim), "bias": randn(V), "g": randn(N), "u": randn(N),
         "labels": torch.randint(V, (N,), generator=gen, device="cuda")}
    t["wc"], t["ws"] = (torch.from_numpy(a).cuda() for a in mx.quantize(randn(V, dim).cpu().numpy() / dim ** 0.5, 4))
    t["codes"], t["scales"] = maxk.mx_empty(N, dim, 4)
    for name, shape in (("Y", (N, dim)), ("H", (N, dim)), ("dX", (N, dim)), ("logits", (N, V)), ("dlogits", (N, V)), ("dlogits2", (N, V)), ("rstd", (N,)), ("logprob", (N,)),
                        ("entropy", (N,)), ("loss", (N,)), ("data", (N, k)), ("dgamma", (dim,))):
        t[name] = torch.zeros(shape, device="cuda")
    t["index"] = torch.zeros(N, k, dtype=torch.int32, device="cuda")
    t["room"] = torch.empty(max(16, maxk.classes_workspace(N, V, k), maxk.classes_workspace(N, V)), dtype=torch.uint8, device="cuda")
    t["room2"] = torch.empty(maxk.rms_norm_grad_workspace(N, dim), dtype=torch.uint8, device="cuda")
    return t


_OUT = ("Y", "codes", "scales", "H", "rstd", "logits", "logprob", "entropy", "data", "index", "dlogits", "dlogits2", "loss", "dX", "dgamma")


def _same(a, b):
    return [n for n in _OUT if not torch.equal(a[n], b[n])]


@pytest.mark.parametrize("N,dim,V,k", [(1, 256, 40000, 20), (3, 100, 47, 5), (16, 512, 9001, 64), (40, 64, 1000, 8)])
def test_captured_and_replayed(N, dim, V, k):
    """Two graphs of the chain with inputs of their own and a workspace in common, replayed in turn between eager work on the same stream; every replay is checked."""
    states, wants = [_state(N, dim, V, k, s) for s in (1, 2)], [_state(N, dim, V, k, s) for s in (1, 2)]
    states[1]["room"], states[1]["room2"] = states[0]["room"], states[0]["room2"]
    for t in wants:
        _chain(t)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        _chain(states[0]), _chain(states[1])
        stream.synchronize()
        for t in states:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                _chain(t)
            graphs.append(g)
        for turn in range(4):
            for t, w, g in zip(states, wants, graphs):
                for n in _OUT:
                    t[n].zero_()
                g.replay()
                stream.synchronize()
                assert _same(t, w) == [], turn
            _chain(wants[0])  # eager work between replays
            if turn == 1:  # other inputs in the same place
                for both in zip(states, wants):
                    for t in both:
                        t["X"].add_(0.25)
                for w in wants:
                    _chain(w)
            stream.synchronize()


def test_another_stream_and_two_at_once():
    """Calls on a side stream, and on two streams at a time with a workspace each."""
    wants, states = [_state(2, 128, 50001, 10, s) for s in (5, 6)], [_state(2, 128, 50001, 10, s) for s in (5, 6)]
    for t in wants:
        _chain(t)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for t, s in zip(states, streams):
            with torch.cuda.stream(s):
                _chain(t)
    torch.cuda.synchronize()
    assert [_same(t, w) for t, w in zip(states, wants)] == [[], []]


class _Counted:
    def __init__(self, module):
        self.module, self.made, self.left = module, [], []

    def __getattr__(self, name):
        def call(*args):
            got = getattr(self.module, name)(*args)
            (self.made if got else self.left).append(name)
            return got

        return call


def test_either_marshalling_gives_the_same(monkeypatch):
    assert binding._FAST is not None
    fast, slow = _state(4, 100, 30000, 7, 9), _state(4, 100, 30000, 7, 9)
    counted = _Counted(binding._FAST)
    monkeypatch.setattr(binding, "_FAST", counted)
    _chain(fast)
    assert counted.left == [] and counted.made == ["rms_norm", "mx_matvec", "logprobs", "logprobs_grad", "distill", "rms_norm_grad"]
    monkeypatch.setattr(binding, "_FAST", None)
    _chain(slow)
    assert _same(fast, slow) == []
    for t in (fast, slow):  # workspaces of torch's allocator, one that is too small
        t["room"] = t["room2"] = None
    _chain(slow)
    monkeypatch.undo()
    _chain(fast)
    assert _same(fast, slow) == []
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    texts = []
    for module in (binding._FAST, None):
        monkeypatch.setattr(binding, "_FAST", module)
        for call in (lambda: maxk.maxk_logprobs(fast["logits"], fast["labels"], fast["logprob"], workspace=small),
                     lambda: maxk.maxk_rms_norm_grad(fast["dY"], fast["H"], fast["gamma"], fast["rstd"], fast["dX"], fast["dgamma"], workspace=small),
                     lambda: maxk.maxk_distill(fast["logits"], fast["data"], fast["index"], fast["loss"], -1.0),
                     lambda: maxk.maxk_rms_norm(fast["X"], fast["gamma"], fast["Y"], eps=0.0),
                     lambda: maxk.maxk_logprobs(fast["logits"], fast["labels"][:2], fast["logprob"]),
                     lambda: maxk.maxk_rms_norm(fast["X"], fast["gamma"].double(), fast["Y"]),
                     lambda: maxk.maxk_logprobs(fast["logits"].t(), None, None, fast["entropy"]),
                     lambda: maxk.maxk_mx_matvec(fast["Y"], fast["wc"], fast["ws"], fast["logits"], fast["bias"].half())):
            with pytest.raises(maxk.MaxKError) as e:
                call()
            texts.append(str(e.value))
        monkeypatch.undo()
    assert texts[:8] == texts[8:] and "status -5" in texts[0] and "status -5" in texts[1]


def test_calls_are_the_sum_of_their_parts():
    """Rows by themselves give what they give together, in the forms that few and many rows take."""
    t = _state(1, 256, 20000, 9, 11)
    rows = torch.randn(700, 20000, device="cuda")
    labels = torch.arange(700, device="cuda")
    lp, H = torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
    maxk.maxk_logprobs(rows, labels, lp, H)
    want, lp_bound, wantH, H_bound, _ = hc.logprobs(rows[[0, 333]], labels[[0, 333]])
    for i, r in enumerate((0, 333)):
        one, e = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        maxk.maxk_logprobs(rows[r:r + 1], labels[r:r + 1], one, e)
        for got in (one, lp[r:r + 1]):
            hc.close(got, want[i:i + 1], lp_bound[i:i + 1])
        for got in (e, H[r:r + 1]):
            hc.close(got, wantH[i:i + 1], H_bound[i:i + 1])


def test_the_example_runs():
    path = Path(__file__).resolve().parent.parent / "examples" / "distill_layers.py"
    spec = importlib.util.spec_from_file_location("distill_layers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for bits in (8, 4):
        taught, losses, (classes, logprobs) = example.train(nodes=3000, degree=10, steps=10, bits=bits)
        assert np.isfinite(taught).all() and np.isfinite(losses).all() and len(set(classes)) == 3 and all(p <= 0 for p in logprobs)
