"""Logits far from 0 beside ordinary ones, and rows whose largest logit is far from 0, against 64 bits: masks of a large finite value, small temperatures.

Sizes are those of every way that a row of more than 8192 columns takes: cut among workgroups (few rows), held by one, and gone through by 256, 512 and 1024 threads."""
import numpy as np
import pytest
import torch

import heads_common as hc
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu

SIZES = [(1, 16384), (3, 50021), (1, 131072), (600, 9001), (150, 20003), (600, 20003), (1100, 20003), (1100, 40009)]
TYPES = [torch.float32, torch.bfloat16]


def batches(rows, N, V, dtype, gen):
    """Rows [R x V] in float32 as matrices of N rows, others between them: (matrix, where the rows are)."""
    R = rows.shape[0]
    if N >= R:
        x = (3 * torch.randn(N, V, generator=gen, device="cuda")).to(dtype)
        at = torch.arange(R, device="cuda") * (N // R)
        x[at] = rows.to(dtype)
        yield x, at
        return
    for first in range(0, R, N):
        last = min(first + N, R)
        yield rows[last - N:last].to(dtype).contiguous(), torch.arange(N, device="cuda")


def check_scores(x, at, gen):
    N, V = x.shape
    labels = torch.randint(V, (N,), generator=gen, device="cuda")
    labels[at[::2]] = x[at[::2]].float().argmax(dim=1)
    g, u = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    lp, lp_bound, H, H_bound, R = hc.logprobs(x[at], labels[at])
    for k in (0, 5, 30):  # (few and many alternatives take different ways)
        logprob, entropy = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
        data = torch.full((N, k), 7.0, device="cuda") if k else None
        index = torch.full((N, k), 7, dtype=torch.int32, device="cuda") if k else None
        maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
        hc.close(logprob[at], lp, lp_bound)
        hc.close(entropy[at], H, H_bound)
        if k:
            want = hc.likeliest(x[at], k)
            assert np.array_equal(index[at].cpu().numpy(), want)
            top = np.take_along_axis(R.logp, want, 1)
            hc.close(data[at], top, R.u + 4 * hc.U * (np.abs(np.where(np.isfinite(top), top, 0)) + 2 * np.abs(R.lnS)))
    for pair in ((g, u), (g, None)):
        dx = torch.full_like(x, 7)
        maxk.maxk_logprobs_grad(x, dx, labels, *pair)
        want, bound = hc.logprobs_grad(R, labels[at], *(None if t is None else t[at] for t in pair))
        hc.close(dx[at], want, bound, x.dtype)


def check_distillation(x, at, temperature, gen):
    N, V = x.shape
    k = 12
    index = torch.randint(V, (N, k), generator=gen, device="cuda").int()  # (masked columns among them)
    index[:, :4] = x.float().topk(4, dim=1).indices.int()
    data = torch.randn(N, k, generator=gen, device="cuda")
    dloss = torch.randn(N, generator=gen, device="cuda")
    want, bound, dx, dx_bound = hc.distill(x[at], data[at], index[at], temperature, dloss[at])
    loss, grad = torch.full((N,), 7.0, device="cuda"), torch.full_like(x, 7)
    maxk.maxk_distill(x, data, index, loss, temperature)
    hc.close(loss[at], want, bound)
    maxk.maxk_distill_grad(x, data, index, dloss, grad, temperature)
    hc.close(grad[at], dx, dx_bound, x.dtype)


def masked_rows(V, dtype, gen):
    """Masks of a large finite value beside ordinary logits: at the row's start, its end, scattered over half of it, and over all but a few columns."""
    col = torch.arange(V, device="cuda")
    rows = []
    for value in (-1e7, -1e8, -1e9, -1e10, -1e20, -1e30, torch.finfo(dtype).min):
        for mask in (col < V * 3 // 100, col >= V - V * 3 // 100, torch.rand(V, generator=gen, device="cuda") < 0.5, (col + 1) % 4001 != 0):
            row = 3 * torch.randn(V, generator=gen, device="cuda")
            row[mask] = value
            rows.append(row)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("N,V", SIZES)
def test_masks_of_a_large_finite_value(N, V, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N + V)
    for x, at in batches(masked_rows(V, dtype, gen), N, V, dtype, gen):
        check_scores(x, at, gen)


@pytest.mark.parametrize("temperature", [1.0, 2.0, 3.0, 5.0])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("N,V", SIZES)
def test_masks_of_a_large_finite_value_in_distillation(N, V, dtype, temperature):
    gen = torch.Generator(device="cuda").manual_seed(N + V)
    for x, at in batches(masked_rows(V, dtype, gen), N, V, dtype, gen):
        check_distillation(x, at, temperature, gen)


def test_what_is_not_finite_beside_a_mask():
    """A NaN whose lane has nothing else than masked columns still makes its row NaN; so does +Inf."""
    for N, V in SIZES:
        x = torch.zeros(max(N, 2), V, device="cuda")
        x[:, V // 2:] = -1e30
        x[0, V - 1], x[-1, V - 3] = float("nan"), float("inf")
        for i in (0, x.shape[0] - 1):
            y = x if N > 1 else x[i:i + 1].contiguous()
            at = i if N > 1 else 0
            logprob, entropy, dx = torch.zeros(y.shape[0], device="cuda"), torch.zeros(y.shape[0], device="cuda"), torch.zeros_like(y)
            labels = torch.zeros(y.shape[0], dtype=torch.int32, device="cuda")
            maxk.maxk_logprobs(y, labels, logprob, entropy)
            assert torch.isnan(logprob[at]) and torch.isnan(entropy[at]), (N, V)
            maxk.maxk_logprobs_grad(y, dx, labels, torch.ones(y.shape[0], device="cuda"))
            assert torch.isnan(dx[at]).all(), (N, V)
            if N > 2:
                assert torch.isfinite(entropy[1:-1]).all() and torch.isfinite(dx[1:-1]).all()


def far_rows(V, gen):
    """Largest logits far from 0: all columns alike, apart by steps of the value's size, one column above ordinary ones or below all others."""
    rows = []
    for size in (5.5e6, 1e7, 1e9, 1e10, 1e12, 1e20, 1e30, 3e38):
        for value in (size, -size):
            rows.append(torch.full((V,), value, device="cuda"))
            rows.append(value * (1 - 2.0 ** -6 * torch.randint(0, 9, (V,), generator=gen, device="cuda")))
            row = 3 * torch.randn(V, generator=gen, device="cuda")
            row[V // 3] = value
            rows.append(row)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("N,V", SIZES)
def test_rows_far_from_zero(N, V, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N + V)
    for x, at in batches(far_rows(V, gen), N, V, dtype, gen):
        check_scores(x, at, gen)


@pytest.mark.parametrize("temperature", [1.0, 3.0])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("N,V", SIZES)
def test_rows_far_from_zero_in_distillation(N, V, dtype, temperature):
    gen = torch.Generator(device="cuda").manual_seed(N + V)
    for x, at in batches(far_rows(V, gen), N, V, dtype, gen):
        check_distillation(x, at, temperature, gen)


@pytest.mark.parametrize("temperature", [1e-6, 1e-9, 1e-20, 1e-36])
@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V", [(3, 50021), (600, 20003), (1100, 20003)])
def test_small_temperatures(N, V, dtype, temperature):
    """Ordinary logits, whose scaled values are far from 0."""
    gen = torch.Generator(device="cuda").manual_seed(N + V)
    x = (3 * torch.randn(N, V, generator=gen, device="cuda")).to(dtype)
    x[1] = x[1].sign()  # many largest ones
    at = torch.arange(0, N, max(1, N // 12), device="cuda")
    at[min(1, at.numel() - 1)] = 1
    check_distillation(x, at, temperature, gen)
