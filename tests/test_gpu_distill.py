"""Distillation from a teacher's largest logits against 64 bits: loss and gradient."""
import numpy as np
import pytest
import torch

import heads_common as hc
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu
INF = float("inf")


def inputs(N, V, k, dtype, seed, teacher=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (3 * torch.randn(N, V, generator=gen, device="cuda")).to(dtype)
    t = x.float() + torch.randn(N, V, generator=gen, device="cuda")
    top = t.topk(k, dim=1)
    order = torch.rand(N, k, generator=gen, device="cuda").argsort(dim=1)  # in any order
    data, index = top.values.gather(1, order).to(teacher), top.indices.gather(1, order)
    index = index.to(torch.uint8 if V <= 256 else torch.int32)
    return x, data, index, torch.randn(N, generator=gen, device="cuda")


def check(x, data, index, dloss, temperature):
    N = x.shape[0]
    want, bound, dx, dx_bound = hc.distill(x, data, index, temperature, dloss)
    loss, only, grad = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.full_like(x, 7)
    maxk.maxk_distill(x, data, index, only, temperature)
    hc.close(only, want, bound)
    maxk.maxk_distill_grad(x, data, index, dloss, grad, temperature, loss)
    hc.close(loss, want, bound)
    hc.close(grad, dx, dx_bound, x.dtype)
    own = x.clone()
    maxk.maxk_distill_grad(own, data, index, dloss, own, temperature)  # in the logits' own memory
    assert torch.equal(own, grad)
    return loss, grad


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V", [1, 2, 7, 32, 47, 64, 65, 100, 256, 257, 512, 1000, 1025, 2048, 2500, 5003, 8191, 12001])
def test_distill(V, dtype):
    for k, temperature, teacher in ((1, 1.0, torch.float32), (min(V, 16), 2.0, dtype), (min(V, 50), 0.5, torch.float16)):
        check(*inputs(33, V, k, dtype, V + k, teacher), temperature)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V,k", [(1, 32768, 20), (3, 131072, 64), (2, 50021, 1000), (600, 4099, 33), (600, 9001, 70), (150, 20003, 64), (1, 1, 1), (5, 9000, 1024), (1500, 300, 40), (3001, 47, 8)])
def test_few_and_many_rows(N, V, k, dtype):
    check(*inputs(N, V, k, dtype, N + V + k), 4.0)


@pytest.mark.parametrize("V", [40, 200, 1000, 3000, 7000, 9000, 17000])
def test_entries_that_are_none_or_several(V):
    """Columns outside the row, -Inf, rows without entries, columns that come more than once, logits that are masked out."""
    N, k = 12, 24
    x, data, index, dloss = inputs(N, V, k, torch.float32, V)
    index = index.to(torch.int32)
    index[0, ::2] = -1
    index[1, 3] = V
    data[2, 5:9] = -INF
    data[3] = -INF
    index[4] = -1
    index[5, 1:4] = index[5, 0].clone()  # four times one column
    index[6] = index[6, 0].clone()
    x[7, index[7, 2].item()] = -INF  # the teacher wants what is masked out
    x[8] = -INF
    x[9] = -INF
    index[9] = -1
    x[10, :V // 2] = -INF
    data[10] = torch.where(x[10, index[10].long()].isinf(), -INF, data[10])
    index[11, 5], index[11, 9] = index[11, 9].item(), index[11, 5].item()
    index[11, 7] = index[11, 20]
    loss, grad = check(x, data, index, dloss, 2.0)
    assert loss[3] == 0 and loss[4] == 0 and (grad[3:5] == 0).all()
    assert loss[7] == INF and torch.isfinite(grad).all()
    assert loss[8] == INF and loss[9] == 0 and (grad[8:10] == 0).all()


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V,k", [(8, 8), (9, 1), (16, 5), (23, 8), (24, 3), (27, 9), (33, 2), (40, 8), (47, 5), (47, 8), (55, 7)])
def test_many_short_rows(V, k, dtype):
    """Rows enough for the form with a lane a row (nine entries: not); a last workgroup that is not full, entries that are none or several, any element's alignment."""
    N = (1 << 19) + 225
    for index_type, teacher in ((torch.uint8, dtype), (torch.int32, torch.float32), (torch.uint16, torch.float16)):
        x, data, index, dloss = inputs(N, V, k, dtype, V + k, teacher)
        index = index.to(torch.int32)
        index[:20] = torch.randint(V, (20, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).int()
        index[20, 0] = V
        data[21, k // 2] = -INF
        data[22] = -INF
        index[23] = 255
        x[24, index[24, k - 1].item()] = -INF
        x[25] = -INF
        x[26] = -INF
        index[26] = 255
        x[27] = torch.finfo(dtype).min
        index = index.to(index_type)
        some = torch.cat([torch.arange(150), torch.arange(N - 300, N)]).cuda()
        want, bound, dx, dx_bound = hc.distill(x[some], data[some], index.to(torch.int32)[some], 2.0, dloss[some])
        loss, only, grad = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.full_like(x, 7)
        maxk.maxk_distill(x, data, index, only, 2.0)
        maxk.maxk_distill_grad(x, data, index, dloss, grad, 2.0, loss)
        assert torch.equal(loss, only)
        hc.close(loss[some], want, bound)
        hc.close(grad[some], dx, dx_bound, dtype)
        assert (loss[22:24] == 0).all() and loss[24] == INF and loss[25] == INF and loss[26] == 0 and (grad[[22, 23, 25, 26]] == 0).all()
        flat, out = (torch.full((N * V + 16,), 3.0, dtype=dtype, device="cuda") for _ in range(2))
        flat[3:3 + N * V].copy_(x.view(-1))
        moved = out[1:1 + N * V].view(N, V)
        maxk.maxk_distill_grad(flat[3:3 + N * V].view(N, V), data, index, dloss, moved, 2.0)
        assert torch.equal(moved, grad) and out[0] == 3 and (out[1 + N * V:] == 3).all()
        maxk.maxk_distill_grad(x, data, index, dloss, x, 2.0)  # in the logits' own memory
        assert torch.equal(x, grad)


def test_non_finite():
    x, data, index, dloss = inputs(5, 60, 6, torch.float32, 3)
    x[0, 10] = float("nan")
    x[1, 10] = INF
    data[2, 1] = float("nan")
    data[3, 1] = INF
    loss, grad = torch.empty(5, device="cuda"), torch.empty_like(x)
    maxk.maxk_distill_grad(x, data, index, dloss, grad, 1.0, loss)
    assert torch.isnan(loss[:4]).all() and torch.isfinite(loss[4]) and torch.isnan(grad[:4]).all() and torch.isfinite(grad[4]).all()


def test_gradients_are_differences():
    N, V, k, T = 4, 25, 5, 3.0
    x, data, index, dloss = inputs(N, V, k, torch.float32, 21)
    index[1, 2] = index[1, 0]
    grad = torch.empty_like(x)
    maxk.maxk_distill_grad(x, data, index, dloss, grad, T)
    t, col = hc.f64(data) / T, index.cpu().numpy().astype(int)
    q = np.exp(t - t.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)

    def value(x):
        z = x / T
        lp = z - z.max(1, keepdims=True)
        lp -= np.log(np.exp(lp).sum(1, keepdims=True))
        return (hc.f64(dloss)[:, None] * q * (np.log(q) - np.take_along_axis(lp, col, 1))).sum()

    base, step = hc.f64(x), 1e-5
    for n, i in ((0, 0), (0, col[0, 1]), (1, col[1, 0]), (2, 24), (3, col[3, 4])):
        up, down = base.copy(), base.copy()
        up[n, i] += step
        down[n, i] -= step
        assert abs((value(up) - value(down)) / (2 * step) - grad[n, i].item()) < 1e-5


def test_no_rows():
    x, d, i, v = torch.empty(0, 9, device="cuda"), torch.empty(0, 2, device="cuda"), torch.empty(0, 2, dtype=torch.uint8, device="cuda"), torch.empty(0, device="cuda")
    maxk.maxk_distill(x, d, i, v)
    maxk.maxk_distill_grad(x, d, i, v, x.clone())
