"""Forms of the class rows' and the norm's kernels by the rules that choose them: rows gone through by 256 and 512 threads with a gradient, teachers of more entries than
lanes there, and more rows than the norm has workgroups."""
import numpy as np
import pytest
import torch

import heads_common as hc
import paper_2312_08656_amd as maxk
import test_gpu_distill as distill
import test_gpu_logprobs as logprobs

pytestmark = pytest.mark.gpu

# More than 16384 columns: 513 to 1024 rows 512 threads; more rows 256 up to 32768 columns of 16 bits, 512 up to 32768 of 32 and 65536 of 16, 1024 beyond
ROWS = [(700, 20003), (1100, 16385), (1100, 32768), (1100, 33001)]


@pytest.mark.parametrize("k", [5, 64, 65, 300])
@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V", ROWS)
def test_distillation_of_wide_rows(N, V, dtype, k):
    x, data, index, dloss = distill.inputs(N, V, k, dtype, N + V + k)
    index[3, :3] = index[3, 0].clone()  # entries of one column
    index[4, 1] = V
    at = torch.cat([torch.arange(6), torch.arange(6, N, N // 10), torch.arange(N - 2, N)]).cuda()
    want, bound, dx, dx_bound = hc.distill(x[at], data[at], index[at], 2.0, dloss[at])
    loss, only, grad = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.full_like(x, 7)
    maxk.maxk_distill(x, data, index, only, 2.0)
    hc.close(only[at], want, bound)
    maxk.maxk_distill_grad(x, data, index, dloss, grad, 2.0, loss)
    hc.close(loss[at], want, bound)
    hc.close(grad[at], dx, dx_bound, dtype)
    maxk.maxk_distill_grad(x, data, index, dloss, x, 2.0)  # in the logits' own memory
    assert torch.equal(x, grad)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V", ROWS)
def test_log_probabilities_of_wide_rows(N, V, dtype):
    x, labels, gen = logprobs.inputs(N, V, dtype, N + V)
    g, u = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    at = torch.cat([torch.arange(8), torch.arange(8, N, N // 10), torch.arange(N - 2, N)]).cuda()
    lp, lp_bound, H, H_bound, R = hc.logprobs(x[at], labels[at])
    for pair in ((g, u), (g, None)):
        logprob, entropy, dx = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.full_like(x, 7)
        maxk.maxk_logprobs_grad(x, dx, labels, *pair, logprob=logprob, entropy=entropy)
        hc.close(logprob[at], lp, lp_bound)
        hc.close(entropy[at], H, H_bound)
        want, bound = hc.logprobs_grad(R, labels[at], *(None if t is None else t[at] for t in pair))
        hc.close(dx[at], want, bound, dtype)
    maxk.maxk_logprobs_grad(x, x, labels, g)  # in the logits' own memory
    assert torch.equal(x, dx)


# one width of each form whose teams are a workgroup, and shorter rows: more than twice 8192 workgroups, so that a workgroup has several rows
@pytest.mark.parametrize("N,dim,dtype", [(20000, 2100, torch.float32), (17001, 5003, torch.bfloat16), (16500, 9001, torch.float16), (70001, 700, torch.bfloat16), (1_100_003, 9, torch.float32)])
def test_norm_of_more_rows_than_workgroups(N, dim, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N)
    X, R = ((2 * torch.randn(N, dim, generator=gen, device="cuda") * torch.exp(torch.randn(N, 1, generator=gen, device="cuda"))).to(dtype) for _ in range(2))
    gamma = 1 + 0.3 * torch.randn(dim, generator=gen, device="cuda")
    H, Y, rstd = torch.full_like(X, 7), torch.full_like(X, 7), torch.full((N,), 7.0, device="cuda")
    codes, scales = maxk.mx_empty(N, dim, 8)
    maxk.maxk_rms_norm(X, gamma, Y, codes, scales, R, H, rstd)
    at = torch.cat([torch.arange(0, N, N // 40), torch.arange(N - 20, N)]).cuda()
    want_H, r, y = hc.norm(X[at], R[at], gamma, 1e-6)
    assert torch.equal(H[at], want_H)
    hc.close(rstd[at], r[:, 0], 2 * hc.U * r[:, 0])
    hc.close(Y[at], y, 4 * hc.U * np.abs(y), dtype)
    for first in range(0, N, 8000):  # a row a workgroup: the same bits
        part = slice(first, min(first + 8000, N))
        h, out, s = torch.empty_like(X[part]), torch.empty_like(X[part]), torch.empty_like(rstd[part])
        c, sc = maxk.mx_empty(h.shape[0], dim, 8)
        maxk.maxk_rms_norm(X[part], gamma, out, c, sc, R[part], h, s)
        assert torch.equal(h, H[part]) and torch.equal(out, Y[part]) and torch.equal(s, rstd[part])
        assert torch.equal(c, codes[part]) and torch.equal(sc, scales[part])
