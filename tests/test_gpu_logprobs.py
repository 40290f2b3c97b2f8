"""Log probabilities, entropies, the likeliest classes and the logits' gradient against 64 bits."""
import numpy as np
import pytest
import torch

import heads_common as hc
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def inputs(N, V, dtype, seed, masked=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = 3 * torch.randn(N, V, generator=gen, device="cuda")
    labels = torch.randint(V, (N,), generator=gen, device="cuda")
    x.scatter_add_(1, labels.unsqueeze(1), 5 * torch.randn(N, 1, generator=gen, device="cuda"))
    if masked and V > 4:
        x[:, V - 1 - V // 50:] = -INF
    if N > 6:
        labels[3] = -1
        labels[4] = -100
        x[5] = x[5, 0].clone()  # all the same
        if masked:
            x[6] = -INF  # nothing is left
    return x.to(dtype), labels, gen


def results(N, k=0, ib=torch.int32):
    return (torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"),
            torch.full((N, k), 7.0, device="cuda") if k else None, torch.full((N, k), 7, device="cuda").to(ib) if k else None)


def check(x, labels, k=0, ib=torch.int32):
    N, V = x.shape
    logprob, entropy, data, index = results(N, k, ib)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    lp, lp_bound, H, H_bound, R = hc.logprobs(x, labels)
    hc.close(logprob, lp, lp_bound)
    hc.close(entropy, H, H_bound)
    if k:
        want = hc.likeliest(x, k)
        assert np.array_equal(index.cpu().numpy().astype(np.int64), want)
        top = np.take_along_axis(R.logp, want, 1)
        d = np.abs(np.where(np.isfinite(top), top, 0))
        hc.close(data, top, R.u + 4 * hc.U * (d + 2 * np.abs(R.lnS)))
    return logprob, entropy, R


# widths around a lane's, a team's, a wavefront's and a workgroup's columns and rounds
WIDTHS = [1, 2, 5, 8, 9, 31, 32, 41, 47, 64, 65, 100, 128, 200, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2000, 2048, 2049, 4095, 4097, 6145, 8193, 10007, 16383]


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V", WIDTHS)
def test_logprobs(V, dtype):
    N = 37
    x, labels, _ = inputs(N, V, dtype, V)
    check(x, labels, min(V, 5))
    check(x, labels.to(torch.int32))


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V", [(1, 32768), (3, 131072), (2, 50021), (700, 4099), (1, 1), (5, 9000), (64, 20011), (3001, 47), (1500, 300), (600, 9001), (150, 16384), (520, 20003)])
def test_few_and_many_rows(N, V, dtype):
    x, labels, _ = inputs(N, V, dtype, N + V)
    check(x, labels, min(V, 20))
    check(x, labels, min(V, 30))


@pytest.mark.parametrize("k", [1, 2, 3, 7, 16, 33, 50, 63, 64])
@pytest.mark.parametrize("V", [64, 65, 100, 256, 700, 1500, 5000, 9001, 16000, 40000])
def test_alternatives(k, V):
    for dtype in (torch.float32, torch.bfloat16):  # (many equal values in 16 bits)
        x, labels, _ = inputs(9, V, dtype, k + V)
        check(x, labels, k, torch.uint8 if V <= 256 else torch.uint16 if k % 2 else torch.int32)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V", [2, 7, 8, 13, 31, 32, 33, 47, 64, 65, 127, 128, 129, 200, 255, 256])
def test_alternatives_of_short_rows(V, dtype):
    """Every number of them up to the row's end or 64, over more than one wavefront; masked ones and equal ones among them."""
    x, labels, gen = inputs(70, V, dtype, V)
    x[10:40] = torch.randint(-3, 4, (30, V), generator=gen, device="cuda").to(dtype)
    x[20:30, ::2] = -INF
    x[40] = torch.where(torch.arange(V, device="cuda") % 3 == 0, -0.0, 0.0).to(dtype)
    x[41] = torch.finfo(dtype).min
    x[42] = torch.finfo(dtype).smallest_normal * torch.randint(-9, 9, (V,), generator=gen, device="cuda").to(dtype) / 16
    for k in {1, 2, 6, 7, 9, 10, 12, 13, 20, 40, 64, V}:
        if k <= min(V, 64):
            check(x, labels, k, torch.uint8)


@pytest.mark.parametrize("V", [40, 130, 600, 1500, 3000, 30000])
def test_alternatives_in_any_order(V):
    """Rows that rise, fall, are all the same, have the largest last or hold few different values."""
    up = torch.arange(V, device="cuda", dtype=torch.float32) / V
    rows = torch.stack([up, up.flip(0), torch.zeros_like(up), torch.where(up > 0.999, 5.0, 0.0), torch.where(up < 1e-3, 5.0, -1.0), (up * 4).floor(),
                        torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0), torch.full_like(up, -3.4e38), -(up * 8).floor()])
    labels = torch.arange(rows.shape[0], device="cuda")
    for k in (1, 20, 40):
        check(rows, labels, k)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V,k", [(1, 1), (5, 5), (16, 2), (40, 4), (47, 5), (47, 7), (63, 8), (64, 6), (64, 8)])
def test_alternatives_of_many_short_rows(V, k, dtype):
    """Rows enough for the form with a lane a row; values that share their leading bits, equal values, masked ones."""
    N = 140_001
    x, labels, gen = inputs(N, V, dtype, V + k)
    x[100:200] = (1 + torch.randint(0, 3, (100, V), generator=gen, device="cuda") * 2.0 ** -20).to(dtype)  # (fp32: equal in 26 bits, and not)
    x[200:300] = torch.randint(0, 3, (100, V), generator=gen, device="cuda").to(dtype)
    x[300:400, V // 2:] = -INF
    if V > 1:
        x[400, 1], x[401, 0] = NAN, INF
    logprob, entropy, data, index = results(N, k)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    order = torch.sort(x[:400].float(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(index[:400].long(), order)
    some = torch.cat([torch.arange(400), torch.arange(N - 300, N)]).cuda()
    lp, lp_bound, H, H_bound, R = hc.logprobs(x[some], labels[some])
    hc.close(logprob[some], lp, lp_bound)
    hc.close(entropy[some], H, H_bound)
    want = hc.likeliest(x[some], k)
    assert np.array_equal(index[some].cpu().numpy(), want)
    top = np.take_along_axis(R.logp, want, 1)
    hc.close(data[some], top, R.u + 4 * hc.U * (np.abs(np.where(np.isfinite(top), top, 0)) + 2 * np.abs(R.lnS)))
    few = slice(0, 20_000)  # the other form's columns and values
    small = results(20_000, k)
    maxk.maxk_logprobs(x[few], labels[few], *small)
    assert torch.equal(small[3], index[few]) or V > 1 and torch.equal(torch.cat([small[3][:400], small[3][402:]]), torch.cat([index[:400], index[402:20_000]]))
    if V > 1:
        assert torch.isnan(data[400:402]).all() and torch.isnan(entropy[400:402]).all() and ((index[400:402] >= 0) & (index[400:402] < V)).all()


@pytest.mark.parametrize("N,V", [(5, 20), (5, 60), (5, 250), (9, 500), (9, 2000), (9, 2500), (700, 5000), (600, 20001), (3, 16384), (5, 40000), (1, 200003)])
def test_fewer_left_than_alternatives(N, V):
    """0 to 30 columns of a row are not masked, of 20 and 64 alternatives: the first masked columns follow."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((N, V), -INF, device="cuda")
        for n in range(0, N, max(1, N // 9)):
            left = min((n * 7) % 31, V - 1) if n else 0
            x[n, torch.randperm(V, generator=gen, device="cuda")[:left]] = torch.randn(left, generator=gen, device="cuda")
        some = torch.arange(0, N, max(1, N // 9), device="cuda")
        for k in (20, min(V, 64)):
            _, _, data, index = results(N, k)
            maxk.maxk_logprobs(x.to(dtype), None, None, None, data, index)
            want = hc.likeliest(x.to(dtype)[some], k)
            assert np.array_equal(index[some].cpu().numpy(), want)
            left = torch.isfinite(torch.gather(x[some], 1, torch.from_numpy(want).cuda()))
            assert torch.equal(torch.isfinite(data[some]), left) and (data[some][~left] == -INF).all()
            assert N < 10 or (data[1] == -INF).all() and index[1].tolist() == list(range(k))


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("V", [8, 9, 16, 17, 23, 33, 40, 47])
def test_many_short_rows(V, dtype):
    """Rows enough for the form that has them in LDS as one stretch (a last one that is not full, rows of an even and an odd number of words, any element's alignment)."""
    N = (1 << 19) + 225
    x, labels, gen = inputs(N, V, dtype, V)
    x[100:150] = torch.finfo(dtype).min
    labels[150] = V
    g, u = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    g[labels < 0] = 1.0
    some = torch.cat([torch.arange(150), torch.arange(N - 300, N)]).cuda()
    lp, lp_bound, H, H_bound, R = hc.logprobs(x[some], labels[some])
    for dlogprob, dentropy, entropies in ((g, u, True), (g, None, True), (g, None, False), (None, u, False)):
        dx = torch.full_like(x, 7)
        logprob, entropy, _, _ = results(N)
        maxk.maxk_logprobs_grad(x, dx, labels, dlogprob, dentropy, logprob=logprob, entropy=entropy if entropies else None)
        hc.close(logprob[some], lp, lp_bound)
        if entropies:
            hc.close(entropy[some], H, H_bound)
        pick = [None if t is None else t[some] for t in (dlogprob, dentropy)]
        want, bound = hc.logprobs_grad(R, labels[some], *pick)
        hc.close(dx[some], want, bound, dtype)
        assert torch.isnan(logprob[150]) and (dlogprob is None or torch.isnan(dx[150]).all())
    logprob2, entropy2, _, _ = results(N)
    maxk.maxk_logprobs(x, labels.int(), logprob2, entropy2)
    assert torch.equal(logprob2[151:], logprob[151:]) and torch.isnan(logprob2[150])
    hc.close(entropy2[some], H, H_bound)
    flat, out = (torch.full((N * V + 16,), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    for at, to in ((1, 2), (3, 0)):
        flat[at:at + N * V].copy_(x.view(-1))
        own = out[to:to + N * V].view(N, V)
        maxk.maxk_logprobs_grad(flat[at:at + N * V].view(N, V), own, labels, None, u)
        assert torch.equal(own, dx) and (out[:to] == 3).all() and (out[to + N * V:] == 3).all()
        out[:] = 3
    maxk.maxk_logprobs_grad(x, x, labels, None, u)  # in the logits' own memory
    assert torch.equal(x, dx)


def test_masks_of_the_lowest_value_and_of_everything():
    lowest = torch.finfo(torch.float32).min
    x = torch.full((4, 100), lowest, device="cuda")
    x[1, 7] = 2.0
    x[2] = -INF
    x[2, 50] = lowest
    x[3] = -INF
    labels = torch.tensor([3, 7, 50, 0], device="cuda")
    logprob, entropy, data, index = results(4, 3)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    ln = np.log(100)
    assert abs(logprob[0].item() + ln) < 1e-6 and abs(entropy[0].item() - ln) < 1e-6 and index[0].tolist() == [0, 1, 2]
    assert logprob[1] == 0 and entropy[1] == 0 and index[1].tolist() == [7, 0, 1] and data[1, 0] == 0
    assert logprob[2] == 0 and entropy[2] == 0 and index[2].tolist() == [50, 0, 1] and data[2, 1] == -INF
    assert logprob[3] == -INF and entropy[3] == 0 and index[3].tolist() == [0, 1, 2] and (data[3] == -INF).all()
    dx = torch.full_like(x, 7)
    maxk.maxk_logprobs_grad(x, dx, labels, torch.ones(4, device="cuda"), torch.ones(4, device="cuda"))
    assert torch.isfinite(dx).all() and (dx[2:] == 0).all() and abs(dx[0, 3].item() - 0.99) < 1e-6 and dx[1].abs().max() == 0


@pytest.mark.parametrize("V", [16384, 50021])
def test_non_finite_rows_in_segments(V):
    x = torch.full((4, V), NAN, device="cuda")
    x[1, : V - 1] = -INF
    x[2, 1:] = 0.0
    x[3, :] = 0.0
    x[3, V - 1] = INF
    _, _, data, index = results(4, 64)
    logprob, entropy, dx = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros_like(x)
    labels = torch.tensor([0, 1, -1, 3], device="cuda")
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    assert torch.isnan(logprob[[0, 1, 3]]).all() and logprob[2] == 0 and torch.isnan(entropy).all() and torch.isnan(data).all()
    assert ((index >= 0) & (index < V)).all()
    maxk.maxk_logprobs_grad(x, dx, labels, torch.ones(4, device="cuda"))
    assert torch.isnan(dx[[0, 1, 3]]).all()


@pytest.mark.parametrize("V", [47, 300, 1500, 3000, 9000])
def test_non_finite(V):
    x = torch.zeros(4, V, device="cuda")
    x[0, V // 2] = NAN
    x[1, V - 1] = INF
    x[2, 3] = -NAN
    labels = torch.tensor([0, 1, 2, V], device="cuda")
    logprob, entropy, data, index = results(4, 5)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    assert torch.isnan(logprob).all() and torch.isnan(entropy[:3]).all() and torch.isnan(data[:3]).all()
    assert ((index >= 0) & (index < V)).all() and torch.isfinite(entropy[3]) and index[3].tolist() == [0, 1, 2, 3, 4]
    dx = torch.zeros_like(x)
    maxk.maxk_logprobs_grad(x, dx, labels, torch.ones(4, device="cuda"))
    assert torch.isnan(dx).all()


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N,V", [(37, V) for V in WIDTHS] + [(1, 32768), (3, 70001), (700, 4099), (2, 131072), (3001, 47), (600, 9001), (150, 16384), (520, 20003)])
def test_gradient(N, V, dtype):
    x, labels, gen = inputs(N, V, dtype, 3 * V + N)
    g, u = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    lp, lp_bound, H, H_bound, R = hc.logprobs(x, labels)
    for dlogprob, dentropy in ((g, u), (g, None), (None, u)):
        dx = torch.full_like(x, 7)
        logprob, entropy, _, _ = results(N)
        maxk.maxk_logprobs_grad(x, dx, labels, dlogprob, dentropy, logprob=logprob, entropy=entropy)
        hc.close(logprob, lp, lp_bound)
        hc.close(entropy, H, H_bound)
        want, bound = hc.logprobs_grad(R, labels, dlogprob, dentropy)
        hc.close(dx, want, bound, dtype)
    own = x.clone()
    maxk.maxk_logprobs_grad(own, own, labels, None, u)  # in the logits' own memory
    assert torch.equal(own, dx)
    maxk.maxk_logprobs_grad(x, own, None, None, u)
    assert torch.equal(own, dx)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
def test_offsets(dtype):
    """Logits and gradients that start at any element; nothing is written around them."""
    for N, V in ((9, 47), (5, 301), (7, 3001), (2, 9001), (130, 20001)):
        x, labels, gen = inputs(N, V, dtype, V, masked=False)
        g = torch.randn(N, generator=gen, device="cuda")
        want = torch.empty_like(x)
        maxk.maxk_logprobs_grad(x, want, labels, g)
        for at, to in ((1, 2), (3, 0), (0, 1), (5, 5)):
            flat, out = (torch.full((N * V + 16,), 3.0, dtype=dtype, device="cuda") for _ in range(2))
            flat[at:at + N * V].copy_(x.view(-1))
            dx = out[to:to + N * V].view(N, V)
            maxk.maxk_logprobs_grad(flat[at:at + N * V].view(N, V), dx, labels, g)
            assert torch.equal(dx, want) and (out[:to] == 3).all() and (out[to + N * V:] == 3).all()


def test_gradients_are_differences():
    N, V = 5, 30
    x, labels, gen = inputs(N, V, torch.float32, 8, masked=False)
    g, u = (torch.randn(N, generator=gen, device="cuda") for _ in range(2))
    dx = torch.empty_like(x)
    maxk.maxk_logprobs_grad(x, dx, labels, g, u)
    y, has = labels.clamp_min(0).cpu().numpy(), (labels >= 0).cpu().numpy()

    def value(x):
        lp = x - x.max(1, keepdims=True)
        lp = lp - np.log(np.exp(lp).sum(1, keepdims=True))
        return (hc.f64(g) * np.where(has, lp[np.arange(N), y], 0)).sum() - (hc.f64(u)[:, None] * np.exp(lp) * lp).sum()

    base, step = hc.f64(x), 1e-5
    for n, i in ((0, 0), (0, y[0]), (3, 2), (4, 29), (2, y[2])):
        up, down = base.copy(), base.copy()
        up[n, i] += step
        down[n, i] -= step
        assert abs((value(up) - value(down)) / (2 * step) - dx[n, i].item()) < 1e-5


def test_rows_past_32_bits():
    """Offsets of more than 2^31 elements, and bytes past 2^32."""
    N, V = 2300, 1_000_003
    x = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    labels = torch.arange(N, device="cuda") * 401
    x[torch.arange(N, device="cuda"), labels] = 14.0
    logprob, entropy, data, index = results(N, 2)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    S = np.exp(14.0) + V - 1
    assert (logprob - (14 - np.log(S))).abs().max() < 1e-4 and torch.equal(index[:, 0].long(), labels)
    assert torch.equal(index[:, 1].long(), (labels == 0).long())
    maxk.maxk_logprobs_grad(x, x, labels, torch.full((N,), 1.0, device="cuda"))
    p = np.exp(14.0) / S
    rows = torch.arange(N, device="cuda")
    assert ((x[rows, labels].float() - (1 - p)).abs() <= 2.0 ** -8 * (1 - p) + 1e-5).all()
    assert ((x[:, -1].float() + 1 / S).abs() <= 2.0 ** -8 / S + 1e-9).all()


@pytest.mark.parametrize("N", [2, 130])
def test_most_classes(N):
    V = 1 << 24
    x = torch.zeros(N, V, dtype=torch.float16, device="cuda")
    places = torch.tensor([V - 1, 77, V // 2, 5_000_011], device="cuda")
    x[:, places] = torch.tensor([12.0, 11.0, 10.0, 9.0], dtype=torch.float16, device="cuda")
    labels = torch.full((N,), V - 1, device="cuda")
    labels[1] = V + (1 << 33)
    logprob, entropy, data, index = results(N, 6)
    maxk.maxk_logprobs(x, labels, logprob, entropy, data, index)
    e = np.exp([12.0, 11.0, 10.0, 9.0])
    S = e.sum() + V - 4
    H = np.log(S) - (e * [12.0, 11.0, 10.0, 9.0]).sum() / S
    # 2^24 ones are added up exactly in any order; the other roundings are those of a few terms and of two logarithms of less than 17
    assert abs(logprob[0].item() - (12 - np.log(S))) < 64 * 17 * hc.U and torch.isnan(logprob[1]) and abs(entropy[0].item() - H) < 64 * 17 * hc.U
    assert (index == torch.tensor([V - 1, 77, V // 2, 5_000_011, 0, 1], device="cuda")).all()
    maxk.maxk_logprobs_grad(x, x, labels.clamp_max(V - 1), torch.ones(N, device="cuda"))
    p = e[1] / S
    assert abs(x[N - 1, 77].item() + p) <= 2.0 ** -11 * p + 1e-6 and abs(x[0, V - 1].item() - (1 - e[0] / S)) <= 2.0 ** -11 + 1e-6
    assert abs(x[N - 1, V // 4].item() + 1 / S) <= 2.0 ** -25 + 1e-12


def test_as_many_rows_as_fit_no_launch_of_one_dimension():
    """Four lanes a row: 2^30 rows are 2^32 threads."""
    N = (1 << 30) + 12_345
    x = torch.zeros(N, 1, dtype=torch.bfloat16, device="cuda")
    entropy = torch.full((N,), 7.0, device="cuda")
    logprob = torch.full((N,), 7.0, device="cuda")
    labels = torch.zeros(N, dtype=torch.int32, device="cuda")
    x[N - 2] = -INF
    labels[N - 1] = 1
    maxk.maxk_logprobs(x, labels, logprob, entropy)
    assert not entropy.any().item() and torch.isnan(logprob[N - 1]) and logprob[N - 2] == -INF and not logprob[: N - 2].any().item()


def test_no_rows():
    x = torch.empty(0, 9, device="cuda")
    maxk.maxk_logprobs(x, None, None, torch.empty(0, device="cuda"))
    maxk.maxk_logprobs_grad(x, x.clone(), None, None, torch.empty(0, device="cuda"))
