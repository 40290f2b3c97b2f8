"""The norm, log probabilities and distillation in 64 bits, from their definitions (NumPy; shares nothing with the library), and how far fp32 arithmetic may be off."""
import numpy as np
import torch

import mx_common

U = 2.0 ** -24  # half a step of fp32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # the smallest steps
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def f64(t):
    return t.detach().double().cpu().numpy()


def close(got, want, bound, dtype=torch.float32):
    """|got - want| <= bound, and the rounding to dtype of a value that is within the bound; what is not finite is the same."""
    got, want = f64(got), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    top = torch.finfo(dtype).max
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    bound = np.broadcast_to(bound, want.shape)[fine]
    g, w = got[fine], want[fine]
    room = bound + HALF_STEP[dtype] * (np.abs(w) + bound) + LEAST[dtype]
    over = (np.abs(g - w) > room) & ~(np.isinf(g) & (np.abs(w) + bound > top))
    assert not over.any(), f"{over.sum()} of {over.size} off, the worst {np.max(np.abs(g - w)[over] / room[over]):.3g} times the room"


# ---- norm ----


def norm(X, residual, gamma, eps):
    """(H as a tensor, r, y): r and y in 64 bits from the rounded H."""
    H = X if residual is None else (X.float() + residual.float()).to(X.dtype)
    h = f64(H)
    r = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    return H, r, h * r * f64(gamma)


def stored(H, gamma, eps, bits):
    """Codes and scales of y as fp32 arithmetic has it: r rounded once, two products."""
    h = f64(H)
    r = (1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)).astype(np.float32)
    y = (h.astype(np.float32) * r) * gamma.cpu().numpy()
    return mx_common.quantize(y, bits)


def norm_grad(dY, H, gamma, rstd, dH):
    """(dx, its bound, dgamma, its terms' sum of magnitudes).

    x = h r, g = dy gamma and the closing operations are a rounding each; the mean of d products adds them up over at most 32 columns of a lane, 10 steps
    between lanes and wavefronts, and 3 roundings of its factors and the division: less than 56 of Σ|g x| / d."""
    dy, h, gam, r = f64(dY), f64(H), f64(gamma), f64(rstd)[:, None]
    x, g = h * r, dy * gam
    inner, most = (g * x).mean(axis=1, keepdims=True), np.abs(g * x).mean(axis=1, keepdims=True)
    arrives = 0.0 if dH is None else f64(dH)
    dx = r * (g - x * inner) + arrives
    return dx, 56 * U * (r * (np.abs(g) + np.abs(x) * most) + np.abs(arrives)), (dy * x).sum(axis=0), np.abs(dy * x).sum(axis=0)


# ---- rows of logits ----


class Row:
    """softmax of rows of logits x times scale, where at least one is left, and the bound of what fp32 has for ln S.

    A term 2^d, d = (x - m) scale log2 e, is off by the roundings of x - m, of the constant and of their product, 3 u |d|, and by 2 u of the
    exponential; terms are added up one after the other in a lane, over 14 steps between lanes, wavefronts and segments, and each time a maximum moves a sum is multiplied by a
    factor that is off as a term is.  A lane's maximum moves at most as often as it has units of 8 columns."""

    def __init__(self, logits, scale=1.0):
        self.scale = scale
        x = f64(logits)
        self.x = x
        self.m = x.max(axis=1, keepdims=True)
        self.empty = np.isneginf(self.m)
        m = np.where(self.empty, 0.0, self.m)
        with np.errstate(invalid="ignore", over="ignore"):
            self.d = (x - m) * scale
            e = np.exp(self.d)
            self.S = e.sum(axis=1, keepdims=True)
            self.lnS = np.log(np.where(self.empty, 1.0, self.S))
            self.logp = np.where(self.empty, -np.inf, self.d - self.lnS)
            self.p = np.where(self.empty, 0.0, e / np.where(self.empty, 1.0, self.S))
            finite = np.where(self.p > 0, self.logp, 0.0)
            self.plogp = self.p * finite
            self.H = -self.plogp.sum(axis=1, keepdims=True)
            self.spread = (self.p * np.abs(np.where(self.p > 0, self.d, 0.0))).sum(axis=1, keepdims=True)
        units = -(-x.shape[1] // 2048) + 1
        self.steps = 10 * units + 32  # additions, and products where a maximum moves
        self.u = U * (self.steps + 4 * self.spread * min(units, 8))
        self.off = np.abs(np.where(np.isfinite(self.d), self.d, 0.0)) * 3 * U + 2 * U  # of a term


def logprobs(logits, labels):
    """(logprob, bound, entropy, bound, Row)."""
    R = Row(logits)
    y = labels.cpu().numpy().astype(np.int64)
    N, V = R.x.shape
    at = np.clip(y, 0, V - 1)[:, None]
    lp = np.take_along_axis(R.logp, at, 1)[:, 0]
    lp = np.where(y < 0, 0.0, np.where(y >= V, np.nan, lp))
    d = np.abs(np.where(np.isfinite(R.d), R.d, 0.0))
    lp_bound = (R.u + 4 * U * (np.take_along_axis(d, at, 1) + np.abs(R.lnS)))[:, 0]
    H_bound = (R.u * (1 + 2 * R.spread) + 6 * U * (np.abs(R.lnS) + R.spread))[:, 0]
    return lp, lp_bound, R.H[:, 0], H_bound, R


def logprobs_grad(R, labels, dlogprob, dentropy):
    """(dx, bound)."""
    N, V = R.x.shape
    y = labels.cpu().numpy().astype(np.int64) if labels is not None else np.full(N, -1)
    g = np.zeros(N) if dlogprob is None else f64(dlogprob)
    u = np.zeros((N, 1)) if dentropy is None else f64(dentropy)[:, None]
    g = np.where(y < 0, 0.0, np.where(y >= V, np.nan, g))[:, None]
    hot = np.zeros((N, V))
    inside = (y >= 0) & (y < V)
    hot[np.nonzero(inside)[0], y[inside]] = 1.0
    dx = g * (hot - R.p) - u * (R.plogp + R.p * R.H)
    dx = np.where(R.empty, np.where(np.isnan(g), np.nan, 0.0), dx)
    lp = np.abs(np.where(R.p > 0, R.logp, 0.0))
    size = np.abs(g) + np.abs(u) * (lp + R.H + np.abs(R.lnS) + R.spread)
    bound = R.p * size * (R.u * (2 + R.spread) + R.off + 8 * U) + 2 * U * hot * np.abs(g)
    return dx, np.where(np.isnan(bound), 0.0, bound)


def likeliest(logits, k):
    """Columns of the k largest logits a row, the lower column first among equals."""
    x = f64(logits)
    return np.argsort(-x, axis=1, kind="stable")[:, :k]


def distill(logits, data, index, temperature, dloss):
    """(loss, bound, dx, bound)."""
    scale = 1.0 / temperature
    R = Row(logits, scale)
    N, V = R.x.shape
    t, col = f64(data) * scale, index.cpu().numpy().astype(np.int64)
    there = (col >= 0) & (col < V) & ~np.isneginf(t)
    t = np.where(there, t, -np.inf)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = t.max(axis=1, keepdims=True)
        m = np.where(np.isneginf(m), 0.0, m)
        e = np.exp(t - m)
        total = e.sum(axis=1, keepdims=True)
        q = np.where(total > 0, e / np.where(total > 0, total, 1.0), 0.0)
        logq = np.where(q > 0, np.log(np.where(q > 0, q, 1.0)), 0.0)
        at = np.where(there, col, 0)
        logp = np.take_along_axis(R.logp, at, 1)
        terms = np.where(q > 0, q * (logq - logp), 0.0)
        loss = terms.sum(axis=1)
    k = q.shape[1]
    with np.errstate(invalid="ignore"):
        mine = np.take_along_axis(np.abs(np.where(np.isfinite(R.d), R.d, 0.0)), at, 1)
        size = (q * (np.abs(logq) + 2 * mine + np.abs(R.lnS) + np.abs(m - t.min(axis=1, where=there, initial=np.inf, keepdims=True)).clip(max=300))).sum(axis=1)
    loss_bound = R.u[:, 0] + (k + 24) * U * (1 + size + np.abs(R.lnS[:, 0]))
    spread = np.zeros((N, V))
    rows = np.repeat(np.arange(N), k)
    np.add.at(spread, (rows, at.reshape(-1)), np.where(there, q, 0.0).reshape(-1))
    w = f64(dloss)[:, None] * scale
    Q = (total > 0).astype(np.float64)
    dx = np.where(R.empty, 0.0, w * (R.p * Q - spread))
    far = np.abs(np.where(there, t - m, 0.0)).max(axis=1, keepdims=True)
    bound = np.abs(w) * (R.p * (R.u + R.off + 6 * U) + spread * U * (3 * far + k + 16))
    return loss, loss_bound, dx, bound
