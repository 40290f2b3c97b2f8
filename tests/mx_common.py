"""The microscaled formats and operators in 64 bits, from their definitions (NumPy; shares nothing with the library)."""
import numpy as np

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def blocks(din):
    return -(-din // BLOCK)


def quantize(X, bits):
    """(codes, scales) of a float matrix (its values taken as they are)."""
    X = np.asarray(X, dtype=np.float64)
    N, din = X.shape
    nb = blocks(din)
    B = np.zeros((N, nb * BLOCK))
    B[:, :din] = X
    B = B.reshape(N, nb, BLOCK)
    finite = np.isfinite(B).all(axis=2)
    amax = np.abs(np.where(finite[..., None], B, 0.0)).max(axis=2)
    with np.errstate(divide="ignore"):
        e = np.where(amax > 0, np.floor(np.log2(np.where(amax > 0, amax, 1.0))), -200.0)
    # log2 rounds up just below a power of two
    e = np.where((amax > 0) & (np.ldexp(1.0, np.clip(e, -400, 400).astype(int)) > amax), e - 1, e)
    e = np.maximum(e - (0 if bits == 8 else 2), -127).astype(int)
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    ratio = np.where(finite[..., None], B, 0.0) / np.ldexp(1.0, e)[..., None]
    if bits == 8:
        q = np.clip(np.rint(ratio * 64), -127, 127)
        return q.astype(np.int8).reshape(N, -1), scales
    a = np.minimum(np.abs(ratio), 6.0)
    upper = np.minimum(np.searchsorted(SIZES, a), 7)
    lower = np.maximum(upper - 1, 0)
    below, above = a - SIZES[lower], SIZES[upper] - a
    code = np.where((below < above) | ((below == above) & (lower % 2 == 0)), lower, upper)
    code = (code | (np.where(finite[..., None], np.signbit(B), False).astype(int) << 3)).reshape(N, -1)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8), scales


def values(codes, scales, din):
    """What codes and scales stand for, in 64 bits."""
    codes = np.asarray(codes)
    N = codes.shape[0]
    if codes.dtype == np.int8:
        q = codes.astype(np.float64) / 64
    else:
        table = np.concatenate([SIZES, -SIZES])
        q = np.empty((N, 2 * codes.shape[1]))
        q[:, 0::2], q[:, 1::2] = table[codes & 15], table[codes >> 4]
    unit = np.ldexp(1.0, scales.astype(int) - 127)
    unit[scales == 255] = np.nan
    return (q.reshape(N, -1, BLOCK) * unit[..., None]).reshape(N, -1)[:, :din]


def scatter(dXs, index, dout):
    dense = np.zeros((dXs.shape[0], dout))
    np.put_along_axis(dense, np.asarray(index).astype(np.int64), np.asarray(dXs, dtype=np.float64), axis=1)
    return dense


def features(rng, N, din, spread=1.0):
    """Rows and columns of different sizes, some rows and some blocks of zeros."""
    X = rng.standard_normal((N, din)) * np.exp(spread * rng.standard_normal((N, 1))) * np.exp(0.5 * spread * rng.standard_normal((1, din)))
    X[rng.random(N) < 0.05] = 0
    if din > BLOCK:
        X[rng.random(N) < 0.05, :BLOCK] = 0
    return X.astype(np.float32)


def columns(rng, N, dout, k):
    keys = rng.random((N, dout))
    return np.sort(np.argsort(keys, axis=1)[:, :k], axis=1)
