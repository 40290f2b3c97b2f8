"""The microscaled formats' plain implementation, pinned to hand-worked values and to the formats' own properties."""
import numpy as np
import pytest

import mx_common as mx


def _round_trip(row, bits):
    X = np.array([row], dtype=np.float32)
    codes, scales = mx.quantize(X, bits)
    return mx.values(codes, scales, X.shape[1])[0], codes[0], scales[0]


def test_hand_worked_block_in_8_bits():
    # largest 1.5: unit 2^0 / 64; halfway cases go to the even code, 1.999 is 127.9 sixty-fourths and saturates
    got, codes, scales = _round_trip([1.5, 1 / 128, 3 / 128, -5 / 128, 0.0, 1.999], 8)
    assert scales.tolist() == [127] and codes[:6].tolist() == [96, 0, 2, -2, 0, 127] and not codes[6:].any()
    np.testing.assert_array_equal(got, [1.5, 0, 2 / 64, -2 / 64, 0, 127 / 64])


def test_hand_worked_block_in_4_bits():
    # largest 6: unit 2^0; 5 lies between 4 and 6 and goes to the even code (4), 0.25 to 0, 0.75 to 1, 1.75 to 2, 2.5 to 2, 3.5 to 4
    got, codes, scales = _round_trip([6, 5, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5], 4)
    np.testing.assert_array_equal(got, [6, 4, 0, 1, -1, 2, 2, -4])
    assert scales.tolist() == [127] and codes[:4].tolist() == [0x67, 0x20, 0x4A, 0xE4] and not codes[4:].any()
    # largest 7.9: above 6 saturates
    assert _round_trip([7.9, 4.9], 4)[0].tolist() == [6, 4]


@pytest.mark.parametrize("bits", [8, 4])
def test_edges_of_the_scale(bits):
    tiny, huge = np.float32(2.0 ** -149), np.finfo(np.float32).max
    for x in (0.0, tiny, 2.0 ** -127, 2.0 ** -126, 2.0 ** -125, 1.0, huge, -huge):
        got, _, scales = _round_trip([x] * 3, bits)
        assert np.isfinite(got).all() and abs(got[0] - x) <= (2.0 ** -7 if bits == 8 else 0.25) * max(abs(x), 2.0 ** -126)
    assert _round_trip([0.0], bits)[2] == [0]
    for bad in (np.inf, -np.inf, np.nan):
        got, _, scales = _round_trip([1.0] * 32 + [bad] + [2.0] * 40, bits)
        assert scales.tolist() == [127 - (0 if bits == 8 else 2), 255, 128 - (0 if bits == 8 else 2)] and np.isnan(got[32:64]).all()
        assert np.isfinite(np.delete(got, range(32, 64))).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_values_are_kept_and_errors_bounded(bits):
    rng = np.random.default_rng(3)
    X = mx.features(rng, 200, 77, spread=3.0)
    codes, scales = mx.quantize(X, bits)
    V = mx.values(codes, scales, 77)
    again = mx.quantize(V, bits)
    np.testing.assert_array_equal(mx.values(*again, 77), V)  # stored values are fixed points
    amax = np.abs(np.pad(X, ((0, 0), (0, 19))).reshape(200, 3, 32)).max(axis=2).repeat(32, axis=1)[:, :77]
    # half a step of the largest binade, or what saturation cuts off
    assert (np.abs(V - X) <= amax * (2.0 ** -6 if bits == 8 else 0.25)).all()
