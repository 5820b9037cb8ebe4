"""The MXFP4 oracle: every code, the rounding's ties, the scale rule's borders, the tile order (CPU only)."""

import numpy as np

from oracle import mxfp4


def test_codes_round_trip_and_ties():
    v = np.concatenate([mxfp4.E2M1, -mxfp4.E2M1])
    assert mxfp4.encode(v).tolist() == list(range(16))
    ties = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}  # to the even code
    for x, c in ties.items():
        assert mxfp4.encode(x) == c and mxfp4.encode(-x) == c + 8
    grid = np.linspace(-6, 6, 4001)
    dec = mxfp4.E2M1[mxfp4.encode(grid) & 7] * np.where(mxfp4.encode(grid) & 8, -1, 1)
    nearest = np.abs(grid[:, None] - np.concatenate([mxfp4.E2M1, -mxfp4.E2M1])).min(axis=1)
    assert np.array_equal(np.abs(grid - dec), nearest)


def test_scale_rule():
    for t in (-126, -100, -3, 0, 5, 125):
        at = 6.0 * 2.0 ** t
        assert mxfp4.scale_exponent(at) == t
        if t < 125:
            assert mxfp4.scale_exponent(at * (1 + 2.0 ** -20)) == t + 1
    assert mxfp4.scale_exponent(0.0) == -126 and mxfp4.scale_exponent(2.0 ** -140) == -126


def test_quant_error_and_pack():
    rng = np.random.default_rng(0)
    w = rng.normal(size=(64, 256)) * 0.02
    q, s = mxfp4.quant(w)
    # half of the widest step (2 * 2^T, between 4 and 6) with 3 * 2^T < amax
    step = np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=1)
    assert np.all(np.abs(mxfp4.dequant(q, s) - w) <= step)
    tq, ts = mxfp4.pack(q, s)
    assert tq.shape == (4, 2, 64, 16) and ts.shape == (2, 2, 64, 2)
    assert np.array_equal(tq[1, 1, 35], q[16 + 3, 64 + 32: 64 + 48]) and ts[0, 1, 35, 1] == s[19, 4 + 2]
    assert np.array_equal(np.sort(tq.reshape(-1)), np.sort(q.reshape(-1)))


def test_largest_magnitudes():
    """From 7 * 2^125 on, values round up to 2^128, beyond bf16; the bf16 value below does not."""
    w = np.zeros((1, 128))
    w[0, 0], w[0, 32], w[0, 64] = 7 * 2.0 ** 125, -255 * 2.0 ** 120, 7 * 2.0 ** 125 - 2.0 ** 120
    d = mxfp4.dequant(*mxfp4.quant(w))
    assert d[0, 0] == 2.0 ** 128 and d[0, 32] == -2.0 ** 128 and d[0, 64] == 3 * 2.0 ** 126
