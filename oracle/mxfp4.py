"""MXFP4 weights and the products with them (oracle; test infrastructure only).

OCP Microscaling FP4: e2m1 codes, two a byte (lower column in the low nibble), with one UE8M0 scale
2^(byte - 127) for 32 columns (byte 255: NaN).  The scale rule is the e4m3 tiles' (paper section 3.1):
the smallest T >= -126 with amax <= 6 * 2^T.
"""

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def scale_exponent(amax):
    amax = np.asarray(amax, dtype=np.float64)
    t = np.full(amax.shape, -126, dtype=np.int64)
    big = amax > 6.0 * 2.0 ** -126
    t[big] = np.ceil(np.log2(amax[big] / 6.0)).astype(np.int64)
    t = np.where(big & (6.0 * np.exp2(t - 1.0) >= amax), t - 1, t)  # a rounded logarithm decides nothing
    t = np.where(big & (6.0 * np.exp2(t.astype(np.float64)) < amax), t + 1, t)
    return np.maximum(t, -126)


def encode(v):
    """Codes of |v| <= 6: nearest value, ties to the even code, sign kept."""
    v = np.asarray(v, dtype=np.float64)
    d = np.abs(np.abs(v)[..., None] - E2M1)
    best = d.min(axis=-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    return (code | np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def quant(w):
    """q [rows, cols / 2], s [rows, cols / 32] of w [rows, cols]."""
    w = np.asarray(w, dtype=np.float64)
    rows, cols = w.shape
    g = w.reshape(rows, cols // GROUP, GROUP)
    t = scale_exponent(np.abs(g).max(axis=2))
    codes = encode(g * np.exp2(-t.astype(np.float64))[..., None]).reshape(rows, cols)
    return codes[:, 0::2] | codes[:, 1::2] << 4, (t + 127).astype(np.uint8)


def dequant(q, s):
    """Values [rows, cols] (exact)."""
    q, s = np.asarray(q), np.asarray(s)
    codes = np.stack([q & 15, q >> 4], axis=-1).reshape(q.shape[0], -1)
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127.0))
    return v * np.repeat(scale, GROUP, axis=1)


def pack(q, s):
    """Tile order: tq [rows / 16, cols / 128, 64, 16], ts [rows / 32, cols / 128, 64, 2]; lane l of a tile is
    row l % 16, columns 32 * (l // 16) .. + 31, and its scales in two tiles stand side by side."""
    rows, half = q.shape
    kt = half // 64
    tq = np.zeros((rows // 16, kt, 64, 16), dtype=np.uint8)
    ts = np.zeros((rows // 32, kt, 64, 2), dtype=np.uint8)
    for lane in range(64):
        r, g = lane % 16, lane // 16
        for c in range(kt):
            tq[:, c, lane] = q[r::16, c * 64 + g * 16: c * 64 + g * 16 + 16]
            ts[:, c, lane] = s[r::16, c * 4 + g].reshape(-1, 2)
    return tq, ts


def grouped_product(x, w, offsets):
    """out[m, n] = sum_k x[m, k] w_e[n, k] in expert e's rows (float64)."""
    out = np.zeros((int(offsets[-1]), w[0].shape[0]))
    for e in range(len(offsets) - 1):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if b > a:
            out[a:b] = np.asarray(x[a:b], dtype=np.float64) @ w[e].T
    return out
