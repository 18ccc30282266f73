"""MXFP4 rows written out from their definition, in 64 bits, on numpy arrays.  Shares nothing with the package."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(D):
    return -(-(D // 2 + D // 32) // 16) * 16


def quantize(x):
    """x: finite or not, [R, D] -> codes uint8 [R, D], scale bytes uint8 [R, D/32]."""
    x = np.asarray(x, dtype=np.float64)
    R, D = x.shape
    b = x.reshape(R, D // 32, 32)
    codes = np.zeros(b.shape, dtype=np.uint8)
    scales = np.zeros(b.shape[:2], dtype=np.uint8)
    for idx in np.ndindex(R, D // 32):
        v = b[idx]
        if not np.isfinite(v).all():
            scales[idx] = 255
            continue
        top = np.abs(v).max()
        e = -127 if top == 0 else min(max(int(np.frexp(top)[1]) - 1 - 2, -127), 127)
        scales[idx] = e + 127
        a = np.abs(v) / 2.0 ** e
        # the nearest of the grid; of two equally near ones the even code; beyond the grid its end
        d = np.abs(a[:, None] - GRID[None, :])
        near = d == d.min(1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)[None, :]
        code = np.where(near.sum(1) > 1, np.argmax(even, 1), np.argmax(near, 1))
        codes[idx] = code + 8 * np.signbit(v)
    return codes.reshape(R, D), scales


def pack(codes, scales):
    R, D = codes.shape
    rows = np.zeros((R, row_bytes(D)), dtype=np.uint8)
    rows[:, :D // 2] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    rows[:, D // 2:D // 2 + D // 32] = scales
    return rows


def values(rows, D):
    """float64 values that packed rows stand for."""
    c = rows[:, :D // 2]
    codes = np.stack((c & 15, c >> 4), 2).reshape(rows.shape[0], D)
    s = rows[:, D // 2:D // 2 + D // 32].astype(np.int64)
    scale = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    return v * np.repeat(scale, 32, axis=1)


def random_rows(rng, R, D, lo=118, hi=127):
    """Rows of random codes, scale bytes from lo on and below hi."""
    return pack(rng.integers(0, 16, (R, D), dtype=np.uint8), rng.integers(lo, hi, (R, D // 32), dtype=np.uint8))


def int_values(rows, D, dtype):
    """float64 values of INT8 / INT4 rows (scale * code + bias)."""
    h = rows[:, :8].copy().view(np.float32).astype(np.float64)
    if dtype == "int8":
        codes = rows[:, 8:8 + D]
    else:
        c = rows[:, 8:8 + D // 2]
        codes = np.stack((c & 15, c >> 4), 2).reshape(rows.shape[0], D)
    return h[:, :1] * codes + h[:, 1:2]


def pool(vals, offsets, mode):
    """Sums (or means) of vals between offsets, and the sums of their magnitudes."""
    n = len(offsets) - 1
    out, mag = np.zeros((n, vals.shape[1])), np.zeros((n, vals.shape[1]))
    for i in range(n):
        v = vals[offsets[i]:offsets[i + 1]]
        k = max(len(v), 1) if mode == "mean" else 1
        out[i], mag[i] = v.sum(0) / k, np.abs(v).sum(0) / k
    return out, mag
