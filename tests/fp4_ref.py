"""4-bit blocks in numpy, for the tests: e2m1 values by their own table, scales by exact comparison, scale bytes by their
place in the tiles."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_code(v):
    """Codes of float64 values of magnitude at most 6, nearest, ties to the even code."""
    a = np.minimum(np.abs(v), 6.0)
    hi = np.clip(np.searchsorted(VALUES, a), 0, 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - VALUES[lo], VALUES[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    return (code | (np.signbit(v).astype(np.int64) << 3)).astype(np.uint8)


def e2m1_value(code):
    v = VALUES[code.astype(np.int64) & 7]
    return np.where(code & 8, -v, v)


def scale_byte(amax):
    """Least s >= 0 with amax <= 6 2^(s - 127); 255 for an infinity or NaN."""
    if not np.isfinite(amax):
        return 255
    s = 0
    while amax > 6.0 * 2.0 ** (s - 127):
        s += 1
    return s


def quantize(x):
    """(codes [rows x cols], scale bytes [rows x blocks], values) of float64 x."""
    rows, K = x.shape
    kb = -(-K // 32)
    code, s, val = np.zeros((rows, K), np.uint8), np.zeros((rows, kb), np.uint8), np.zeros((rows, K))
    for j in range(kb):
        at = slice(j * 32, min(K, (j + 1) * 32))
        for i in range(rows):
            b = x[i, at]
            s[i, j] = scale_byte(np.abs(b).max() if np.isfinite(b).all() else np.nan)
            if s[i, j] == 255:
                val[i, at] = np.nan
                continue
            code[i, at] = e2m1_code(b * 2.0 ** (127 - int(s[i, j])))
            val[i, at] = e2m1_value(code[i, at]) * 2.0 ** (int(s[i, j]) - 127)
    return code, s, val


def unpack(q, cols):
    """Codes [rows x cols] of the bytes, and those past cols."""
    both = np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)
    return both[:, :cols], both[:, cols:]


def scale_bytes(scale, rows, cols):
    """The scale bytes [rows x ceil(cols / 32)] out of their tiles [row tiles x column tiles x 512]."""
    r, b = np.meshgrid(np.arange(rows), np.arange(-(-cols // 32)), indexing="ij")
    return scale[r // 128, b // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4]


def gelu(u):
    from scipy.special import erfc
    return 0.5 * u * erfc(-u / np.sqrt(2.0))
