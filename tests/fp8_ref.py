"""8-bit blocks in numpy, for the tests: e4m3 values by their own table, scales by exact comparison."""
import numpy as np


def e4m3_table():
    """The values of the codes 0 .. 126 (non-negative finite), ascending."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append((m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


TABLE = e4m3_table()


def e4m3_code(v):
    """Codes of float64 values of magnitude at most 448 (1.0625 past it rounds down to it), nearest, ties to the
    even code; NaN is 127."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(TABLE, np.nan_to_num(a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - TABLE[lo], TABLE[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(a), 127, np.where(a >= TABLE[126], 126, code))
    return (code | (np.signbit(v).astype(np.int64) << 7)).astype(np.uint8)


def e4m3_value(code):
    c = code.astype(np.int64)
    v = np.append(TABLE, np.nan)[c & 127]
    return np.where(c & 128, -v, v)


def scale_byte(amax):
    """Least s >= 0 with amax <= 448 2^(s - 127); 255 for an infinity or NaN."""
    if not np.isfinite(amax):
        return 255
    s = 0
    while amax > 448.0 * 2.0 ** (s - 127):
        s += 1
    return s


def quantize(x, block_rows):
    """(q codes [rows x pitch], scale bytes [row blocks x K blocks], values) of float64 x."""
    rows, K = x.shape
    kb, rb = -(-K // 128), -(-rows // block_rows)
    q = np.zeros((rows, kb * 128), np.uint8)
    s = np.zeros((rb, kb), np.uint8)
    val = np.zeros((rows, K))
    for i in range(rb):
        for j in range(kb):
            at = (slice(i * block_rows, min(rows, (i + 1) * block_rows)), slice(j * 128, min(K, (j + 1) * 128)))
            b = x[at]
            s[i, j] = scale_byte(np.abs(b).max() if np.isfinite(b).all() else np.nan)
            if s[i, j] == 255:
                val[at] = np.nan
                q[at] = 127
                continue
            q[at] = e4m3_code(b * 2.0 ** (127 - int(s[i, j])))
            val[at] = e4m3_value(q[at]) * 2.0 ** (int(s[i, j]) - 127)
    return q, s, val


def gelu(u):
    from scipy.special import erfc
    return 0.5 * u * erfc(-u / np.sqrt(2.0))
