"""The paged KV cache's operators from their definitions in numpy, in 64 bits, for the tests: sequences as plain arrays of
rows (Eq. 1), visibility row by row (Eq. 3), e4m3 rounding by search over the format's values."""
import numpy as np

# the finite non-negative e4m3 values in the order of their codes 0 .. 126
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def quantise_row(x):
    """(codes, byte) of one row: smallest power of two from 2^-110 up at which the largest magnitude is within 448, ties to even."""
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), 255
    e = -110
    while np.abs(x).max() > 448.0 * 2.0 ** e:
        e += 1
    y = np.abs(x) * 2.0 ** -e
    i = np.clip(np.searchsorted(E4M3, y, side="right") - 1, 0, 126)
    # (bf16 ends below 2^128: at the scale 2^120 the format's values end with 240, code 119)
    i, j = np.minimum(i, 119 if e == 120 else 126), np.minimum(i + 1, 119 if e == 120 else 126)
    up = (y - E4M3[i] > E4M3[j] - y) | ((y - E4M3[i] == E4M3[j] - y) & (i % 2 == 1))
    c = np.where(up, j, i).astype(np.uint8)
    return np.where(np.signbit(x), c | 0x80, c).astype(np.uint8), e + 127


def values(codes, byte):
    v = E4M3[np.minimum(codes & 127, 126)] * np.where(codes >= 128, -1.0, 1.0)
    return v * (np.nan if byte == 255 else 2.0 ** (byte - 127))


def places(k, m, rows):
    """(is summary, number among those) of a sequence's rows 0 .. rows - 1, by counting through Eq. 1."""
    out, text, summ = [], 0, 0
    while len(out) < rows:
        for _ in range(k):
            out.append((False, text)); text += 1
        for _ in range(m):
            out.append((True, summ)); summ += 1
    return out[:rows]


def visible(k, m, C, row, rows, text_only=False):
    """Boolean over rows 0 .. rows - 1: what row `row` sees, row by row."""
    a = np.arange(rows)
    chunk, r = a // (k + m), a % (k + m)
    text = r < k
    qc, qr = row // (k + m), row % (k + m)
    if qr < k:
        return (text & (chunk >= qc - C) & (a <= row)) | (~text & (chunk < qc - C))
    return (chunk == qc) & (a <= row) & (text | (not text_only))


def attention(q, key, val, k, m, C, first, scale, text_only=False):
    """Rows first .. of a sequence: q [n, Hq, D], key / val [first + n, Hkv, D], in 64 bits.  Returns out, lse, the sum of
    p |v| for each output (what relative roundings of p act on) and the largest sum of |q_d k_d| scale of a visible key."""
    n, Hq, D = q.shape
    G = Hq // key.shape[1]
    out, lse, mag, big = np.zeros((n, Hq, D)), np.zeros((n, Hq)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for i in range(n):
        see = visible(k, m, C, first + i, first + n, text_only)
        for h in range(Hq):
            kk, vv = key[see, h // G], val[see, h // G]
            s = scale * (kk @ q[i, h])
            top = s.max()
            p = np.exp(s - top)
            l = p.sum()
            out[i, h], lse[i, h] = (p / l) @ vv, top + np.log(l)
            mag[i, h] = (p / l) @ np.abs(vv)
            big[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, mag, big


def check(got_out, got_lse, ref, D):
    """Bounds of the kernels' arithmetic, element by element.  bf16 rounds by at most 2^-8 of the value, once each probability
    (times its value row's scale) and once the output.  A score is a sum of D products of exact bf16 (e4m3) factors in fp32:
    off by at most D 2^-24 of the sum of magnitudes `big`; that much, and 2^-20 for exponential and sums, relative on each p."""
    out, lse, mag, big = ref
    ds = (D + 8) * 2.0 ** -24 * big
    tol = 2.0 ** -8 * (1.0 + 2.0 ** -8) * (mag + np.abs(out)) + (2 * ds + 2.0 ** -19)[..., None] * mag + 1e-30
    bad = np.abs(got_out - out) > tol
    assert not bad.any(), (int(bad.sum()), float((np.abs(got_out - out) / tol).max()))
    ltol = ds + 2.0 ** -20 * (1.0 + np.abs(lse))
    assert (np.abs(got_lse - lse) <= ltol).all(), float((np.abs(got_lse - lse) / ltol).max())
