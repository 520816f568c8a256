"""Plain implementations of the paged operators in 64 bits (numpy): the page format, appending, and the attention."""
from __future__ import annotations

import numpy as np

S_OVERFLOW, S_BAD_TABLE = 1, 2


def e4m3_values() -> np.ndarray:
    """The values of the 256 codes: sign, four exponent bits (bias 7), three fraction bits; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = np.nan if (e, m) == (15, 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[b] = -v if b & 128 else v
    return out


VALUES = e4m3_values()
GRID = VALUES[:127]                                   # 0 .. 448, ascending with the code


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; beyond 448 the largest code; NaN stays NaN; the sign of zero stays."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.clip(np.searchsorted(GRID, a), 1, 126)
    lo = hi - 1
    up = (GRID[hi] - a < a - GRID[lo]) | ((GRID[hi] - a == a - GRID[lo]) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8)
    code = np.where(np.isnan(x), 0x7f, code)
    return (code | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def same_codes(a: np.ndarray, b: np.ndarray) -> bool:
    """Equal bytes, any NaN equal to any NaN."""
    nan = ((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f)
    return bool(np.all(nan | (a == b)))


def scale_value(byte) -> np.ndarray:
    return np.where(np.asarray(byte) == 255, np.nan, np.exp2(np.asarray(byte, dtype=np.float64) - 127))


def needed(x: np.ndarray) -> int:
    """Byte of the smallest scale 2^n, n >= -126, whose 448-fold reaches every finite element."""
    a = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    n = -126
    while a > 448.0 * 2.0 ** n:
        n += 1
    return n + 127


class Pool:
    """One pool on the host: codes uint8 [n_pages, Hkv, P, D] and scale bytes [n_pages, Hkv], for K and V."""

    def __init__(self, k, v, ks, vs):
        self.k, self.v, self.ks, self.vs = (np.array(x) for x in (k, v, ks, vs))

    def append(self, page, slot, x_k, x_v):
        """Rows of one sequence that go into one page, from token `slot` on: [n, Hkv, D]."""
        for codes, scales, x in ((self.k, self.ks, x_k), (self.v, self.vs, x_v)):
            for h in range(codes.shape[1]):
                e = needed(x[:, h])
                if slot:
                    was = int(scales[page, h])
                    e = max(e, was)
                    if e > was:
                        codes[page, h, :slot] = encode(VALUES[codes[page, h, :slot]] * 2.0 ** (was - e))
                scales[page, h] = e
                codes[page, h, slot:slot + len(x)] = encode(x[:, h] * 2.0 ** (127 - e))

    def tokens(self, pages, n):
        """Values of the first n tokens of a list of pages: K, V [n, Hkv, D]."""
        def take(codes, scales):
            if not len(pages):
                return np.zeros((0, codes.shape[1], codes.shape[3]))
            v = VALUES[codes[pages]] * scale_value(scales[pages])[:, :, None, None]
            return v.transpose(0, 2, 1, 3).reshape(-1, codes.shape[1], codes.shape[3])[:n]
        return take(self.k, self.ks), take(self.v, self.vs)


def append(pool: Pool, table, k, v, row_seq, row_index) -> int:
    """Rows r (k, v [rows, Hkv, D] in 64 bits) as token row_index[r] of table row row_seq[r]; consecutive rows of a sequence that share a
    page belong together.  Returns the status bits."""
    status, r, P = 0, 0, pool.k.shape[2]
    while r < len(row_seq):
        s, t = int(row_seq[r]), int(row_index[r])
        n = 1
        while r + n < len(row_seq) and row_seq[r + n] == s and row_index[r + n] == t + n and (t + n) // P == t // P:
            n += 1
        if s < 0 or s >= len(table):
            status |= S_BAD_TABLE
        elif t // P >= table.shape[1]:
            status |= S_OVERFLOW
        elif not 0 <= table[s, t // P] < len(pool.k):
            status |= S_BAD_TABLE
        else:
            pool.append(int(table[s, t // P]), t % P, k[r:r + n], v[r:r + n])
        r += n
    return status


def attend(q, scale, keys, values):
    """One row: q [Hq, D]; keys, values [n, Hkv, D].  Returns o [Hq, D] and lse [Hq]; nothing visible: 0 and -inf."""
    Hq, D = q.shape
    n, Hkv = keys.shape[:2]
    if n == 0:
        return np.zeros((Hq, D)), np.full(Hq, -np.inf)
    G = Hq // Hkv
    s = scale * np.einsum("hgd,nhd->hgn", q.reshape(Hkv, G, D), keys)
    m = s.max(axis=2, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(axis=2, keepdims=True)
    o = np.einsum("hgn,nhd->hgd", e / l, values)
    return o.reshape(Hq, D), (m + np.log(l)).reshape(Hq)


def attention_bounds(q, scale, keys, values, o, lse):
    """How far a row's o [Hq, D] (bf16) and lse [Hq] (fp32) may be from 64 bits, from the roundings that the kernel makes:
      queries   two e4m3 terms of q / 2^e with the row's largest magnitude in [128, 256): what is left of an element is at most half of
                the smallest e4m3 step (2^-10), 2^-17 of that magnitude: a score moves by scale * 2^-17 * |q|max * sum |k|
      scores    D products summed in fp32 and scaled, the maximum subtracted: (D + 4) 2^-23 of scale * sum |q k|, and 2^-22 for the exponential
      P         fp16: 2^-11 of each probability
      sums      n terms in fp32: n 2^-23
      o         bf16: 2^-8
    A relative error x of every exp(score) moves o by at most 2 x max |v|, and log of their sum by x."""
    Hq, D = q.shape
    n, Hkv = keys.shape[:2]
    if n == 0:
        return np.zeros((Hq, D)), np.zeros(Hq)
    G = Hq // Hkv
    qh = np.abs(q).reshape(Hkv, G, D)
    kmax = np.abs(keys)
    by_q = scale * 2.0 ** -17 * qh.max(axis=2) * kmax.sum(axis=2).max(axis=0)[:, None]
    by_s = (D + 4) * 2.0 ** -23 * scale * np.einsum("hgd,nhd->hgn", qh, kmax).max(axis=2)
    x = (by_q + by_s + 2.0 ** -22 + n * 2.0 ** -23).reshape(Hq)
    vmax = np.repeat(np.abs(values).max(axis=(0, 2)), G)
    return np.abs(o) * 2.0 ** -8 + ((2 * x + 2.0 ** -11) * vmax)[:, None], x + 2.0 ** -22 * np.abs(lse)
