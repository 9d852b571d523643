"""8-bit rows and matrices in numpy, 64 bits: e4m3 elements with a power-of-two
scale per block of 128 (rows) or 128 x 128 (matrices).

The e4m3 numbers are written out as a table (4 exponent bits with bias 7, 3
mantissa bits, subnormals of 2^-9, 0x7f = NaN) and an element is found by its
neighbours in the table; nothing here is shared with the kernels.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
# values of the codes 0x00..0x7e
TABLE = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10)
                  for c in range(127)])


def encode(v: np.ndarray) -> np.ndarray:
    """Codes of the e4m3 numbers nearest to v (64 bits, |v| <= 448; ties to the even
    code); what is not finite becomes NaN."""
    v = np.asarray(v, np.float64)
    a = np.abs(np.where(np.isfinite(v), v, 0.0))
    hi = np.minimum(np.searchsorted(TABLE, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = TABLE[hi] - a, a - TABLE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code + np.where(np.signbit(v), 128, 0)
    return np.where(np.isfinite(v), code, 0x7F).astype(np.uint8)


def decode(code: np.ndarray) -> np.ndarray:
    c = np.asarray(code, np.uint8)
    v = np.append(TABLE, np.nan)[c & 127]
    return np.where(c & 128, -v, v)


def scale_byte(top: np.ndarray) -> np.ndarray:
    """e + 127 for blocks of largest finite magnitude `top`."""
    top = np.asarray(top, np.float64)
    m, x = np.frexp(top)                 # top = m 2^x, 1/2 <= m < 1
    e = np.where(m <= 0.875, x - 9, x - 8)  # 448 = 0.875 2^9
    return np.where(top > 0, np.maximum(e, -127), -127).astype(np.int64) + 127


def pad(n: int, to: int) -> int:
    return -(-n // to) * to


def _tops(v: np.ndarray) -> np.ndarray:
    return np.abs(np.where(np.isfinite(v), v, 0.0))


def quant_rows(x: np.ndarray):
    """Rows [R][K] to (codes [R][pitch], scale bytes [R][blocks])."""
    R, K = x.shape
    v = np.zeros((R, pad(K, BLOCK)))
    v[:, :K] = x
    b = v.reshape(R, v.shape[1] // BLOCK, BLOCK)
    s = scale_byte(_tops(b).max(2))
    with np.errstate(invalid="ignore"):
        q = encode(b * 2.0 ** (127.0 - s)[:, :, None])
    return q.reshape(R, -1), s.astype(np.uint8)


def row_values(q: np.ndarray, s: np.ndarray, K: int) -> np.ndarray:
    b = decode(q).reshape(q.shape[0], q.shape[1] // BLOCK, BLOCK)
    return (b * 2.0 ** (s[:, :b.shape[1]].astype(np.float64) - 127)[:, :, None]) \
        .reshape(q.shape)[:, :K]


def quant_matrix(W: np.ndarray):
    """A matrix [N][K] to (codes [N][pitch], scale bytes [ceil(N / 128)][blocks])."""
    N, K = W.shape
    v = np.zeros((pad(N, BLOCK), pad(K, BLOCK)))
    v[:N, :K] = W
    b = v.reshape(v.shape[0] // BLOCK, BLOCK, v.shape[1] // BLOCK, BLOCK)
    s = scale_byte(_tops(b).max((1, 3)))
    with np.errstate(invalid="ignore"):
        q = encode(b * 2.0 ** (127.0 - s)[:, None, :, None])
    return q.reshape(v.shape)[:N], s.astype(np.uint8)


def matrix_values(q: np.ndarray, s: np.ndarray, K: int) -> np.ndarray:
    s = np.repeat(s, BLOCK, 0)[:q.shape[0]]
    return row_values(q, s, K)


def round_trip(x: np.ndarray) -> np.ndarray:
    return row_values(*quant_rows(x), x.shape[1])


def neighbours(lo: np.ndarray, hi: np.ndarray):
    """The least and largest value that rows take when each element lies anywhere in
    [lo, hi] before it is quantised.  A block's scale then lies between that of its
    least and of its largest possible top (those and the next ones are tried); the
    stored value is monotonic in the
    element for each scale."""
    tl = np.where((lo <= 0) & (hi >= 0), 0.0, np.minimum(np.abs(lo), np.abs(hi)))
    th = np.maximum(np.abs(lo), np.abs(hi))
    R, K = lo.shape
    nb = -(-K // BLOCK)

    def exponents(t):
        z = np.zeros((R, nb * BLOCK))
        z[:, :K] = t
        return scale_byte(z.reshape(R, nb, BLOCK).max(2))

    el, eh = exponents(tl), exponents(th)
    out = []
    for v, pick in ((lo, np.minimum), (hi, np.maximum)):
        best = None
        for e in [el] + [np.maximum(eh - i, el) for i in range(4)]:
            two = np.repeat(2.0 ** (e.astype(np.float64) - 127), BLOCK, 1)[:, :K]
            x = decode(encode(np.clip(v / two, -448, 448))) * two
            best = x if best is None else pick(best, x)
        out.append(best)
    return out
