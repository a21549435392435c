"""Plain forms in 64 bits of the operators between a layer's output and a token: numpy, a row at a time, from the definitions."""
import math

import numpy as np

BLOCK = 128


def e4m3_values() -> np.ndarray:
    """The 256 values of the format: sign, 4 exponent bits (bias 7), 3 mantissa bits, 0x7F / 0xFF NaN."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out[c] = math.nan if c & 127 == 127 else (-v if s else v)
    return out


E4M3 = e4m3_values()
_POSITIVE = E4M3[:127]


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Codes of |x| <= 448, nearest, ties to the even code."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == _POSITIVE[hi], hi, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_columns(d: int) -> int:
    return 4 * ((d + 511) // 512)


def quantize(x: np.ndarray):
    """(codes [rows x d], scale bytes [rows x scale_columns]) of x in 64 bits."""
    rows, d = x.shape
    codes = np.empty((rows, d), np.uint8)
    scales = np.full((rows, scale_columns(d)), 127, np.uint8)
    for r in range(rows):
        for b in range((d + BLOCK - 1) // BLOCK):
            v = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(v).all():
                scales[r, b], codes[r, b * BLOCK:(b + 1) * BLOCK] = 255, 127
                continue
            most, e = np.abs(v).max(), 0
            if most > 0:
                e = -126
                while most > 448 * 2.0 ** e:
                    e += 1
            scales[r, b] = e + 127
            codes[r, b * BLOCK:(b + 1) * BLOCK] = to_e4m3(v / 2.0 ** e)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    d = codes.shape[1]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return E4M3[codes] * np.repeat(s, BLOCK, axis=1)[:, :d]


def sample_row(z, u, t=1.0, k=0, p=1.0, m=0.0):
    """(place, probability) of one row: everything sorted, everything in 64 bits."""
    z = np.asarray(z, dtype=np.float64)
    u = min(max(float(u), 0.0), 1 - 2.0 ** -24)
    places = np.flatnonzero(z > -np.inf)
    if places.size == 0:
        return -1, 0.0
    order = places[np.argsort(-z[places], kind="stable")]
    if not t > 0:
        return int(order[0]), 1.0
    top = z[order[0]]
    far = np.where(z[order] == top, 0.0, top - z[order])
    c = max(math.log2(math.e) / t, 1e-300)
    near = far * c <= 64
    order, w = order[near], np.exp2(-far[near] * c)
    if k > 0:
        order, w = order[:k], w[:k]
    if p < 1:
        ahead = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        stay = ahead < p * w.sum()
        stay[0] = True
        order, w = order[stay], w[stay]
    if m > 0:
        stay = w >= min(m, 1.0)
        order, w = order[stay], w[stay]
    run = np.cumsum(w)
    at = min(int(np.searchsorted(run, u * run[-1], side="right")), len(w) - 1)
    return int(order[at]), float(w[at] / run[-1])
