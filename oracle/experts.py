"""Block-scaled 8-bit matrices and the mixture-of-experts layer, in float64 NumPy.

Plain definitions, one block, token or expert at a time. Test infrastructure only; shares no code
with the HIP path.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
E4M3_MAX = 448.0
AMAX_MIN = 2.0 ** -60


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 e4m3 codes (sign, 4 exponent bits of bias 7, 3 fraction bits;
    no infinities, NaN at 0x7f and 0xff)."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        a = m * 2.0 ** -9 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            a = np.nan
        v[c] = -a if s else a
    return v


_VALUES = e4m3_values()


def decode_e4m3(codes) -> np.ndarray:
    return _VALUES[np.asarray(codes, dtype=np.uint8)]


def encode_e4m3(x) -> np.ndarray:
    """Nearest e4m3 code, ties to the even code; |x| up to 464 (beyond: NaN, as for NaN)."""
    x = np.asarray(x, dtype=np.float64)
    pos = _VALUES[:127]                       # ascending, codes 0 .. 126
    a = np.abs(x)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isnan(a) | (a > 464.0), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantize_fp8(x, block_rows: int):
    """Codes and float32 scales of one matrix [R][C]; the scale, its inverse and the products are
    float32 values, as the definition states."""
    x = np.asarray(x, dtype=np.float32)
    R, C = x.shape
    nr, nc = -(-R // block_rows), -(-C // BLOCK)
    codes = np.zeros((R, C), dtype=np.uint8)
    scales = np.zeros((nr, nc), dtype=np.float32)
    for i in range(nr):
        for j in range(nc):
            rows = slice(i * block_rows, min(R, (i + 1) * block_rows))
            cols = slice(j * BLOCK, min(C, (j + 1) * BLOCK))
            b = x[rows, cols]
            if not np.all(np.isfinite(b)):
                scales[i, j] = np.nan
                codes[rows, cols] = 0x7f
                continue
            a = np.float32(max(np.max(np.abs(b)), np.float32(AMAX_MIN)))
            scales[i, j] = a / np.float32(E4M3_MAX)
            codes[rows, cols] = encode_e4m3(b * (np.float32(E4M3_MAX) / a))
    return codes, scales


def spread(scales, rows: int, cols: int, block_rows: int) -> np.ndarray:
    """Every element's block scale [rows][cols], float64."""
    r = np.arange(rows) // block_rows
    c = np.arange(cols) // BLOCK
    return np.asarray(scales, dtype=np.float64)[r][:, c]


def matmul_fp8(x, xs, w, ws):
    """(y, bound): the product in float64, and sum |x| |w| of each output."""
    a = decode_e4m3(x) * spread(xs, *x.shape, 1)
    b = decode_e4m3(w) * spread(ws, *w.shape, BLOCK)
    return a @ b.T, np.abs(a) @ np.abs(b).T


def moe_route(x, w_router, k: int, bias=None, score: str = "softmax", renorm: bool = True,
              scale: float = 1.0, n_valid=None):
    """(ids, weights, keys): full sort of every token's keys; NaN last, equal keys to the lower
    expert, -0 equal to +0."""
    x, w = np.asarray(x, np.float64), np.asarray(w_router, np.float64)
    T, E = x.shape[0], w.shape[0]
    ids = np.full((T, k), -1, dtype=np.int32)
    weights = np.zeros((T, k))
    keys = np.zeros((T, E))
    with np.errstate(all="ignore"):
        for t in range(T):
            z = np.array([np.sum(x[t] * w[e]) for e in range(E)])
            if score == "sigmoid":
                p = 1.0 / (1.0 + np.exp(-z))
            else:
                e = np.exp(z - np.max(z))
                p = e / np.sum(e)
            key = z if bias is None else p + np.asarray(bias, np.float64)
            keys[t] = key
            if n_valid is not None and t >= n_valid:
                continue
            order = sorted(range(E), key=lambda e: (np.isnan(key[e]), -key[e] if
                                                    not np.isnan(key[e]) else 0.0, e))
            ids[t] = order[:k]
            c = p[ids[t]]
            if renorm:
                total = np.sum(c)
                c = c / total if total != 0.0 else np.zeros(k)
            weights[t] = scale * c
    return ids, weights, keys


def moe_ffn(x, ids, weights, gate_up, down, h_rel: float = 0.0, h_abs: float = 0.0):
    """(y, bound): the layer in float64, and how far float32 arithmetic may be off at each output:
    sums of n terms by n 2^-23 of the sum of their magnitudes (rounded or truncated at each
    step), SiLU by 2^-20 and by its slope (at most 1.1) times the error of g, h by h_rel of its
    value and h_abs when it enters the down product."""
    x = np.asarray(x, np.float64)
    T, d = x.shape
    E, _, inter, _ = gate_up.shape
    y, bound = np.zeros((T, d)), np.zeros((T, d))
    u23 = 2.0 ** -23
    for t in range(T):
        for r in range(ids.shape[1]):
            e = int(ids[t, r])
            if e < 0 or e >= E:
                continue
            G, U, D = gate_up[e, 0], gate_up[e, 1], down[e]
            g, u = G @ x[t], U @ x[t]
            eg = d * u23 * (np.abs(G) @ np.abs(x[t]))
            eu = d * u23 * (np.abs(U) @ np.abs(x[t]))
            s = g / (1.0 + np.exp(-g))
            h = s * u
            eh = 1.1 * eg * (np.abs(u) + eu) + np.abs(s) * eu + (2.0 ** -20 + h_rel) * np.abs(h)
            eh = eh + h_abs
            w = float(weights[t, r])
            y[t] += w * (D @ h)
            bound[t] += abs(w) * (np.abs(D) @ (eh + (inter + ids.shape[1] + 2) * u23 *
                                               (np.abs(h) + eh)))
    return y, bound
