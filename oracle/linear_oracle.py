"""CPU oracle of the checkpointed linear layer, in float64, written from the definitions in include/efsparse.h.

Matrices are float64 arrays (exact images of float32 or bfloat16 inputs).  The products also return the sum of the
products' magnitudes, from which the tests derive how far a float32 sum may be off.
"""

import math

import numpy as np

GROUP = 32
LEAST_EXP = -100
INT8, E4M3 = 0, 1
NONE, RELU, GELU, GELU_TANH, SILU = range(5)

# the non-negative e4m3 numbers, by code: 0 to 126
_E4M3 = np.array([(m / 8 * 2.0 ** -6) if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def _fits(amax, e, fmt):
    v = math.ldexp(amax, -e)
    return round(v) <= 127 if fmt == INT8 else v <= 448.0


def _most(e, fmt):
    """The largest code's value under 2^e that stands for a finite number (at most the largest bfloat16)."""
    v = math.ldexp(float.fromhex("0x1.FEp127"), -e)
    return min(127.0, math.floor(v)) if fmt == INT8 else float(_E4M3[_E4M3 <= v].max())


def _group_exp(amax, fmt):
    e = max(LEAST_EXP, math.frexp(amax)[1] - 12) if amax > 0 else LEAST_EXP
    while not _fits(amax, e, fmt):
        e += 1
    return e


def _nearest_e4m3(v):
    """Codes of v (magnitudes up to 448): the nearest number, ties to the even code."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - _E4M3[lo], _E4M3[hi] - a
    c = np.where(d_lo < d_hi, lo, np.where(d_hi < d_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    return (c + 128 * np.signbit(v)).astype(np.uint8)


def ckpt_pack(x, fmt):
    """(codes uint8 [n][32 G], scales uint8 [n][G]) of x [n][c]."""
    x = np.asarray(x, np.float64)
    n, c = x.shape
    G = -(-c // GROUP)
    codes = np.zeros((n, G * GROUP), np.uint8)
    scales = np.zeros((n, G), np.uint8)
    for r in range(n):
        for g in range(G):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            if not np.isfinite(v).all():
                scales[r, g] = 255
                continue
            e = _group_exp(float(np.abs(v).max()), fmt)
            scales[r, g] = e + 127
            s = np.clip(np.ldexp(v, -e), -_most(e, fmt), _most(e, fmt)) if e > 100 else np.ldexp(v, -e)
            codes[r, g * GROUP:g * GROUP + len(v)] = (np.rint(s).astype(np.int64) & 255 if fmt == INT8 else _nearest_e4m3(s))
    return codes, scales


def ckpt_unpack(codes, scales, fmt, c):
    """What a checkpoint stands for, float64 [n][c]."""
    if fmt == INT8:
        v = codes.view(np.int8).astype(np.float64)
    else:
        v = np.append(_E4M3, np.nan)[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    e = np.repeat(scales.astype(np.int64) - 127, GROUP, axis=1)
    return np.where(e == 128, np.nan, np.ldexp(v, e))[:, :c]


def _erfc(z):
    return np.vectorize(math.erfc, otypes=[np.float64])(z)


def _sigmoid(u):
    return np.where(u >= 0, 1 / (1 + np.exp(-np.abs(u))), np.exp(-np.abs(u)) / (1 + np.exp(-np.abs(u))))


def act(z, kind):
    z = np.asarray(z, np.float64)
    if kind == RELU:
        return np.where(np.isnan(z), z, np.maximum(z, 0))
    if kind == GELU:
        return z * _erfc(-z / math.sqrt(2)) / 2
    if kind == GELU_TANH:
        return z * _sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if kind == SILU:
        return z * _sigmoid(z)
    return z


def act_slope(z, kind):
    """d act / dz."""
    z = np.asarray(z, np.float64)
    if kind == RELU:
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
    if kind == GELU:
        return _erfc(-z / math.sqrt(2)) / 2 + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == GELU_TANH:
        k = 2 * math.sqrt(2 / math.pi)
        u = k * (z + 0.044715 * z ** 3)
        return _sigmoid(u) + z * _sigmoid(u) * _sigmoid(-u) * k * (1 + 3 * 0.044715 * z * z)
    if kind == SILU:
        return _sigmoid(z) + z * _sigmoid(z) * _sigmoid(-z)
    return np.ones_like(z)


def forward(x, w, bias=None):
    """(z = x w^T + bias, the magnitudes' sum)."""
    b = 0.0 if bias is None else bias
    return x @ w.T + b, np.abs(x) @ np.abs(w).T + np.abs(b)


def dgrad(dy, w):
    return dy @ w, np.abs(dy) @ np.abs(w)


def wgrad(dy, kept):
    return dy.T @ kept, np.abs(dy).T @ np.abs(kept)
