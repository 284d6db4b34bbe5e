"""Plain CPU definition of a paged cache held in 8 bits (test infrastructure, as ``oracle.paged``).

  * ``numbers``: what each byte of e4m3 stands for, from its sign, exponent and mantissa;
  * ``quantise``: one part of a row (the latent, or the shared key) to bytes and its scale's exponent, the nearest of
    the 127 finite magnitudes by search, ties to the even byte;
  * ``append``: a token's row (``oracle.producers`` in fp64) quantised into its slot;
  * ``values``: the numbers that a cache stands for, which ``oracle.paged.attend`` then attends over;
  * ``read``: cached positions back as latents and shared keys.

Parity status: pinned by tests/test_paged_q8_oracle.py (hand-written numbers, torch's own e4m3, the scale's rule).
"""
from __future__ import annotations

import math

import numpy as np

from . import producers

__all__ = ["numbers", "exponent", "quantise", "append", "values", "read"]

LEAST, MOST, BIAS = -100, 119, 127


def numbers():
    """The 256 numbers of e4m3: 1 sign, 4 exponent (bias 7), 3 mantissa bits; no infinities, NaN at 0x7f and 0xff."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = math.nan if b & 127 == 127 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        out[b] = -v if b & 128 else v
    return out


def exponent(top):
    """The least e in [LEAST, MOST] with top <= 448 2^e (MOST where there is none)."""
    for e in range(LEAST, MOST):
        if top <= math.ldexp(448.0, e):
            return e
    return MOST


def quantise(x):
    """(bytes uint8, e) of one part of a row, x [n] in fp64."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    e = exponent(float(np.abs(x[fine]).max()) if fine.any() else 0.0)
    size = numbers()[:127]
    v = np.abs(np.where(fine, x, 0.0)) * 2.0 ** -e
    up = np.minimum(np.searchsorted(size, v), 126)
    down = np.maximum(up - 1, 0)
    high, low = size[up] - v, v - size[down]
    byte = np.where((high < low) | ((high == low) & (up % 2 == 0)), up, down)
    byte = byte + 128 * np.signbit(x)
    return np.where(fine, byte, 127).astype(np.uint8), e


def append(latent_raw, kpe_raw, position, slot, cache, scales, gamma=None, eps=1e-6, base=10000.0, offset=0):
    """(cache [n_pages, page, d_c + d_rope] bytes, scales [n_pages, page, 2] bytes) with the tokens' rows in their slots."""
    cache, scales = np.array(cache), np.array(scales)
    n_pages, page = cache.shape[:2]
    y, _ = producers.rms_norm(latent_raw, gamma, eps)
    for t, s in enumerate(slot):
        if 0 <= s < n_pages * page:
            k = producers.rope(np.asarray(kpe_raw, np.float64)[None, t:t + 1], np.array([offset + int(position[t])]), base)[0, 0]
            (c8, e_c), (k8, e_k) = quantise(y[t]), quantise(k)
            cache[s // page, s % page] = np.concatenate([c8, k8])
            scales[s // page, s % page] = e_c + BIAS, e_k + BIAS
    return cache, scales


def values(cache, scales, d_c):
    """The numbers that a cache stands for, fp64."""
    s = 2.0 ** (np.asarray(scales, np.float64) - BIAS)
    v = numbers()[np.asarray(cache)]
    v[..., :d_c] *= s[..., :1]
    v[..., d_c:] *= s[..., 1:]
    return v


def read(cache, scales, table, position, request, d_c):
    """Rows at position[t] of request[t]: 0 at negative positions, NaN outside the table or the pool."""
    n_pages, page, width = cache.shape
    out = np.zeros((len(position), width))
    for t, (p, r) in enumerate(zip(position, request)):
        if p < 0:
            continue
        i = int(table[r, p // page]) if 0 <= r < table.shape[0] and p < table.shape[1] * page else -1
        out[t] = values(cache[i, p % page], scales[i, p % page], d_c) if 0 <= i < n_pages else np.nan
    return out[:, :d_c], out[:, d_c:]
