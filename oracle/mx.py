"""Rows in the microscaled format, their products and the products' gradient.  Test infrastructure only.

A row is blocks of 32 elements (the last padded with zeros); block j holds one scale byte c and 32
codes, and a code stands for 2^(c - 127) times its value:

* 4 bits: sign, two exponent bits (bias 1), one fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6;
* 6 bits: sign, two exponent bits (bias 1), three fraction bits: i / 8, then (1 + i / 8) 2^e, e = 0 .. 2.

The scale is 2^(floor(log2 amax) - 2), 2^-127 at least (and for a block of zeros); an element takes
the nearest value, a tie the even code, and never more than the largest.  A block with an infinity
or a NaN has c = 255, which makes its elements NaN, and zero codes.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def magnitudes(bits: int) -> list:
    """The non-negative values in the order of their codes."""
    frac = bits - 3
    out = []
    for code in range(1 << (bits - 1)):
        e, f = code >> frac, code & ((1 << frac) - 1)
        out.append(f / (1 << frac) if e == 0 else (1 + f / (1 << frac)) * 2.0 ** (e - 1))
    return out


def quantize(x, bits: int):
    """(codes int [m, nb, 32], scales int [m, nb]) of fp64 values x [m x d]."""
    x = np.asarray(x, dtype=np.float64)
    m, d = x.shape
    nb = -(-d // BLOCK)
    mags = np.array(magnitudes(bits))
    codes = np.zeros((m, nb, BLOCK), dtype=np.int64)
    scales = np.zeros((m, nb), dtype=np.int64)
    for r in range(m):
        for b in range(nb):
            v = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            amax = np.abs(v).max()
            e = -127 if amax == 0 else max(math.frexp(amax)[1] - 1 - 2, -127)
            scales[r, b] = e + 127
            a = np.abs(v) / 2.0 ** e
            dist = np.abs(a[:, None] - mags[None, :])
            best = dist.min(axis=1, keepdims=True)
            near = dist == best                                  # one value, or two at a tie
            even = near & (np.arange(len(mags)) % 2 == 0)
            pick = np.where(even.any(axis=1), even.argmax(axis=1), near.argmax(axis=1))
            codes[r, b, :len(v)] = pick + np.signbit(v) * (1 << (bits - 1))
    return codes, scales


def pack(codes, bits: int) -> np.ndarray:
    """Bytes [m, nb, 4 bits] of codes, from the lowest bit of a block's first byte on."""
    c = np.asarray(codes)
    bit = (c[..., None] >> np.arange(bits)) & 1
    return np.packbits(bit.reshape(*c.shape[:2], 32 * bits).astype(np.uint8), axis=-1, bitorder="little")


def unpack(packed, bits: int) -> np.ndarray:
    p = np.asarray(packed)
    bit = np.unpackbits(p, axis=-1, bitorder="little").reshape(p.shape[0], p.shape[1], BLOCK, bits)
    return (bit.astype(np.int64) << np.arange(bits)).sum(axis=-1)


def values(codes, scales, dim: int, bits: int) -> np.ndarray:
    """fp64 values [m x dim]."""
    mags = np.array(magnitudes(bits))
    c = np.asarray(codes)
    v = np.where(c >> (bits - 1), -1.0, 1.0) * mags[c & ((1 << (bits - 1)) - 1)]
    s = np.asarray(scales)
    v = v * np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))[..., None]
    return v.reshape(c.shape[0], -1)[:, :dim]


def scores(q: np.ndarray, x: np.ndarray) -> np.ndarray:
    """S = Q X^T of values."""
    return q @ x.T


def scores_grad(g: np.ndarray, x: np.ndarray, transposed: bool = False) -> np.ndarray:
    """dL/dQ = G X, or (transposed, x the queries' values) dL/dX = G^T Q."""
    g = np.asarray(g, dtype=np.float64)
    return (g.T if transposed else g) @ x
