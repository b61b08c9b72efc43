"""The sketch cache's format and the attention over it, in fp64 numpy.
TEST INFRASTRUCTURE ONLY: used by tests/, never by the library.

A row's D values are held in groups of 32 (the last may be short).  A group's
exponent e is the least integer with amax <= L 2^e (L = 7 for fp4, 464 for fp8), held to
[-100, 125 or 119]; a value is held as the representable multiple of 2^e nearest to it,
of two equally near ones that with the even code, at most the largest; a group with an
infinity or a NaN is held as NaN (scale byte 255, codes 0).  Bytes of a slot as
include/sa_sketch.h states them: blocks of 8 rows by 8 values, then the scale bytes by
octet of rows, group and row.

Everything here goes code by code through the list of representable values; no bit of
the library's arithmetic is repeated.
"""
from __future__ import annotations

import numpy as np

from oracle import stca as ostca

GROUP = 32
E_MIN = -100
E_MAX = {"fp4": 125, "fp8": 119}
LIMIT = {"fp4": 7.0, "fp8": 464.0}
BITS = {"fp4": 4, "fp8": 8}


def magnitudes(fmt: str) -> np.ndarray:
    """The representable magnitudes in code order."""
    if fmt == "fp4":   # 1 sign, 2 exponent (bias 1), 1 fraction bit
        e, f, bias, part = np.divmod(np.arange(8), 2) + (1, 2)
    else:              # 1 sign, 4 exponent (bias 7), 3 fraction bits; the last code is NaN
        e, f, bias, part = np.divmod(np.arange(127), 8) + (7, 8)
    return np.where(e == 0, f / part * 2.0 ** (1 - bias), (1 + f / part) * 2.0 ** (e - bias))


def exponent(amax: float, fmt: str) -> int:
    """The least e in range with amax <= L 2^e."""
    e = E_MIN
    while e < E_MAX[fmt] and amax > np.ldexp(LIMIT[fmt], e):
        e += 1
    return e


def quantise(x, fmt: str):
    """x [..., D] -> (codes uint8 [..., D], scale bytes uint8 [..., G])."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    G = -(-D // GROUP)
    mags = magnitudes(fmt)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros(x.shape[:-1] + (G,), np.uint8)
    for at in np.ndindex(*x.shape[:-1]):
        for g in range(G):
            sl = slice(g * GROUP, min(D, (g + 1) * GROUP))
            v = x[at][sl]
            if not np.all(np.isfinite(v)):
                scales[at][g] = 255
                continue
            e = exponent(np.abs(v).max(), fmt)
            y = np.ldexp(v, -e)
            d = np.abs(np.abs(y)[:, None] - mags[None, :])
            best = d.min(1, keepdims=True)
            # of the nearest codes (neighbours, if two) the even one
            near = d == best
            c = np.where(near.sum(1) == 1, near.argmax(1), near.argmax(1) + (near.argmax(1) & 1))
            codes[at][sl] = c + np.where(np.signbit(y), 1 << (BITS[fmt] - 1), 0)
            scales[at][g] = e + 127
    return codes, scales


def dequantise(codes, scales, fmt: str) -> np.ndarray:
    """The fp64 values that codes [..., D] with scale bytes [..., G] stand for."""
    D = codes.shape[-1]
    half = 1 << (BITS[fmt] - 1)
    mags = magnitudes(fmt)
    if fmt == "fp8":
        mags = np.append(mags, np.nan)
    v = mags[codes & (half - 1)] * np.where(codes >= half, -1.0, 1.0)
    s = np.repeat(scales, GROUP, axis=-1)[..., :D].astype(np.int64)
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127))


def slot_bytes(k: int, D: int, fmt: str) -> int:
    octets, G = -(-k // 8), -(-D // GROUP)
    return -(-(octets * G * 8 * (GROUP * BITS[fmt] // 8 + 1)) // 128) * 128


def places(k: int, D: int, fmt: str):
    """(index of each value's code [k, D], counted in codes; of each scale byte [k, G])."""
    G = -(-D // GROUP)
    r, d = np.arange(k)[:, None], np.arange(D)[None, :]
    code = (((r // 8) * G + d // GROUP) * 4 + d % GROUP // 8) * 64 + (r % 8) * 8 + d % 8
    g = np.arange(G)[None, :]
    scale = -(-k // 8) * G * 8 * GROUP * BITS[fmt] // 8 + ((r // 8) * G + g) * 8 + r % 8
    return code, scale


def pack(slot: np.ndarray, x, n: int, fmt: str) -> None:
    """Writes rows 0 .. n - 1 of x [k, D] into the slot's bytes."""
    k, D = x.shape
    codes, scales = quantise(x[:n], fmt)
    at, sat = places(k, D, fmt)
    G = scales.shape[-1]
    # a short last group is written whole, its missing values zero
    full = np.zeros((n, G * GROUP), np.uint8)
    full[:, :D] = codes
    at = places(k, G * GROUP, fmt)[0]
    if fmt == "fp8":
        slot[at[:n]] = full
    else:
        for j in range(0, G * GROUP, 2):
            slot[at[:n, j] // 2] = full[:, j] | (full[:, j + 1] << 4)
    slot[sat[:n]] = scales


def unpack(slot: np.ndarray, n: int, k: int, D: int, fmt: str) -> np.ndarray:
    """The values [k, D] of a slot, zeros from row n on."""
    at, sat = places(k, D, fmt)
    out = np.zeros((k, D))
    if n:
        codes = slot[at[:n]] if fmt == "fp8" else (slot[at[:n] // 2] >> (4 * (at[:n] % 2))) & 15
        out[:n] = dequantise(codes.astype(np.uint8), slot[sat[:n]], fmt)
    return out


def _users(X, n):
    return [b for b in range(len(n)) if n[b] > 0]


def stca_cached_fwd(X, n, q, Wq, Wk, Wv, h, scale=None):
    """stca_fwd over rows 0 .. n[b] - 1 of X [B, k, D]; out 0 and lse -inf where n[b] = 0."""
    B, R, D = q.shape
    out, lse = np.zeros((B, R, D)), np.full((B, R, h), -np.inf)
    for b in _users(X, n):
        out[b:b + 1], lse[b:b + 1] = ostca.stca_fwd(X[b:b + 1, :n[b]], q[b:b + 1], Wq, Wk, Wv, h, scale)
    return out, lse


def stca_cached_bwd(X, n, q, Wq, Wk, Wv, h, dout, scale=None):
    """Gradients of <dout, out> for q and the weights."""
    B, R, D = q.shape
    g = {"dq": np.zeros((B, R, D)), "dWq": np.zeros((D, D)), "dWk": np.zeros((D, D)), "dWv": np.zeros((D, D))}
    for b in _users(X, n):
        one = ostca.stca_bwd(X[b:b + 1, :n[b]], q[b:b + 1], Wq, Wk, Wv, h, dout[b:b + 1], scale)
        g["dq"][b] = one["dq"][0]
        for w in ("dWq", "dWk", "dWv"):
            g[w] += one[w]
    return g
