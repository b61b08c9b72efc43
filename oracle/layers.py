"""Layer norm and linear layers in fp64 numpy, by their formulas, with how far a result in lower
precision may be off (element by element).  TEST INFRASTRUCTURE ONLY: used by tests/, never by the
library.

As in oracle/recent.py: a single-precision operation is off by at most U = 2^-23 of its result, a
sum of n terms by n U of the sum of their magnitudes, a rounding to bf16 by 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np
from math import erf, pi

from oracle.recent import HALF, U

_erf = np.vectorize(erf, otypes=[np.float64])


def norm_fwd(x, gamma, beta, eps, dtype):
    """y, stats [N, 2] and how far each may be off."""
    x, gamma, beta = (np.asarray(v, np.float64) for v in (x, gamma, beta))
    D = x.shape[1]
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    m_off = (D + 2) * U * np.abs(x).mean(1, keepdims=True)
    # x - mean is off by the mean's error and a rounding; the mean of its squares by twice their product
    c_off = m_off + U * (np.abs(x) + np.abs(mean))
    v_off = (2 * np.abs(x - mean) * c_off + c_off ** 2).mean(1, keepdims=True) + (D + 3) * U * var + 2 * U * eps
    # 1 / sqrt is convex: largest where var is smallest
    least = np.maximum(var + eps - v_off, (var + eps) / 4)
    r_off = 0.5 * v_off * least ** -1.5 + 4 * U * rstd
    y = (x - mean) * rstd * gamma + beta
    y_off = np.abs(gamma) * (c_off * (rstd + r_off) + np.abs(x - mean) * r_off + 2 * U * np.abs(x - mean) * rstd)
    y_off += (U + HALF[dtype]) * (np.abs(y) + np.abs(beta) * (U / HALF[dtype]))
    return y, np.concatenate([mean, rstd], 1), y_off, np.concatenate([m_off, r_off], 1)


def norm_bwd(x, gamma, stats, dy, dtype):
    """{dx, dgamma, dbeta} and how far each may be off, for stats as given."""
    x, gamma, stats, dy = (np.asarray(v, np.float64) for v in (x, gamma, stats, dy))
    N, D = x.shape
    mean, rstd = stats[:, :1], stats[:, 1:]
    xh = (x - mean) * rstd
    x_off = 2 * U * (np.abs(xh) + np.abs(x - mean) * rstd)
    g = dy * gamma
    a, b = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    a_off = (D + 3) * U * np.abs(g).mean(1, keepdims=True)
    b_off = (np.abs(g) * x_off).mean(1, keepdims=True) + (D + 4) * U * np.abs(g * xh).mean(1, keepdims=True)
    dx = rstd * (g - a - xh * b)
    dx_off = rstd * (U * np.abs(g) + a_off + np.abs(xh) * b_off + x_off * np.abs(b) + 4 * U * (np.abs(g) + np.abs(a) + np.abs(xh * b)))
    ref = {"dx": dx, "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    off = {"dx": dx_off + HALF[dtype] * np.abs(dx),
           "dgamma": (np.abs(dy) * x_off).sum(0) + (N + 3) * U * np.abs(dy * xh).sum(0),
           "dbeta": (N + 1) * U * np.abs(dy).sum(0)}
    return ref, off


def act(z, name):
    if name == "swiglu":
        a, b = np.split(z, 2, 1)
        return a / (1 + np.exp(-a)) * b
    if name == "silu":
        return z / (1 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + _erf(z / np.sqrt(2)))
    return np.maximum(z, 0) if name == "relu" else z


def act_grad(z, dy, name):
    """dy act'(z), of z's shape."""
    if name in ("silu", "swiglu"):
        a = np.split(z, 2, 1)[0] if name == "swiglu" else z
        s = 1 / (1 + np.exp(-a))
        d = s * (1 + a * (1 - s))
        if name == "silu":
            return dy * d
        return np.concatenate([dy * np.split(z, 2, 1)[1] * d, dy * a * s], 1)
    if name == "gelu":
        return dy * (0.5 * (1 + _erf(z / np.sqrt(2))) + z * np.exp(-z * z / 2) / np.sqrt(2 * pi))
    return np.where(z > 0, dy, 0.0) if name == "relu" else dy


def linear_fwd(x, W, bias, name, residual, dtype):
    """y, z and how far each may be off.

    |silu'| and |gelu'| are at most 1.13; the activations' own arithmetic is off by no more than 8 U
    of |z| (times the gate)."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    z = x @ W
    z_off = (x.shape[1] + 2) * U * (np.abs(x) @ np.abs(W))
    if bias is not None:
        z = z + bias
        z_off = z_off + U * np.abs(z)
    y = act(z, name)
    if name == "swiglu":
        (a, b), (ea, eb) = np.split(z, 2, 1), np.split(z_off, 2, 1)
        y_off = (1.13 * ea + 9 * U * np.abs(a)) * (np.abs(b) + eb) + np.abs(act(a, "silu")) * eb
    else:
        y_off = z_off if name in ("none", "relu") else 1.13 * z_off + 9 * U * np.abs(z)
    if residual is not None:
        y = y + residual
        y_off = y_off + U * np.abs(y)
    return y, z, y_off + HALF[dtype] * np.abs(y), z_off + HALF[dtype] * np.abs(z)


def linear_bwd(x, W, pre, dy, name, dtype):
    """{dx, dW, db} (unrounded) and how far each may be off but for its last rounding.

    An activation's derivative is at most 1.13 and off by no more than 16 U; a gate multiplies both."""
    x, W, dy = (np.asarray(v, np.float64) for v in (x, W, dy))
    dz = act_grad(pre, dy, name)
    e = np.zeros_like(dz)
    if name == "swiglu":
        a, b = np.split(np.asarray(pre, np.float64), 2, 1)
        e = 16 * U * np.concatenate([np.abs(dy * b) * (1 + np.abs(a)), np.abs(dy) * np.abs(a)], 1)
    elif name in ("silu", "gelu"):
        e = 16 * U * np.abs(dy) * (1 + np.abs(pre))
    low = HALF["bf16"] * np.abs(dz) if dtype == "bf16" and name not in ("none", "relu") else 0.0
    N, C = dz.shape
    ref = {"dx": dz @ W.T, "dW": x.T @ dz, "db": dz.sum(0)}
    off = {"dx": (e + low + (C + 2) * U * np.abs(dz)) @ np.abs(W).T,
           "dW": np.abs(x).T @ (e + low + (N + 2) * U * np.abs(dz)),
           "db": (e + (N + 2) * U * np.abs(dz)).sum(0)}
    return ref, off
