"""Invariant layers in float64: dense layers, layer norm and 8-bit checkpoints.

Formulas (rows r, columns c):

  dense       z = x W + b, y = act(z) + res
              dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum_r dz
  layer norm  n = (x - mean_c x) / sqrt(mean_c (x - mean)^2 + eps), y = n gamma + beta
              a = dy gamma, dx = (a - mean_c a - n mean_c(a n)) rstd,
              dgamma = sum_r dy n, dbeta = sum_r dy
  checkpoint  groups of 32 columns, step 2^(c - 127): c - 127 = floor(log2 max|x|) - 6, one more
              where max|x| is at least 127.5 of those steps, at least -127, at most 121; integers to
              nearest, ties to even, at most 127 (which cuts only above 127.5 2^121, where the next
              step's 64 is out of float32); c = 255 for a group that holds an infinity or a NaN
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
ACTIVATIONS = ("none", "relu", "silu", "gelu")

_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(name, z):
    """(act(z), act'(z)); relu' is 0 at 0."""
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if name == "silu":
        # 1 / (1 + exp(-z)) without overflow
        s = 0.5 * (1.0 + np.tanh(0.5 * z))
        return z * s, s + z * s * (1.0 - s)
    if name == "gelu":
        p = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
        return z * p, p + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return z, np.ones_like(z)


def dense_fwd(x, W, b=None, res=None, name="none"):
    """(y, z)."""
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64)
    if b is not None:
        z = z + b
    y = act(name, z)[0]
    return (y if res is None else y + res), z


def dense_bwd(x, W, dy, z=None, name="none"):
    """(dx, dW, db)."""
    dz = np.asarray(dy, np.float64)
    if name != "none":
        dz = dz * act(name, z)[1]
    return dz @ np.asarray(W, np.float64).T, np.asarray(x, np.float64).T @ dz, dz.sum(0)


def layer_norm_fwd(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd)."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def layer_norm_bwd(x, gamma, dy, mean, rstd):
    """(dx, dgamma, dbeta) with the given statistics."""
    n = (np.asarray(x, np.float64) - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    dy = np.asarray(dy, np.float64)
    a = dy if gamma is None else dy * gamma
    dx = (a - a.mean(1, keepdims=True) - n * (a * n).mean(1, keepdims=True)) * np.asarray(rstd, np.float64)[:, None]
    return dx, (dy * n).sum(0), dy.sum(0)


def pack8(x):
    """(q int8 [rows, cols], c uint8 [rows, ceil(cols / 32)])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    groups = (cols + GROUP - 1) // GROUP
    v = np.zeros((rows, groups * GROUP))
    v[:, :cols] = x
    v = v.reshape(rows, groups, GROUP)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    e = np.frexp(top)[1] - 7                     # top < 2^(e + 7)
    e = np.where(top >= np.ldexp(127.5, e), e + 1, e)
    e = np.where(top == 0, -127, np.clip(e, -127, 121))
    q = np.clip(np.rint(np.ldexp(v, -e[..., None])), -127, 127)
    c = np.where(bad, 255, e + 127)
    return q.reshape(rows, groups * GROUP)[:, :cols].astype(np.int8), c.astype(np.uint8)


def unpack8(q, c):
    """The values, in float64."""
    step = np.where(c == 255, np.nan, np.ldexp(1.0, c.astype(int) - 127))
    return q.astype(np.float64) * np.repeat(step, GROUP, 1)[:, : q.shape[1]]
