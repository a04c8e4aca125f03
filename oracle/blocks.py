"""A residual block's layers in float64: gated dense layers, dropout and the norms around a block.

Formulas (rows r, columns c):

  gated     [g | u] = x W + b, y = act(g) u
            dz = [dy u act'(g) | dy act(g)], dx = dz W^T, dW = x^T dz, db = sum_r dz
  mask      Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
            1, 2, 3", 2011): a round maps (x0, x1, x2, x3) to (hi(M1 x2) ^ x1 ^ k0, lo(M1 x2), hi(M0 x0) ^
            x3 ^ k1, lo(M0 x0)) and adds the Weyl constants to the key
  residual  s = r + scale gate drop(N1(h)), y = N2(s), with n = x rstd (rms) or (x - mean) rstd (layer) and
            N = n gamma (+ beta)
            d = ds + N2'(dy), t = scale drop(d), dgate = t N1(h), dh = N1'(t gate), where N' takes dy to
            rstd (a - n mean_c(a n) [- mean_c(a)]), a = dy gamma
"""
from __future__ import annotations

import numpy as np

from .layers import act

M0, M1 = 0xD2511F53, 0xCD9E8D57
W0, W1 = 0x9E3779B9, 0xBB67AE85
MASK = (1 << 32) - 1


def gated_fwd(x, W, b=None, name="silu"):
    """(y, z)."""
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64)
    if b is not None:
        z = z + b
    n = z.shape[1] // 2
    return act(name, z[:, :n])[0] * z[:, n:], z


def gated_dz(dy, z, name="silu"):
    dy, z = np.asarray(dy, np.float64), np.asarray(z, np.float64)
    n = dy.shape[1]
    a, slope = act(name, z[:, :n])
    return np.concatenate([dy * z[:, n:] * slope, dy * a], 1)


def gated_bwd(x, W, dy, z, name="silu"):
    """(dx, dW, db)."""
    dz = gated_dz(dy, z, name)
    return dz @ np.asarray(W, np.float64).T, np.asarray(x, np.float64).T @ dz, dz.sum(0)


def philox(counter, key):
    """The four words (arrays) of a counter of four words and a key of two."""
    x = [np.asarray(c, np.uint64) for c in counter]
    k0, k1 = key
    for _ in range(10):
        p, q = x[0] * np.uint64(M0), x[2] * np.uint64(M1)
        low, up = np.uint64(MASK), np.uint64(32)
        x = [(q >> up) ^ x[1] ^ np.uint64(k0), q & low, (p >> up) ^ x[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + W0) & MASK, (k1 + W1) & MASK
    return x


def threshold(p):
    return int(np.rint(65536.0 * p))


def kept(rows, cols, p, seed, offset=0):
    """Where the mask keeps a value; rows: a number of rows, or their numbers."""
    row = (np.arange(rows) if np.isscalar(rows) else np.asarray(rows)).astype(np.uint64)[:, None]
    col = np.arange(cols, dtype=np.uint64)[None, :]
    offset &= (1 << 64) - 1
    shape = np.broadcast(row, col).shape
    words = philox([np.broadcast_to(row & np.uint64(MASK), shape),
                    ((row >> np.uint64(32)) << np.uint64(17)) + (col >> np.uint64(3)),
                    np.full(shape, offset & MASK, np.uint64), np.full(shape, offset >> 32, np.uint64)],
                   (seed & MASK, seed >> 32))
    place = (col & np.uint64(7)).astype(int)
    word = np.choose(np.broadcast_to(place // 2, shape), words)
    bits = (word >> (16 * (place % 2)).astype(np.uint64)) & np.uint64(0xFFFF)
    return bits >= threshold(p)


def factors(rows, cols, p, seed, offset=0):
    """What each value is multiplied by: 0 or 65536 / (65536 - t)."""
    t = threshold(p)
    return kept(rows, cols, p, seed, offset) * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def dropped(v, f):
    """v through the mask with factors f: what is dropped is not looked at."""
    with np.errstate(invalid="ignore"):
        return np.where(f > 0, v * f, 0.0)


def norm_stats(x, norm, eps=1e-5):
    """(mean or None, rstd)."""
    x = np.asarray(x, np.float64)
    if norm == "rms":
        return None, 1 / np.sqrt((x * x).mean(1) + eps)
    mean = x.mean(1)
    return mean, 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)


def normed(x, stats):
    mean, rstd = stats
    x = np.asarray(x, np.float64)
    return (x if mean is None else x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]


def affine(n, weights):
    g, b = weights
    n = n if g is None else n * g
    return n if b is None else n + b


def residual_norm_fwd(h, r=None, gate=None, scale=1.0, norm="rms", post=None, pre=None, eps=1e-5, f=None):
    """(s, y or None, stats of N1, stats of N2); f: the mask's factors."""
    v, first, last, y = np.asarray(h, np.float64), None, None, None
    if post is not None:
        first = norm_stats(v, norm, eps)
        v = affine(normed(v, first), post)
    if f is not None:
        v = dropped(v, f)
    s = scale * (v if gate is None else v * gate)
    if r is not None:
        s = s + r
    if pre is not None:
        last = norm_stats(s, norm, eps)
        y = affine(normed(s, last), pre)
    return s, y, first, last


def _through(n, rstd, gamma, dy, norm):
    a = dy if gamma is None else dy * gamma
    inner = n * (a * n).mean(1, keepdims=True)
    return np.asarray(rstd, np.float64)[:, None] * (a - inner - (a.mean(1, keepdims=True) if norm == "layer" else 0.0))


def residual_norm_bwd(h, s, first, last, dy=None, ds=None, gate=None, scale=1.0, norm="rms", post=None, pre=None, f=None):
    """(dr, dh, dgate or None, (dgamma, dbeta) of N1 or None, of N2 or None) with the given statistics."""
    d = np.zeros_like(np.asarray(dy if ds is None else ds, np.float64))
    if ds is not None:
        d = d + ds
    dpost = dpre = dgate = None
    if pre is not None:
        dy = np.asarray(dy, np.float64)
        n = normed(s, last)
        d = d + _through(n, last[1], pre[0], dy, norm)
        dpre = ((dy * n).sum(0), dy.sum(0))
    t = scale * (d if f is None else dropped(d, f))
    h = np.asarray(h, np.float64)
    n1 = None if post is None else normed(h, first)
    if gate is not None:
        o = h if post is None else affine(n1, post)
        dgate = t * o if f is None else np.where(f > 0, t * np.where(f > 0, o, 0.0), 0.0)
        if np.ndim(gate) == 1:
            dgate = dgate.sum(0)
        t = t * gate
    dh = t
    if post is not None:
        dpost = ((t * n1).sum(0), t.sum(0))
        dh = _through(n1, first[1], post[0], t, norm)
    return d, dh, dgate, dpost, dpre
