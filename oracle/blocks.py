"""What stands between the layers, in double precision: dropout, layer norm, residual connections, gated feed-forward blocks.

Written from the formulas; shares no code with the HIP library.  The generator is Philox4x32 with ten rounds (Salmon, Moraes,
Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), pinned in the tests by the test vectors that its authors
publish.
"""
from __future__ import annotations

import numpy as np

_LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key):
    """counter: four arrays (or numbers) of 32-bit words, key: two.  Returns four uint64 arrays of 32-bit words."""
    c0, c1, c2, c3 = np.broadcast_arrays(*(np.asarray(c, dtype=np.uint64) for c in counter))
    k0, k1 = (int(k) for k in key)
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = ((b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & _LOW,
                          (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & _LOW)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def dropout_factor(n, f, p, seed, step, site=0):
    """[n, f]: 0 for a dropped element, 1 / (1 - p) for the others; p is taken as a float32."""
    p = float(np.float32(p))
    if p == 0.0:
        return np.ones((n, f))
    seed, groups = seed % (1 << 64), (f + 3) // 4
    words = philox4x32((np.arange(groups)[None, :], np.arange(n)[:, None], site, step % (1 << 32)),
                       (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack(words, axis=-1).reshape(n, 4 * groups)[:, :f]
    return np.where(words < np.uint64(round(p * 2.0 ** 32)), 0.0, 1.0 / (1.0 - p))


def dropout(X, factor):
    """Selects, so that what is dropped is 0 whatever it was."""
    with np.errstate(invalid="ignore"):
        return np.where(factor == 0.0, 0.0, np.asarray(X, dtype=np.float64) * factor)


def _activation(z, act):
    if act == "relu":
        return np.maximum(z, 0.0), np.where(np.isnan(z), z, z > 0)
    if act == "elu":
        return np.where(z > 0, z, np.expm1(np.minimum(z, 0.0))), np.exp(np.minimum(z, 0.0))
    return z, np.ones_like(z)


def normalise(X, eps):
    X = np.asarray(X, dtype=np.float64)
    mean = X.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((X - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return (X - mean) * rstd, mean, rstd


def layer_norm_forward(X, gamma, beta, eps, act="none", factor=1.0):
    """(Y, z): dropout(act(z)) and z = gamma xhat + beta."""
    z = normalise(X, eps)[0] * np.asarray(gamma, dtype=np.float64) + np.asarray(beta, dtype=np.float64)
    return _activation(z, act)[0] * factor, z


def layer_norm_backward(X, gamma, beta, eps, dY, act="none", factor=1.0):
    """(dX, dgamma, dbeta)."""
    xhat, _, rstd = normalise(X, eps)
    gamma = np.asarray(gamma, dtype=np.float64)
    dz = np.asarray(dY, dtype=np.float64) * factor * _activation(xhat * gamma + beta, act)[1]
    g = dz * gamma
    dX = rstd * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dX, (dz * xhat).sum(axis=0), dz.sum(axis=0)


def gate(kind, a):
    """The activation of a gate and its derivative."""
    from scipy.special import expit, ndtr
    if kind == "gelu":
        return a * ndtr(a), ndtr(a) + a * np.exp(-0.5 * a * a) / np.sqrt(2.0 * np.pi)
    s, t = expit(a), expit(-a)
    return (a * s, s + a * s * t) if kind == "silu" else (s, s * t)


def gated_forward(X, W, b, kind):
    """(H, Z): act(A) * U and Z = [A | U]."""
    Z = np.asarray(X, dtype=np.float64) @ np.asarray(W, dtype=np.float64)
    if b is not None:
        Z = Z + np.asarray(b, dtype=np.float64)
    k = Z.shape[1] // 2
    return gate(kind, Z[:, :k])[0] * Z[:, k:], Z


def gated_backward(X, W, Z, dH, kind):
    """(dW, db, dX, D) from Z = [A | U]."""
    k = Z.shape[1] // 2
    a, da = gate(kind, Z[:, :k])
    dH = np.asarray(dH, dtype=np.float64)
    D = np.concatenate([dH * Z[:, k:] * da, dH * a], axis=1)
    X, W = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64)
    return X.T @ D, D.sum(axis=0), D @ W.T, D


def held8(X, columns=None):
    """(q, a / 127): a row of X .* columns in 8 bits.  The integers are defined by operations rounded to float32, with an exponent range
    without end (rows below 2^-100 are taken times 2^64)."""
    x = np.asarray(X, dtype=np.float32)
    if columns is not None:
        x = x * np.asarray(columns, dtype=np.float32)
    top = np.abs(x).max(axis=1, keepdims=True)
    up = np.where(top < np.float32(2.0 ** -100), np.float32(2.0 ** 64), np.float32(1.0))
    a = top * up
    with np.errstate(divide="ignore", invalid="ignore"):
        per_unit = np.where(top > 0, np.float32(127.0) / a, np.float32(0.0))
        q = np.rint(x * up * per_unit)
    q = np.where(np.isfinite(top), q, 0.0)
    scale = np.where(np.isfinite(top), top.astype(np.float64) / 127.0, np.nan)[:, 0]
    return q.astype(np.int8), scale


def rms_norm(H, eps):
    """(xhat, rstd [n, 1])."""
    H = np.asarray(H, dtype=np.float64)
    rstd = 1.0 / np.sqrt((H ** 2).mean(axis=1, keepdims=True) + eps)
    return H * rstd, rstd


def rms_norm_backward(xhat, rstd, gamma, dY):
    """(gradient with respect to H, dgamma)."""
    dY = np.asarray(dY, dtype=np.float64)
    g = dY * np.asarray(gamma, dtype=np.float64)
    return rstd * (g - xhat * (g * xhat).mean(axis=1, keepdims=True)), (dY * xhat).sum(axis=0)


def act(kind, z):
    """An activation of the products and its derivative."""
    return gate(kind, z) if kind in ("sigmoid", "silu", "gelu") else _activation(z, kind)


def linear_forward(X, W, b, kind, R=None):
    """(Y, Z): act(Z) + R and Z = X W + b."""
    Z = np.asarray(X, dtype=np.float64) @ np.asarray(W, dtype=np.float64)
    if b is not None:
        Z = Z + np.asarray(b, dtype=np.float64)
    Y = act(kind, Z)[0]
    return Y if R is None else Y + np.asarray(R, dtype=np.float64), Z


def linear_backward(X, W, Z, dY, kind):
    """(dW, db, dX, D)."""
    D = np.asarray(dY, dtype=np.float64) * act(kind, Z)[1]
    X, W = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64)
    return X.T @ D, D.sum(axis=0), D @ W.T, D
