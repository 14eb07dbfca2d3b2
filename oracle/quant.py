"""float64 oracle of 8-bit serving: rows in 8-bit codes, alone or behind the residual's
addition and a norm, and the linear layer over 8-bit codes, as their definitions.

Arrays are float64 values (decode the element type first) and integer codes.
"""
from fractions import Fraction

import numpy as np
from scipy.special import erfc


def codes(u, exact=False):
    """(q, scale) of the rows of u: q = rint(127 u / max|u|), ties to even, scale = max|u| / 127.
    A row of zeros has scale 0, one with a value that is not finite scale NaN, both codes 0.
    exact: u is what it is, as elements, their sums and products are: next to halfway between two
    codes rational arithmetic decides.  Else u is off by some 2^-52, as what a norm's float64
    arithmetic gave, and a quotient that is halfway by some 2^-45: quotients go to the nearest
    multiple of 2^-40 first, which puts them back there."""
    u = np.asarray(u, np.float64)
    m = np.abs(u).max(1)
    ok = np.isfinite(u).all(1)
    live = ok & (m > 0)
    q = np.zeros(u.shape, np.int64)
    t = 127 * u[live] / m[live, None]
    q[live] = np.rint(np.rint(t * 2.0 ** 40) * 2.0 ** -40).astype(np.int64)
    if exact:
        rows = np.flatnonzero(live)
        for i, j in np.argwhere(np.abs(t - np.floor(t) - 0.5) <= 2.0 ** -39):
            q[rows[i], j] = round(127 * Fraction(u[rows[i], j]) / Fraction(m[rows[i]]))
    return q, np.where(ok, m / 127, np.nan)


def rms(s, gamma, eps):
    """(q, scale) of s / sqrt(mean(s^2) + eps) * gamma: the codes are those of s * gamma."""
    s = np.asarray(s, np.float64)
    q, scale = codes(s * gamma, exact=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1 / np.sqrt((s * s).mean(1) + eps)
        return q, np.where(scale == 0, 0.0, scale * r)


def layer(s, gamma, beta, eps):
    """(q, scale) of (s - mean) / sqrt(var + eps) * gamma + beta."""
    s = np.asarray(s, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        d = s - s.mean(1, keepdims=True)
        return codes(d / np.sqrt((d * d).mean(1, keepdims=True) + eps) * gamma + beta)


def keep(W, mask, b_r, b_c):
    """The codes W with the blocks that the mask drops at 0."""
    return np.where(np.kron(mask != 0, np.ones((b_r, b_c), bool)), W, 0)


def linear(X, xscale, W, wscale, bias=None, gelu=False):
    """(Y, A): Y = g(xscale wscale (X W^T) + bias) in float64 from codes, and A the sizes
    |xscale wscale (X W^T)| that a rounding before the bias is relative to."""
    # (products and sums of codes are whole numbers below 2^53: exact in float64)
    p = np.asarray(X, np.float64) @ np.asarray(W, np.float64).T
    p = p * np.asarray(xscale, np.float64)[:, None] * np.asarray(wscale, np.float64)
    y = p if bias is None else p + np.asarray(bias, np.float64)
    return (0.5 * y * erfc(-y / np.sqrt(2)) if gelu else y), np.abs(p)
