"""Plain float64 forms of the operators of include/gt_layer.h, with the sums of
absolute values that scale their rounding errors, and the tolerances of their
tests.

Rounding: a value rounded to a type is off by at most half a step, relative
2^-24 in fp32 and 2^-8 in bf16 (torch.finfo(t).eps / 2).  A sum of n terms in
fp32 is off by at most n 2^-24 times the sum of their absolute values.
"""
from __future__ import annotations

import numpy as np

from tests.helpers import bf16_bits_to_f32, score_rounding_bound

U32 = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def widen(x):
    return (bf16_bits_to_f32(x) if x.dtype == np.uint16 else x).astype(np.float64)


def rows_of(rowptr):
    return np.repeat(np.arange(rowptr.size - 1), np.diff(rowptr))


def add_rows(n, at, values):
    out = np.zeros((n,) + values.shape[1:])
    np.add.at(out, at, values)
    return out


class Diff:
    """Differential attention and its gradients; scales S* are the same sums over
    absolute values of every factor."""

    def __init__(self, rowptr, colidx, Q, K, V, lam, scale, dO=None, lse=None):
        q, k, v, lam = widen(Q), widen(K), widen(V), lam.astype(np.float64)
        n, maps, _ = q.shape
        h = maps // 2
        i, j = rows_of(rowptr), colidx.astype(np.int64)
        scale = float(scale)
        with np.errstate(all="ignore"):
            s = np.sum(q[i] * k[j], -1) * scale
            top = np.full((n, maps), -np.inf)
            np.maximum.at(top, i, s)
            ref = np.where(np.isneginf(top), 0.0, top)  # (a map of -inf scores alone is empty)
            total = add_rows(n, i, np.exp(s - ref[i]))
            self.lse = ref + np.log(total)
            L = self.lse if lse is None else lse.astype(np.float64)
            a = np.where(np.isneginf(L[i]), 0.0, np.exp(s - np.where(np.isneginf(L), 0.0, L)[i]))
        a0, a1 = a[:, 0::2], a[:, 1::2]
        mix, amix = a0 - lam * a1, a0 + np.abs(lam) * a1
        self.out = add_rows(n, i, mix[..., None] * v[j])
        self.Sout = add_rows(n, i, amix[..., None] * np.abs(v[j]))
        if dO is None:
            return
        do = widen(dO)
        c = np.repeat(np.sum(do[i] * v[j], -1), 2, 1)
        ca = np.repeat(np.sum(np.abs(do[i] * v[j]), -1), 2, 1)
        delta, delta_a = add_rows(n, i, a * c), add_rows(n, i, a * ca)
        g = np.stack([np.ones(h), -lam], 1).reshape(-1)
        ds, dsa = g * a * (c - delta[i]) * scale, np.abs(g) * a * (ca + delta_a[i]) * abs(scale)
        self.dQ, self.SdQ = add_rows(n, i, ds[..., None] * k[j]), add_rows(n, i, dsa[..., None] * np.abs(k[j]))
        self.dK, self.SdK = add_rows(n, j, ds[..., None] * q[i]), add_rows(n, j, dsa[..., None] * np.abs(q[i]))
        self.dV = add_rows(n, j, mix[..., None] * do[i])
        self.SdV = add_rows(n, j, amix[..., None] * np.abs(do[i]))
        self.dlam, self.Sdlam = -delta[:, 1::2].sum(0), delta_a[:, 1::2].sum(0)


class DiffBounds:
    """How far results may be off, in units of the scales above.  A score is off
    by at most e (tests.helpers.score_rounding_bound, per row and map); so a
    weight is off by a factor of 1 + 2e (its own score and the normaliser), or
    with a given lse by e and the rounding of lse and of its product with
    log2(e), |lse| 2^-22.  A sum over a row's d entries adds (d + 16) 2^-24 (16
    for the exponential, rescalings, merges and the quotient), a dot product of
    2D elements 2D 2^-24, twice for c and Delta."""

    def __init__(self, rowptr, colidx, Q, K, scale, dtype, lse):
        n, maps, D = Q.shape
        deg = np.diff(rowptr).astype(np.float64)
        degt = np.bincount(colidx, minlength=n).astype(np.float64)
        e = score_rounding_bound(rowptr, colidx, Q, K, abs(float(scale)))
        fin = np.where(np.isfinite(lse), np.abs(lse), 0.0)
        r, pair = ROUND[dtype], lambda x: np.maximum(x[:, 0::2], x[:, 1::2])
        self.lse = 2 * e + (deg[:, None] + 16) * U32 + 4 * U32 * fin
        self.out = (2 * pair(e) + (deg[:, None] + 16) * U32 + r)[..., None]
        w = e + 4 * U32 * fin  # of a weight, by the given lse
        base = (4 * D + 32) * U32 + r
        self.dQ = (2 * w + deg[:, None] * 3 * U32 + base)[..., None]
        wt = np.zeros_like(w)
        i = rows_of(rowptr)
        np.maximum.at(wt, colidx, 2 * w[i] + deg[i][:, None] * 3 * U32)
        self.dK = (wt + degt[:, None] * U32 + base)[..., None]
        self.dV = (pair(wt) + degt[:, None] * U32 + base)[..., None]
        self.dlam = np.max(2 * w + deg[:, None] * 3 * U32, 0)[1::2] + base


def worst(x, ref, scale, bound):
    """The largest error in units of its tolerance."""
    x = x.astype(np.float64)
    assert np.all(np.isfinite(x))
    tol = np.maximum(np.abs(ref), scale) * bound + 1e-35
    return float(np.max(np.abs(x - ref) / tol)) if x.size else 0.0


def rope(pos, X, dims, theta, layout, inverse):
    """Rotary positions of X [N, H, D], and |x| + |y| of each element's pair."""
    x = widen(X)
    out, size = x.copy(), np.abs(x)
    off, total = 0, sum(dims)
    for axis, width in enumerate(dims):
        for k in range(width // 2):
            if layout == "pairs":
                a, b, e = off + 2 * k, off + 2 * k + 1, 2 * k / width
            elif layout == "halves":
                a, b, e = off + k, off + width // 2 + k, 2 * k / width
            else:
                a, b = off // 2 + k, total // 2 + off // 2 + k
                e = 2 * a / total
            with np.errstate(invalid="ignore"):
                t = (pos[:, axis].astype(np.float64) * theta ** -e)[:, None]
                c, s = np.cos(t), np.sin(t) * (-1 if inverse else 1)
            out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
            size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        off += width
    return out, size


class Norm:
    """Layer norm and its gradients, with scales of their rounding errors: an
    element's distance from the mean is off by at most k 2^-24 times |x| plus
    the mean of the row's |x|, every later factor and sum by k 2^-24 of its own
    absolute value, with k = `sums` = F / 32 + 32 (a lane's additions, the tree over the
    lanes, and the roundings of the factors)."""

    def __init__(self, X, gamma, beta, eps, dO=None, mean=None, rstd=None):
        x = widen(X)
        n, f = x.shape
        self.mean, var = x.mean(1), x.var(1)
        with np.errstate(divide="ignore"):
            self.rstd = 1 / np.sqrt(var + float(np.float32(eps)))
        m, r = (self.mean, self.rstd) if mean is None else (mean.astype(np.float64), rstd.astype(np.float64))
        self.sums = (f / 32 + 32) * U32
        gm = np.ones(f) if gamma is None else gamma.astype(np.float64)
        bt = np.zeros(f) if beta is None else beta.astype(np.float64)
        xa = np.abs(x) + np.abs(x).mean(1, keepdims=True)
        xhat, xhat_a = (x - m[:, None]) * r[:, None], xa * r[:, None]
        self.Smean, self.Srstd = np.abs(x).mean(1), self.rstd * (1 + self.rstd ** 2 * (xa * np.abs(x - self.mean[:, None])).mean(1))
        self.out = xhat * gm + bt
        # (a relative error of rstd is at most that of the variance)
        self.Sout = np.abs(gm) * (xhat_a + np.abs(xhat) * (self.Srstd / self.rstd)[:, None]) + np.abs(bt)
        if dO is None:
            return
        do = widen(dO)
        g = do * gm
        self.dX = r[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
        ga = np.abs(g)
        self.SdX = r[:, None] * (ga + ga.mean(1, keepdims=True) + (np.abs(xhat) + xhat_a) * (ga * (np.abs(xhat) + xhat_a)).mean(1, keepdims=True))
        self.dgamma, self.Sdgamma = (do * xhat).sum(0), (np.abs(do) * (xhat_a + np.abs(xhat))).sum(0)
        self.dbeta, self.Sdbeta = do.sum(0), np.abs(do).sum(0)
