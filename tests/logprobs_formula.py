"""Log probabilities, entropy, best classes and their gradient in numpy, fp64, with the sums that bound the errors of fp32 ones."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def logits_32(logits, bias):
    """z as fp32 has it: one addition."""
    z = np.asarray(logits, dtype=np.float32)
    with np.errstate(all="ignore"):
        return (z + np.asarray(bias, dtype=np.float32) if bias is not None else z) + np.float32(0)


def answer(z, ids):
    """z: fp32 [rows, C].  logp, entropy, norm, and the magnitudes: largest distance that counts and sums over p |d|, p d^2."""
    z = z.astype(np.float64)
    n, C = z.shape
    with np.errstate(all="ignore"):
        M = np.where(np.isnan(z), -np.inf, z).max(1)  # of the numbers; of none: minus infinity
        d = z - M[:, None]
        e = np.exp(d)
        given = (ids >= 0) & (ids < C)
        y = np.where(given, ids, 0)
        own = np.where(given, e[np.arange(n), y], 0.0)
        rest = e.copy()
        rest[np.arange(n)[given], y[given]] = 0
        others = rest.sum(1)
        total = others + own
        log_s = np.where(own > 0.5 * total, np.log1p(others / own) + d[np.arange(n), y], np.log(total))
        logp = np.where(own > 0.5 * total, -np.log1p(others / own), d[np.arange(n), y] - log_s)
        p = e / total[:, None]
        pd = np.where(p > 0, p * d, np.where(np.isnan(p), np.nan, 0.0))
        H = log_s - pd.sum(1)
        A, B = np.where(p > 0, p * (8 - d), 0.0).sum(1), np.where(p > 0, p * (8 - d) ** 2, 0.0).sum(1)
    return dict(logp=np.where(given, logp, 0.0), entropy=H, M=M, log_s=log_s, p=p, d=d, own_d=d[np.arange(n), y], A=A, B=B, given=given)


def bounds(w, C):
    """A lane adds at most C / 64 + 8 terms (C where a row's lanes are few), whose exponentials are off by (2 |d| + 4) u; then at most two dozen joins of eight roundings.
    The hardware's exponential has no results below 2^-126: each of C terms may be that much short (of a sum that is 1 at least), times its distance of less than 128 in t."""
    chain = (C if C <= 256 else C / 64 + 8) + 200
    rel = chain * U + 2 * U * w["A"]
    logp = rel * np.minimum(1, 1.5 * np.abs(w["logp"])) + 4 * U * (np.abs(w["own_d"]) + np.abs(w["logp"]))
    entropy = rel * (1 + w["A"]) + 4 * U * w["B"] + 4 * U * np.abs(w["log_s"])
    logp, entropy = logp + C * 2.0 ** -126, entropy + C * 2.0 ** -119
    return dict(logp=np.where(w["given"], logp, 0.0), entropy=entropy, log_s=rel + 4 * U * np.abs(w["log_s"]))


def best(z, n_top):
    """Classes in the order of (z, lower class first); a NaN is in none."""
    order = np.argsort(np.where(np.isnan(z), np.inf, -z.astype(np.float64)), axis=1, kind="stable")[:, :n_top]
    picked = np.take_along_axis(z, order, 1)
    return np.where(np.isnan(picked), -1, order)


def gradient(z, ids, M, log_s, logp, H, gl, gh, inplace=None):
    """dz and a bound of its error in fp32, from what the forward pass gave (fp32 numbers, as they are)."""
    z, M, log_s, logp, H, gl, gh = (np.asarray(x, dtype=np.float64) for x in (z, M, log_s, logp, H, gl, gh))
    n, C = z.shape
    with np.errstate(all="ignore"):
        given = (ids >= 0) & (ids < C)
        gl = np.where(given, gl, 0.0)
        log = z - M[:, None] - log_s[:, None]
        p = np.exp(log)
        part = np.where(p > 0, p * (log + H[:, None]), np.where(np.isnan(p), np.nan, 0.0))
        first = -p * gl[:, None]
        at = np.flatnonzero(given)
        first[at, ids[at]] = -np.expm1(logp[at]) * gl[at]
        g = first - gh[:, None] * part
        far = np.where(p > 0, np.abs(z - M[:, None]) + 3 * np.abs(log), 0.0)
        delta = U * far + 4 * U
        bound = np.abs(first) * (delta + 4 * U) + np.abs(gh)[:, None] * p * ((delta + 6 * U) * (np.where(p > 0, np.abs(log), 0) + np.abs(H)[:, None]) + U * far + 2.0 ** -126)
    return g, bound + 4 * U * np.abs(g) + 1e-44
