"""The token operators in 64 bits (numpy), and how far a 32-bit computation of
each result may be from them.

The bounds follow from the operations, with u = 2^-24 the rounding of binary32:

* a sum of N products in any order is within (N + 2) u of the sum of the
  magnitudes;
* y = (z - m) / T takes three roundings, exp another, so exp(y) is within
  (4 |y| + 4) u relatively, and S = sum exp(y) within (4 E|y| + 4 + N) u, E the
  mean over the distribution and N the longest chain of additions (the elements
  a thread adds, V / 256 at most, and the joins: V / 256 + 64 covers them);
* log S is then that far off absolutely, and by two roundings of its own;
* a result stored in a 16-bit type is rounded once more, by at most its type's
  unit roundoff, or half of its smallest subnormal.
"""
import numpy as np

U = 2.0 ** -24
UNIT = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}


def rounded(x, dtype):
    """How far storing x in dtype moves it, at most."""
    return UNIT[dtype] * np.abs(x) + TINY[dtype]


def embed_grad(dy, tokens, old, scale, accumulate):
    """(grad, bound) of binary32 sums; old: what grad held."""
    v, d = old.shape
    g, mag = np.zeros((v, d)), np.zeros((v, d))
    count = np.zeros((v, 1))
    used = (tokens >= 0) & (tokens < v)
    np.add.at(g, tokens[used], dy[used])
    np.add.at(mag, tokens[used], np.abs(dy[used]))
    np.add.at(count, tokens[used], 1.0)
    g, mag = scale * g, abs(scale) * mag
    bound = (count + 2) * U * mag
    if accumulate:
        bound = np.where(count > 0, bound + 2 * U * (np.abs(g) + np.abs(old)), 0.0)
        g = np.where(count > 0, g + old, old)
    return g, bound


def softmax(z, temp):
    """m, y, e, S, log S of every row, with m = 0 and log S = -inf in rows that hold
    only -inf."""
    with np.errstate(all="ignore"):
        m = z.max(axis=1, keepdims=True)
        m = np.where(m == -np.inf, 0.0, m)
        y = (z - m) / temp
        e = np.exp(y)
        s = e.sum(axis=1, keepdims=True)
        return m, y, e, s, np.log(s)


def _mean(e, s, x):
    with np.errstate(all="ignore"):
        return np.where(e > 0, e * x, 0.0).sum(axis=1, keepdims=True) / np.where(s > 0, s, 1.0)


def log_sum_bound(y, e, s, ls):
    v = y.shape[1]
    with np.errstate(all="ignore"):
        return U * (4 * _mean(e, s, np.abs(y)) + 8 + v / 256 + 64 + 4 * np.abs(
            np.where(s > 0, ls, 0.0)))


def logprobs(z, tokens, temp, top):
    """dict of logp, entropy, top_id, top_logp and the bounds b_logp, b_entropy,
    b_top; a negative token's row is skipped."""
    n, v = z.shape
    m, y, e, s, ls = softmax(z, temp)
    bl = log_sum_bound(y, e, s, ls)
    bad = np.isnan(z).any(axis=1) | (z == np.inf).any(axis=1)
    empty = (s[:, 0] == 0)
    off = np.zeros(n, bool) if tokens is None else (tokens < 0) | (tokens >= v)
    with np.errstate(all="ignore"):
        lp = np.where(empty[:, None], -np.inf, y - ls)
        blp = bl + 4 * U * np.abs(np.where(np.isfinite(y), y, 0.0))
        h = np.where(empty, 0.0, (ls - _mean(e, s, y))[:, 0])
        ey = _mean(e, s, np.abs(y))
        bh = (bl * (1 + ey) + U * (4 * _mean(e, s, y * y) + (v / 256 + 72) * ey))[:, 0]
        lp[bad] = np.nan
        h = np.where(bad, np.nan, h)
    r = {}
    if tokens is not None:
        at = np.clip(tokens, 0, v - 1)
        r["logp"] = np.where(off, 0.0, lp[np.arange(n), at])
        r["b_logp"] = blp[np.arange(n), at]
    r["entropy"], r["b_entropy"] = np.where(off, 0.0, h), bh
    if top:
        # largest first, ties to the lowest index; NaN below -inf
        order = np.argsort(np.where(np.isnan(z), np.inf, -z), axis=1, kind="stable")
        nan_last = np.argsort(np.take_along_axis(np.isnan(z), order, 1), axis=1, kind="stable")
        ids = np.take_along_axis(order, nan_last, 1)[:, :top]
        r["top_id"] = np.where(off[:, None], -1, ids)
        r["top_logp"] = np.where(off[:, None], -np.inf, np.take_along_axis(lp, ids, 1))
        r["b_top"] = np.take_along_axis(blp, ids, 1)
    return r


def logprobs_grad(z, tokens, temp, g, gh):
    """(dlogits, bound); g, gh: the gradients of logp and entropy, or None."""
    n, v = z.shape
    m, y, e, s, ls = softmax(z, temp)
    bl = log_sum_bound(y, e, s, ls)
    off = (s[:, 0] == 0)
    if tokens is not None:
        off = off | (tokens < 0) | (tokens >= v)
    g = np.zeros(n) if g is None else g
    gh = np.zeros(n) if gh is None else gh
    with np.errstate(all="ignore"):
        lq = np.where(e > 0, y - ls, 0.0)
        q = e / np.where(s > 0, s, 1.0)
        h = (np.where(s > 0, ls, 0.0) - _mean(e, s, y))
        by_h = gh[:, None] * q * (lq + h)
        d = -g[:, None] * q - by_h
        # q is off by its exponent's error, log q and the entropy by theirs
        rel = bl + U * (4 * np.abs(np.where(np.isfinite(y), y, 0.0)) + 8)
        bh = bl * (1 + np.abs(h)) + U * 8 * _mean(e, s, y * y)
        mag = np.abs(g)[:, None] * q + np.abs(gh)[:, None] * q * (np.abs(lq) + np.abs(h))
        bound = mag * (rel + 8 * U) + np.abs(gh)[:, None] * q * (rel + bh)
        if tokens is not None:
            rows = np.arange(n)
            at = np.clip(tokens, 0, v - 1)
            d[rows, at] += g
            bound[rows, at] += 4 * U * np.abs(g)
        d, bound = d / temp, (bound + 4 * U * np.abs(d)) / temp
    d[off], bound[off] = 0.0, 0.0
    return d, bound


def distill(z, ids, teacher, temp, weight):
    """(loss, dlogits, bound of the loss, bound of dlogits)."""
    n, v = z.shape
    m, y, e, s, ls = softmax(z, temp)
    bl = log_sum_bound(y, e, s, ls)
    here = (ids >= 0) & (ids < v)
    t = np.where(here, teacher, -np.inf)
    _, ty, te, ts, tl = softmax(t, temp)
    off = (ts[:, 0] == 0) | (weight == 0)
    with np.errstate(all="ignore"):
        p = te / np.where(ts > 0, ts, 1.0)
        lp = np.where(p > 0, ty - tl, 0.0)
        at = np.clip(ids, 0, v - 1)
        zy = np.take_along_axis(y, at, 1)
        lq = np.where(s > 0, zy - ls, -np.inf)
        loss = np.where(p > 0, p * (lp - lq), 0.0).sum(axis=1)
        bt = U * (4 * np.abs(np.where(te > 0, ty, 0.0)) + 4 * _mean(te, ts, np.abs(ty)) + 80
                  + 4 * np.abs(np.where(ts > 0, tl, 0.0)))
        bp = bt + bl + 4 * U * np.abs(np.where(np.isfinite(zy), zy, 0.0))
        fin = np.where((p > 0) & np.isfinite(lq), np.abs(lp - lq), 0.0)
        b_loss = (p * (bp + fin * (bt + (ids.shape[1] + 4) * U))).sum(axis=1)
        loss, b_loss = weight * loss, np.abs(weight) * b_loss
        q = e / np.where(s > 0, s, 1.0)
        d = q.copy()
        bound = q * (bl + U * (4 * np.abs(np.where(np.isfinite(y), y, 0.0)) + 12))
        for j in range(ids.shape[1]):
            rows = np.nonzero(here[:, j])[0]
            d[rows, ids[rows, j]] -= p[rows, j]
            bound[rows, ids[rows, j]] += p[rows, j] * (bt[rows, j] + (ids.shape[1] + 4) * U)
        w = (weight / temp)[:, None]
        d, bound = d * w, np.abs(w) * (bound + 4 * U * np.abs(d))
    loss = np.where(off, 0.0, loss)
    d[off], bound[off] = 0.0, 0.0
    return loss, d, np.where(off, 0.0, b_loss), bound
