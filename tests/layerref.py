"""The layer operators and the verification of drafts in 64 bits (numpy), and how far
a 32-bit computation of each result may be from them.

The bounds follow from the operations, with u = 2^-24 the rounding of binary32:

* a gate's smaller part s = t / (1 + t), t = 2^(-|g| log2 e): the power's argument is
  off by 2 u |g| log2 e ln 2 (a constant and a product), the power by 2 u, the sum by u,
  the reciprocal by 2 u, the product by u, so s, and 1 - s with one rounding more, are
  within eg = (2 |g| + 8) u relatively;
* a state is a sum over earlier rows of products of gates.  Whatever way the rows are
  grouped, a gate enters a product once, with its own error and one rounding of the
  product; an input is rounded once as k x, and a partial sum at most four times at a
  row (in its thread, where threads, and tiles, are joined, at the end).  With M_t = f
  M_{t-1} + k |x_t| the sums of magnitudes, the error is at most E_t = f E_{t-1} +
  (eg + 6 u) (f M_{t-1} + k |x_t|);
* the same holds going back, with e_t = dy_t + f_{t+1} e_{t+1};
* products that fall below binary32's range lose at most its smallest normal number;
* a result stored in a 16-bit type is rounded once more.
"""
import numpy as np

U = 2.0 ** -24
LEAST = 2.0 ** -120


def spans(n, starts, batch):
    if starts is not None:
        return [(int(a), int(b)) for a, b in zip(starts[:-1], starts[1:])]
    return [(i * (n // batch), (i + 1) * (n // batch)) for i in range(batch)]


def gates(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g)), 1.0 / (1.0 + np.exp(g)), (2 * np.abs(g) + 8) * U


def scan(x, gate, seqs, h0):
    """dict of y, before (the state that enters each row), state, and the bounds by,
    bbefore, bstate; rows of no sequence are NaN."""
    n, d = x.shape
    f, k, eg = gates(gate)
    y, before = np.full((n, d), np.nan), np.full((n, d), np.nan)
    by, bb = np.zeros((n, d)), np.zeros((n, d))
    state, bs = np.zeros((len(seqs), d)), np.zeros((len(seqs), d))
    with np.errstate(all="ignore"):
        for i, (a, b) in enumerate(seqs):
            h = np.zeros(d) if h0 is None else h0[i].astype(float)
            mag, err = np.abs(h), np.zeros(d)
            for t in range(a, b):
                before[t], bb[t] = h, err
                h = f[t] * h + k[t] * x[t]
                step = f[t] * mag + k[t] * np.abs(x[t])
                err = f[t] * err + (eg[t] + 6 * U) * step + LEAST
                mag = step
                y[t], by[t] = h, err
            state[i], bs[i] = h, err
    return dict(y=y, before=before, state=state, by=by, bbefore=bb, bstate=bs)


def scan_grad(dy, x, gate, seqs, h0, d_state):
    """dict of dx, dgate, dh0 and bounds bdx, bdgate, bdh0."""
    n, d = x.shape
    f, k, eg = gates(gate)
    fw = scan(x, gate, seqs, h0)
    r = {w: np.full((n, d), np.nan) for w in ("dx", "dgate")}
    r.update({w: np.zeros((n, d)) for w in ("bdx", "bdgate")})
    r["dh0"], r["bdh0"] = np.zeros((len(seqs), d)), np.zeros((len(seqs), d))
    with np.errstate(all="ignore"):
        for i, (a, b) in enumerate(seqs):
            e = np.zeros(d) if d_state is None else d_state[i].astype(float)
            mag, err = np.abs(e), np.zeros(d)
            for t in range(b - 1, a - 1, -1):
                e, mag = dy[t] + e, np.abs(dy[t]) + mag
                err = err + 3 * U * mag
                gap = fw["before"][t] - x[t]
                wide = np.abs(fw["before"][t]) + np.abs(x[t])
                r["dx"][t] = k[t] * e
                r["bdx"][t] = k[t] * (err + (eg[t] + 2 * U) * mag) + LEAST
                r["dgate"][t] = e * gap * f[t] * k[t]
                r["bdgate"][t] = f[t] * k[t] * (
                    err * np.abs(gap) + mag * (fw["bbefore"][t] + U * wide)
                    + mag * np.abs(gap) * (2 * eg[t] + 6 * U)) + LEAST
                e = f[t] * e
                err = f[t] * err + (eg[t] + 3 * U) * f[t] * mag + LEAST
                mag = f[t] * mag
            r["dh0"][i], r["bdh0"][i] = e, err
    return r


def clip(grads, outs, scale, most, step, acc):
    """(norm, its bound, outs, their bounds); the norm and factor are 64-bit numbers
    rounded once, sums of squares off by 2^-30 at most."""
    norm = abs(scale) * np.sqrt(sum((g * g).sum() for g in grads))
    by = step * scale * (min(1.0, most / norm) if norm > 0 else 1.0)
    res, bounds = [], []
    for g, o in zip(grads, outs):
        y = by * g + (o if acc else 0.0)
        res.append(y)
        bounds.append((2 * U + 2.0 ** -29) * np.abs(by * g) + U * np.abs(y) + 2.0 ** -126)
    return norm, (U + 2.0 ** -30) * norm, res, bounds


def softmax(z, temp):
    with np.errstate(all="ignore"):
        m = z.max()
        y = (z - (0.0 if m == -np.inf else m)) / temp
        e = np.where(y < -700, 0.0, np.exp(y))
        s = e.sum()
        return e if s == 0 else e / s


def draw(w, u):
    """The lowest index whose running sum exceeds u times the sum; else the last of
    weight > 0; -1 without any."""
    run = np.cumsum(w)
    over = np.nonzero(run > u * run[-1])[0]
    some = np.nonzero(w > 0)[0]
    return int(over[0]) if len(over) else int(some[-1]) if len(some) else -1


def verify(target, draft, tokens, u, temp):
    """target [b, k + 1, v], draft [b, k, v] or None, tokens [b, k]: (out, accepted)."""
    b, rows, v = target.shape
    out, accepted = np.full((b, rows), -1), np.zeros(b, int)
    for i in range(b):
        j = 0
        while True:
            p = softmax(target[i, j], temp)
            if j == rows - 1 or not 0 <= tokens[i, j] < v:
                nxt = draw(p, u[i, -1])
                break
            x = tokens[i, j]
            q = np.eye(1, v, x)[0] if draft is None else softmax(draft[i, j], temp)
            if not u[i, j] * q[x] < p[x]:
                with np.errstate(invalid="ignore"):
                    left = p - q if draft is not None else np.where(q > 0, 0.0, p)
                    left = np.where(left > 0, left, 0.0)
                nxt = draw(left if left.sum() > 0 else p, u[i, -1])
                break
            out[i, j] = x
            j += 1
        out[i, j], accepted[i] = nxt, j
    return out, accepted
