"""Attention over long sequences with inputs that mark where a term of a sum
came from, so that a tile left out or counted twice shows far outside a
rounding, however many keys there are (test infrastructure).

Every score is 0: a query of c visible keys gives each of them 1 / c. Keys and
rows belong to classes, tile after tile; a value (key, query, gradient) is one
at its class's place, so a result holds, class by class, a count over c, which
float64 forms from running sums. `lost`: a range of keys (rows) that the
results leave out - the mistake that the bounds have to show.
"""

import numpy as np

from oracle.attention import U, U32

TILE = 32           # of keys and of rows, the smallest that the kernels walk


def classes(n, count):
    return np.arange(n) // TILE % count


def seen(n, m, causal, window):
    """Keys lo .. hi - 1 that each of n queries sees."""
    p = np.arange(n) + (m - n)
    if not causal:
        return np.zeros(n, dtype=int), np.full(n, m)
    hi = np.clip(p + 1, 0, m)
    return np.minimum(np.clip(p + 1 - window, 0, m) if window else 0 * p, hi), hi


def seers(n, m, causal, window):
    """Rows lo .. hi - 1 that see each of m keys."""
    t = np.arange(m) - (m - n)
    if not causal:
        return np.zeros(m, dtype=int), np.full(m, n)
    lo = np.clip(t, 0, n)
    return lo, np.maximum(np.clip(t + window, 0, n) if window else 0 * t + n, lo)


def _running(weight, kind, count):
    """[len + 1, count]: sums of the weights before each place, class by class."""
    out = np.zeros((len(weight) + 1, count))
    out[np.arange(1, len(weight) + 1), kind] = weight
    return np.cumsum(out, 0, out=out)


def _kept(n, lost):
    w = np.ones(n)
    if lost:
        w[lost[0]:lost[1]] = 0.0
    return w


def marks(n, count):
    """[n, count]: one at the class's place."""
    x = np.zeros((n, count))
    x[np.arange(n), classes(n, count)] = 1.0
    return x


def forward(n, m, dim, causal, window, kind, lost=None):
    """For values marks(m, dim): out [n, dim], lse [n], and their bounds.
    Probabilities before their division are one, so counts and sums are exact;
    what is left is the quotient, the weights of cuts of the keys (exp2 of log-
    sums of up to log2(m), off by a step of these each, so 64 steps in all),
    and the rounding of out."""
    lo, hi = seen(n, m, causal, window)
    at = _running(_kept(m, lost), classes(m, dim), dim)
    got = at[hi] - at[lo]
    total = got.sum(1)
    out = got / np.maximum(total, 1.0)[:, None]
    with np.errstate(divide="ignore"):
        lse = np.log(total)
    low = 2.0 ** -25 if kind == "fp16" else 0.0
    return (out, lse, (U[kind] + 64 * U32) * out + low,
            np.where(total > 0, 4 * U32 * (np.abs(lse) + 1.0), 0.0))


def signs(m, dim):
    """dp of each key: 1, or -1 for every fourth class."""
    return np.where(classes(m, dim) % 4 == 3, -1.0, 1.0)


class Gradients:
    """Problem A (keys marked): q = 0, k = marks, so dq holds the keys' sums;
    problem B (rows marked): k = 0, q = marks, so dk holds the rows' sums. In
    both v = sign e_0 and dout = e_0 + (the row's mark, at places 1 on), so
    dp = sign and dv holds the rows' sums of probabilities."""

    def __init__(self, n, m, dim, causal, window, scale, kind):
        self.n, self.m, self.dim, self.scale, self.kind = n, m, dim, scale, kind
        self.causal, self.window = causal, window
        self.v = np.zeros((m, dim))
        self.v[:, 0] = signs(m, dim)
        self.dout = np.zeros((n, dim))
        self.dout[:, 1:] = marks(n, dim - 1)
        self.dout[:, 0] = 1.0
        self.lo, self.hi = seen(n, m, causal, window)
        self.count = (self.hi - self.lo).astype(float)
        self.p = 1.0 / np.maximum(self.count, 1.0) * (self.count > 0)
        run = np.concatenate([[0.0], np.cumsum(signs(m, dim))])
        self.delta = (run[self.hi] - run[self.lo]) * self.p      # out, at place 0
        with np.errstate(divide="ignore"):
            self.lse = np.log(self.count)
        self.out = np.zeros((n, dim))
        self.out[:, 0] = self.delta
        # of a probability formed from lse in float32, relative
        self.t = 8 * U32 * (np.log(np.maximum(self.count, 1.0)) + 1.0)

    def _delta_error(self):
        """D from the rounded out, or from a float32 sum of c terms of which
        the signs cancel some."""
        return U[self.kind] * np.abs(self.delta) + (16 + np.sqrt(self.count)) * U32 + self.t

    def dq(self, lost=None):
        """Of problem A, and its bound."""
        u = U[self.kind]
        at = _running(_kept(self.m, lost), classes(self.m, self.dim), self.dim)
        n_c = at[self.hi] - at[self.lo]
        sign = np.where(np.arange(self.dim) % 4 == 3, -1.0, 1.0)
        ds = (sign - self.delta[:, None]) * self.p[:, None]
        want = self.scale * n_c * ds
        e = (self._delta_error() * self.p)[:, None] + (u + self.t + 64 * U32)[:, None] * np.abs(ds)
        bound = self.scale * n_c * e * (1 + u)
        return want, self._rounded(want, bound)

    def _rounded(self, want, bound):
        u = U[self.kind]
        low = 2.0 ** -25 if self.kind == "fp16" else 0.0
        return bound * (1 + u) + u * np.abs(want) + low

    def _over_rows(self, weight, kind, count):
        at = _running(weight, kind, count)
        lo, hi = seers(self.n, self.m, self.causal, self.window)
        return at[hi] - at[lo]

    def dv(self, lost=None):
        """Of both problems, and its bound."""
        u, kept = U[self.kind], _kept(self.n, lost)
        kind = 1 + classes(self.n, self.dim - 1)
        want = self._over_rows(self.p * kept, kind, self.dim)
        bound = self._over_rows(self.p * kept * (u + self.t + 64 * U32), kind, self.dim)
        for x in (want, bound):
            x[:, 0] = x[:, 1:].sum(1)
        return want, self._rounded(want, bound)

    def dk(self, lost=None):
        """Of problem B, and its bound."""
        u, kept, kind = U[self.kind], _kept(self.n, lost), classes(self.n, self.dim)
        sign = signs(self.m, self.dim)[:, None]
        s_p = self._over_rows(self.p * kept, kind, self.dim)
        s_d = self._over_rows(self.p * self.delta * kept, kind, self.dim)
        want = self.scale * (sign * s_p - s_d)
        # |ds| = p |sign - D| <= p (1 + |D|)
        e = self.p * kept * (self._delta_error()
                             + (u + self.t + 64 * U32) * (1 + np.abs(self.delta)))
        bound = self.scale * self._over_rows(e, kind, self.dim) * (1 + u)
        return want, self._rounded(want, bound)
