"""Float64 oracle of attention over packed sequences, its gradients and the
8-bit rows of a cache (test infrastructure), one sequence and head at a time,
with bounds of what float32 sums and 16-bit operands may change."""

import numpy as np

U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half a step of a rounding, relative
U32 = 2.0 ** -23      # a whole step of float32: matrix cores cut sums, they do not round them


def visible(n, m, causal, window):
    """n x m: which keys a query sees."""
    pos = np.arange(n)[:, None] + (m - n)
    j = np.arange(m)[None, :]
    vis = np.ones((n, m), dtype=bool)
    if causal:
        vis = j <= pos
        if window:
            vis &= j > pos - window
    return vis


def probabilities(q, k, vis, scale):
    s = np.where(vis, scale * (q @ k.T), -np.inf)
    if s.shape[1] == 0:
        return s, np.full(s.shape[0], -np.inf)
    top = s.max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = top[:, 0] + np.log(total[:, 0])
    return p / np.where(total == 0, 1.0, total), lse


def head_forward(q, k, v, causal, window, scale):
    """One head of one sequence: out, lse."""
    p, lse = probabilities(q, k, visible(len(q), len(k), causal, window), scale)
    return p @ v, lse


def head_backward(q, k, v, g, causal, window, scale):
    """dq, dk, dv for the gradient g of out."""
    p, _ = probabilities(q, k, visible(len(q), len(k), causal, window), scale)
    dp = g @ v.T
    ds = p * (dp - (p * dp).sum(1, keepdims=True))
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ g


def score_error(q, k, scale):
    """Per query, a bound of the error of a score (natural units) formed by
    float32 sums of exact products, scaled and put through exp2: dim + 8
    roundings of at most the sum of magnitudes. The relative error of a
    probability is twice that (its own and that of the sum it is divided by)."""
    if len(k) == 0:
        return np.zeros((len(q), 1))
    return (q.shape[1] + 8) * U32 * scale * (np.abs(q) @ np.abs(k).T).max(1, keepdims=True)


def forward_bound(q, k, v, causal, window, scale, kind):
    """Bound of |out - exact|: probabilities rounded for the product (relative
    u; in fp16 those below its normal range by half of 2^-24 of the largest),
    scores in float32, m terms added in float32, and the rounding of out."""
    u = U[kind]
    p, lse = probabilities(q, k, visible(len(q), len(k), causal, window), scale)
    t = 2 * score_error(q, k, scale) + (len(k) + 8) * U32
    low = 2.0 ** -25 * np.abs(v).sum(0, keepdims=True) if kind == "fp16" else 0.0
    body = (u + t) * (p @ np.abs(v)) + low
    return body * (1 + u) + u * np.abs(p @ v) + (2.0 ** -25 if kind == "fp16" else 0.0)


def lse_bound(q, k, lse, scale):
    """One score's error, the sum's, and log's and the product's roundings."""
    t = score_error(q, k, scale)[:, 0] + (len(k) + 8) * U32
    return t + 4 * U32 * np.where(np.isfinite(lse), np.abs(lse) + 1.0, 0.0)


def backward_bound(q, k, v, g, out, causal, window, scale, kind):
    """Bounds of the errors of dq, dk, dv where out (as handed to the gradient)
    is exact up to its rounding and lse up to float32's."""
    u = U[kind]
    p, lse = probabilities(q, k, visible(len(q), len(k), causal, window), scale)
    lse = np.where(np.isfinite(lse), lse, 0.0)[:, None]
    t = score_error(q, k, scale) + 4 * U32 * (np.abs(lse) + 1.0)      # of p, relative
    dp = g @ v.T
    delta = (p * dp).sum(1, keepdims=True)
    ds = p * (dp - delta)
    d = q.shape[1] + 8
    e_dp = d * U32 * (np.abs(g) @ np.abs(v).T)
    e_delta = (u + d * U32) * (np.abs(g) * np.abs(out)).sum(1, keepdims=True)
    low = 2.0 ** -25 if kind == "fp16" else 0.0        # half the smallest fp16 step
    e_ds = p * (t * np.abs(dp - delta) + e_dp + e_delta)
    e_ds = e_ds * (1 + u) + u * np.abs(ds) + low * (p > 0)
    e_p = (u + t) * p * (1 + u) + low * (p > 0)
    n, m = len(q), len(k)
    dq, dk, dv = scale * (ds @ k), scale * (ds.T @ q), p.T @ g
    b_dq = scale * ((e_ds + m * U32 * np.abs(ds)) @ np.abs(k))
    b_dk = scale * ((e_ds + n * U32 * np.abs(ds)).T @ np.abs(q))
    b_dv = (e_p + n * U32 * p).T @ np.abs(g)
    return b_dq + u * (np.abs(dq) + b_dq) + low, b_dk, b_dv


def e4m3_round(x):
    """The nearest e4m3 number, ties to even; |x| <= 448."""
    _, e = np.frexp(x)                              # |x| = f 2^e, f in [1/2, 1)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def stored(x, kind):
    """What an 8-bit cache gives back for finite rows x (..., dim), and the
    scales of the rows."""
    top = 1.875 * 2.0 ** (15 if kind == "fp16" else 127)
    x = np.clip(np.asarray(x, dtype=np.float64), -top, top)
    most = np.abs(x).max(-1)
    f, e = np.frexp(most)
    e = np.where(f <= 0.875, e - 9, e - 8)
    e = np.maximum(e, -15 if kind == "fp16" else -110)
    s = np.where(most == 0, 1.0, np.ldexp(1.0, e))
    return e4m3_round(x / s[..., None]) * s[..., None], s
