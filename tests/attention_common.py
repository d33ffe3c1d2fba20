"""Inputs, calls and checks shared by the attention tests."""

import numpy as np

import oracle.attention as oa


def starts(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def rounded(rng, shape, kind, size=1.0):
    """Normal values that the 16-bit type holds exactly, as a tensor."""
    import torch
    x = torch.from_numpy(rng.standard_normal(shape) * size)
    return x.to(torch.bfloat16 if kind == "bf16" else torch.float16)


def f64(x):
    return x.detach().cpu().double().numpy()


def oracle_forward(q, k, v, nq, nk, causal, window, scale, kind):
    """q [Tq, H, D], k, v [Tk, G, D] float64; out, lse and their bounds."""
    sq, sk = starts(nq), starts(nk)
    h, g = q.shape[1], k.shape[1]
    out, b_out = np.zeros(q.shape), np.zeros(q.shape)
    lse, b_lse = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    for b in range(len(nq)):
        r, c = slice(sq[b], sq[b + 1]), slice(sk[b], sk[b + 1])
        for i in range(h):
            j = i // (h // g)
            args = q[r, i], k[c, j], v[c, j]
            out[r, i], lse[r, i] = oa.head_forward(*args, causal, window, scale)
            b_out[r, i] = oa.forward_bound(*args, causal, window, scale, kind)
            b_lse[r, i] = oa.lse_bound(q[r, i], k[c, j], lse[r, i], scale)
    return out, lse, b_out, b_lse


def oracle_backward(q, k, v, g, out, nq, nk, causal, window, scale, kind):
    """dq, dk, dv and their bounds."""
    sq, sk = starts(nq), starts(nk)
    h, kv = q.shape[1], k.shape[1]
    grads = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)]
    bounds = [np.zeros(x.shape) for x in grads]
    for b in range(len(nq)):
        r, c = slice(sq[b], sq[b + 1]), slice(sk[b], sk[b + 1])
        for i in range(h):
            j = i // (h // kv)
            args = q[r, i], k[c, j], v[c, j], g[r, i]
            places = [(r, i), (c, j), (c, j)]
            got = oa.head_backward(*args, causal, window, scale)
            far = oa.backward_bound(*args, out[r, i], causal, window, scale, kind)
            for x, y, p, a, e in zip(grads, bounds, places, got, far):
                x[p] += a
                y[p] += e
    u = oa.U[kind]
    low = 2.0 ** -25 if kind == "fp16" else 0.0
    for i in (1, 2):                                # rounded after the group's sum
        bounds[i] = bounds[i] * (1 + u) + u * np.abs(grads[i]) + low
    return grads, bounds


def within(got, want, bound, name):
    """Every element within its bound (and equal where that is not a number)."""
    got = np.asarray(got, dtype=np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), name
    assert np.isfinite(got[fine]).all(), f"{name}: not finite"
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    assert off.size == 0 or off.max() <= 1e-30, (
        f"{name}: {off.max():.3e} past its bound, {np.mean(off > 1e-30):.2%} of the elements")
