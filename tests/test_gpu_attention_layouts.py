"""Rows whose heads lie far apart: [heads, tokens, dim] arrays and strides
where offsets of a tile's rows leave 32 bits."""

import numpy as np
import pytest

from attention_common import f64, oracle_backward, oracle_forward, rounded, within
from test_gpu_attention import _backward, _forward

pytestmark = pytest.mark.gpu


def _check(views, n, m, kind, causal, scale, seed=0):
    """views: q, k, v, dout, out, dq, dk, dv."""
    import torch
    qw, kw, vw, gw, ow, *grads = views
    rng = np.random.default_rng(seed)
    q, k, v, go = (rounded(rng, tuple(x.shape), kind) for x in (qw, kw, vw, gw))
    for x, y in zip((qw, kw, vw, gw), (q, k, v, go)):
        x.copy_(y)
    for x in (ow, *grads):
        x.fill_(float("nan"))
    out, lse = _forward(qw, kw, vw, n, m, scale, causal, out=ow)
    o64, l64, b_out, b_lse = oracle_forward(f64(q), f64(k), f64(v), n, m, causal, 0, scale, kind)
    within(f64(out), o64, b_out, "out")
    within(f64(lse), l64, b_lse, "lse")
    _backward(gw, qw, kw, vw, out, lse, n, m, scale, causal, into=grads)
    want, bound = oracle_backward(f64(q), f64(k), f64(v), f64(go), np.abs(f64(out)) + np.abs(o64), n, m,
                                  causal, 0, scale, kind)
    for x, w, b, name in zip(grads, want, bound, ("dq", "dk", "dv")):
        within(f64(x), w, b, name)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("h,g,d,n,m", [(8, 2, 64, [200, 33], [200, 33]), (6, 2, 128, [150], [70]),
                                       (4, 4, 72, [1, 90], [600, 90]), (40, 1, 64, [30], [100])])
def test_head_major_arrays(kind, h, g, d, n, m):
    import torch
    dt = torch.bfloat16 if kind == "bf16" else torch.float16

    def make(tokens, heads):
        return torch.empty((heads, tokens, d), dtype=dt, device="cuda").transpose(0, 1)
    t, s = sum(n), sum(m)
    views = [make(t, h), make(s, g), make(s, g), make(t, h), make(t, h), make(t, h), make(s, g),
             make(s, g)]
    _check(views, n, m, kind, True, 0.125)


@pytest.mark.parametrize("head", [(1 << 27) - 8, 1 << 27, (1 << 27) + 8])
def test_heads_a_quarter_of_a_gigabyte_apart(head):
    """Groups of four heads that span just under 2^30 bytes, 2^30 and more."""
    import torch
    n, h, g, d = 150, 8, 2, 64
    flat = torch.empty(h * head + 8 * n * d, dtype=torch.bfloat16, device="cuda")
    views = [flat.as_strided((n, x, d), (8 * d, head, 1), i * d)
             for i, x in enumerate((h, g, g, h, h, h, g, g))]
    _check(views, [n], [n], "bf16", True, 0.125)
