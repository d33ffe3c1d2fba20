"""The bounds of the marked long sequences (attention_marks.py) show a tile of
32 keys or rows that is left out, checked on results of the oracle that leave
one out; and its running sums agree with the oracle's products."""

import numpy as np
import pytest

import attention_marks as am
import oracle.attention as oa


@pytest.mark.parametrize("n,m,causal,window", [(70, 70, True, 0), (5, 200, True, 0), (40, 90, False, 0),
                                               (130, 130, True, 40), (90, 60, True, 0),
                                               (90, 60, True, 33)])
def test_running_sums_are_the_oracles(n, m, causal, window):
    dim, scale, kind = 16, 0.25, "bf16"
    zero = np.zeros
    out, lse, _, _ = am.forward(n, m, dim, causal, window, kind)
    o, l = oa.head_forward(zero((n, dim)), zero((m, dim)), am.marks(m, dim), causal, window, scale)
    assert np.allclose(out, o, atol=1e-13) and np.allclose(lse, l, atol=1e-13)
    g = am.Gradients(n, m, dim, causal, window, scale, kind)
    o, l = oa.head_forward(zero((n, dim)), zero((m, dim)), g.v, causal, window, scale)
    assert np.allclose(g.out, o, atol=1e-13) and np.allclose(g.lse, l, atol=1e-13)
    dq, _, dv = oa.head_backward(zero((n, dim)), am.marks(m, dim), g.v, g.dout, causal, window, scale)
    _, dk, dv2 = oa.head_backward(am.marks(n, dim), zero((m, dim)), g.v, g.dout, causal, window, scale)
    for got, want in ((g.dq()[0], dq), (g.dk()[0], dk), (g.dv()[0], dv), (g.dv()[0], dv2)):
        assert np.allclose(got, want, atol=1e-13)


def _shown(right, wrong, bound, rows):
    """The share of the rows of which some element lies outside its bound."""
    off = np.abs(wrong - right) > bound
    return off.reshape(len(off), -1).any(1)[rows].mean()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n,m,dim,causal,window", [(100000, 100000, 64, True, 0),
                                                   (300, 131072, 64, False, 0),
                                                   (20000, 20000, 128, True, 5000)])
def test_a_lost_tile_shows(kind, n, m, dim, causal, window):
    """Every row that sees the lost keys shows them. Of lost rows, the keys
    that see at most 20000 rows of probabilities like theirs show them."""
    lost = (m // 2, m // 2 + am.TILE)
    lo, hi = am.seen(n, m, causal, window)
    hit = (lo <= lost[0]) & (hi >= lost[1])
    out, lse, b_out, b_lse = am.forward(n, m, dim, causal, window, kind)
    o, l, _, _ = am.forward(n, m, dim, causal, window, kind, lost)
    assert _shown(out, o, b_out, hit) == 1.0
    # a log-sum's own precision: 32 keys of 131072 are 2.4e-4, its bound 6e-6
    assert _shown(lse[:, None], l[:, None], b_lse[:, None], hit) == 1.0
    g = am.Gradients(n, m, dim, causal, window, 0.125, kind)
    want, bound = g.dq()
    assert _shown(want, g.dq(lost)[0], bound, hit) == 1.0
    rows = (n // 2, n // 2 + am.TILE)
    lo, hi = am.seers(n, m, causal, window)
    near = (lo <= rows[0]) & (hi >= rows[1]) & (lo > rows[0] - 10000)
    for got in (g.dv, g.dk):
        want, bound = got()
        assert _shown(want, got(rows)[0], bound, near if causal else slice(None)) == 1.0
