"""Probabilities and gradients over fp16's range: many keys make both small,
where the type has few bits or none."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _exact(q, k, v, g, scale, causal):
    """One head's gradients on the device in float64, elementary products of a
    few thousand rows at a time."""
    import torch
    q, k, v, g = (x.double() for x in (q, k, v, g))
    n, m = q.shape[0], k.shape[0]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    out, lse = torch.zeros_like(q), torch.zeros(n, dtype=torch.float64, device=q.device)
    kt, vt = k.t().contiguous(), v.t().contiguous()
    for a in range(0, n, 2048):
        r = slice(a, min(a + 2048, n))
        s = (q[r] @ kt) * scale
        if causal:
            pos = torch.arange(r.start, r.stop, device=q.device) + (m - n)
            s.masked_fill_(torch.arange(m, device=q.device)[None] > pos[:, None], -float("inf"))
        top = s.amax(1, keepdim=True)
        p = (s - top).exp()
        total = p.sum(1, keepdim=True)
        lse[r] = (top + total.log())[:, 0]
        p /= total
        out[r] = p @ v
        dv += p.t().contiguous() @ g[r]
        dp = g[r] @ vt
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        dq[r] = scale * (ds @ k)
        dk += scale * (ds.t().contiguous() @ q[r])
    return out, lse, (dq, dk, dv)


@pytest.mark.parametrize("n,m,d,causal,size", [(300, 131072, 64, False, 1.0),
                                               (300, 131072, 64, False, 2.0 ** -8),
                                               (40000, 40000, 64, True, 1.0),
                                               (300, 40000, 128, True, 32.0)])
def test_fp16_gradients_of_many_keys(n, m, d, causal, size):
    """By the norm of the error beside that of the exact result rounded to
    fp16 (which holds the loss of what fp16 cannot say at all). Probabilities,
    p (dp - D) and the result are each rounded once, relative to their size
    and independently: sqrt(2) times; D from a rounded out and float32 sums
    add a little: at most 2."""
    import torch
    import paper_1806_06144_amd as ep
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    q, g = (torch.randn((n, 1, d), device="cuda", generator=gen).half() for _ in range(2))
    k, v = (torch.randn((m, 1, d), device="cuda", generator=gen).half() for _ in range(2))
    g = (g * size).half()
    scale = d ** -0.5
    out, lse, want = _exact(q[:, 0], k[:, 0], v[:, 0], g[:, 0], float(np.float32(scale)), causal)
    sq, sk = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, m))
    grads = [torch.full_like(x, float("nan")) for x in (q, k, v)]
    ep.ep_attention_backward(g, q, k, v, out.half()[:, None].contiguous(),
                             lse.float()[:, None].contiguous(), *grads, sq, sk, scale, causal)
    for x, w, name in zip(grads, want, ("dq", "dk", "dv")):
        off = (x[:, 0].double() - w).norm().item()
        least = (w.half().double() - w).norm().item()
        print(f"{name}: {off / least:.3f} times the rounded result's error")
        assert off <= 2 * least, name


def test_fp16_slopes_past_the_range():
    """p (dp - D) above 65504 in every other row and below 1e-3 in the others,
    of which dq and dk lie within the range: keys and queries are small."""
    import torch
    import paper_1806_06144_amd as ep
    n, m, d, scale = 70, 90, 64, 0.125
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, g = (torch.randn((n, 1, d), device="cuda", generator=gen) for _ in range(2))
    k, v = (torch.randn((m, 1, d), device="cuda", generator=gen) for _ in range(2))
    large = (torch.arange(n, device="cuda") % 2 == 0)[:, None, None]
    g = (g * torch.where(large, 2.0 ** 13, 2.0 ** -10)).half()
    q, k, v = (q * 2.0 ** -9).half(), (k * 2.0 ** -9).half(), (v * 64).half()
    out, lse, want = _exact(q[:, 0], k[:, 0], v[:, 0], g[:, 0], scale, False)
    s = v[:, 0].double() @ g[:, 0].double().t().contiguous() / m     # (scores are below 0.001)
    assert (s - s.mean(0)).abs().max() > 1e5
    sq, sk = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, m))
    grads = [torch.full_like(x, float("nan")) for x in (q, k, v)]
    ep.ep_attention_backward(g, q, k, v, out.half()[:, None].contiguous(),
                             lse.float()[:, None].contiguous(), *grads, sq, sk, scale, False)
    # The terms of an element add up, rounded by 2^-11 of each, to at most
    # scale 2^-11 sum |ds| |k| (|q|), and 2^-11 of the result; float32 and the
    # result's own smallest step beside that.
    ds = ((s - s.mean(0)).abs().t().contiguous() * 1.01)
    for x, w, terms in ((grads[0], want[0], ds @ k[:, 0].double().abs()),
                        (grads[1], want[1], ds.t().contiguous() @ q[:, 0].double().abs()),
                        (grads[2], want[2], (g[:, 0].double().abs().sum(0) / m / scale)[None])):
        room = 1.1 * 2.0 ** -11 * (scale * terms + w.abs()) + 2.0 ** -25
        assert x.isfinite().all() and ((x[:, 0].double() - w).abs() <= room).all()


@pytest.mark.parametrize("n,g,terms", [(1, 1, 512), (200, 1, 512), (1, 2048, 16384), (40, 512, 65536)])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_many_small_probabilities_beside_a_large_one(kind, n, g, terms):
    """One key's probability 1, before the division, and 131071 of 1.5 x 2^-24
    beside it, together 0.0117: below what fp16 holds with any accuracy. Keys
    cut over workgroups or, where there are many heads (all of them alike, by
    a stride of 0), not; terms: that a lane adds at most."""
    import torch
    import paper_1806_06144_amd as ep
    from oracle.attention import U
    dt = torch.float16 if kind == "fp16" else torch.bfloat16
    m, d = 131072, 64
    q = torch.zeros((n, g, d), dtype=dt, device="cuda")
    q[:, :, 0] = 16.0                                # scores 16 k[0]: 0, and -16.25
    k, v = (torch.zeros((m, 1, d), dtype=dt, device="cuda") for _ in range(2))
    k[1:, 0, 0] = -1.015625
    v[1:] = 1.0
    k, v = (x.expand(-1, g, -1) for x in (k, v))
    s, t = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, m))
    out, lse = torch.empty_like(q), torch.empty((n, g), device="cuda")
    ep.ep_attention(q, k, v, out, lse, s, t, 1.0, False)
    rest = (m - 1) * np.exp(-16.25)
    want = rest / (1 + rest)
    # all probabilities are rounded alike (relative u), then the result; each of a lane's terms
    # costs its float32 sum a step beside the large one, and exp2 some (an exponent of 23.4)
    room = (terms + 64) * 2.0 ** -23
    assert (out.double() - want).abs().max().item() <= want * (2 * U[kind] + room)
    assert (lse.double() - np.log1p(rest)).abs().max().item() <= 4e-6 + room
