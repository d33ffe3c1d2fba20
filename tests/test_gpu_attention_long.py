"""Long sequences: marked inputs, whose results show a tile of 32 keys or rows
that is left out or counted twice (attention_marks.py), and random ones by the
norm of a row's error."""

import numpy as np
import pytest

import attention_marks as am
import oracle.attention as oa
from attention_common import f64, within

pytestmark = pytest.mark.gpu


def _dtype(kind):
    import torch
    return torch.bfloat16 if kind == "bf16" else torch.float16


def _rows(x, heads, kind):
    """[tokens, dim] as device rows, the same for every head."""
    import torch
    x = torch.from_numpy(x).to(_dtype(kind)).cuda()
    return x[:, None].expand(-1, heads, -1).contiguous()


def _starts(n):
    import torch
    return torch.tensor([0, n], dtype=torch.int32, device="cuda")


# kind, heads, kv_heads, dim, queries, keys, causal, window
CASES = [("bf16", 2, 1, 64, 100000, 100000, True, 0),        # many rows, keys not cut
         ("fp16", 1, 1, 128, 30000, 30000, True, 0),
         ("fp16", 3, 1, 72, 300, 131072, False, 0),          # many rows, keys cut
         ("bf16", 2, 2, 128, 400, 60000, True, 0),
         ("bf16", 1, 1, 64, 20000, 20000, True, 5000),
         ("fp16", 4, 1, 64, 1, 100000, True, 0),             # few rows, keys cut
         ("bf16", 2, 1, 128, 5, 50000, True, 20000),
         ("fp16", 1, 1, 64, 40000, 300, False, 0)]           # many rows, few keys


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward_counts_every_key_once(case):
    import torch
    import paper_1806_06144_amd as ep
    kind, h, g, d, n, m, causal, window = case
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((n, h, d), device="cuda", generator=gen).to(_dtype(kind))
    k, v = _rows(np.zeros((m, d)), g, kind), _rows(am.marks(m, d), g, kind)
    out, lse = torch.empty_like(q), torch.empty((n, h), device="cuda")
    ep.ep_attention(q, k, v, out, lse, _starts(n), _starts(m), None, causal, window)
    want, l, b_out, b_lse = am.forward(n, m, d, causal, window, kind)
    for i in range(h):
        within(f64(out[:, i]), want, b_out, "out")
        within(f64(lse[:, i]), l, b_lse, "lse")


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_gradients_count_every_key_and_row_once(case):
    import torch
    import paper_1806_06144_amd as ep
    kind, h, g, d, n, m, causal, window = case
    want = am.Gradients(n, m, d, causal, window, 0.125, kind)
    dout, out = (_rows(x, h, kind) for x in (want.dout, want.out))
    lse = torch.from_numpy(want.lse).float().cuda()[:, None].expand(-1, h).contiguous()
    v = _rows(want.v, g, kind)
    group = h // g

    def run(q, k):
        q, k = _rows(q, h, kind), _rows(k, g, kind)
        grads = [torch.full_like(x, float("nan")) for x in (q, k, v)]
        ep.ep_attention_backward(dout, q, k, v, out, lse, *grads, _starts(n), _starts(m), 0.125,
                                 causal, window)
        return grads

    def check(x, pair, times, name):
        w, b = pair
        for i in range(x.shape[1]):
            within(f64(x[:, i]), times * w, times * b, name)
    dq, dk, dv = run(np.zeros((n, d)), am.marks(m, d))
    check(dq, want.dq(), 1, "dq")
    check(dv, want.dv(), group, "dv")
    assert (dk == 0).all()
    dq, dk, dv = run(am.marks(n, d), np.zeros((m, d)))
    check(dk, want.dk(), group, "dk")
    check(dv, want.dv(), group, "dv")
    assert (dq == 0).all()


@pytest.mark.parametrize("store", ["same", "e4m3"])
@pytest.mark.parametrize("kind,d,n,m,page,causal,window", [("bf16", 64, 1, 131072, 64, True, 0),
                                                           ("fp16", 128, 3, 50000, 16, True, 0),
                                                           ("bf16", 128, 2, 30000, 8, True, 9000),
                                                           ("fp16", 64, 200, 60000, 256, True, 0),
                                                           ("bf16", 128, 3000, 20000, 16, True, 0),
                                                           ("fp16", 96, 300, 20000, 4, False, 0)])
def test_cache_attention_counts_every_key_once(store, kind, d, n, m, page, causal, window):
    import torch
    import paper_1806_06144_amd as ep
    h, g = 4, 2
    pages = -(-m // page)
    shape = (pages, page, g, d)
    dt = torch.float8_e4m3fn if store == "e4m3" else _dtype(kind)
    kp, vp = (torch.zeros(shape, dtype=torch.uint8 if store == "e4m3" else dt, device="cuda")
              for _ in range(2))
    kp, vp = kp.view(dt), vp.view(dt)
    scales = ([torch.full(shape[:3], float("nan"), device="cuda") for _ in range(2)]
              if store == "e4m3" else [])
    cache = ep.EpCache(kp, vp, *scales)
    table = torch.arange(pages, dtype=torch.int32).flip(0)[None].contiguous().cuda()
    length = torch.tensor([m], dtype=torch.int32, device="cuda")
    ep.ep_cache_write(cache, _rows(np.zeros((m, d)), g, kind), _rows(am.marks(m, d), g, kind), table,
                      length, _starts(m))
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((n, h, d), device="cuda", generator=gen).to(_dtype(kind))
    out, lse = torch.empty_like(q), torch.empty((n, h), device="cuda")
    ep.ep_cache_attention(q, cache, out, lse, table, length, _starts(n), None, causal, window)
    want, l, b_out, b_lse = am.forward(n, m, d, causal, window, kind)
    for i in range(h):
        within(f64(out[:, i]), want, b_out, "out")
        within(f64(lse[:, i]), l, b_lse, "lse")


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_random_rows_by_norm(kind):
    """Rows of 100000 keys. A row's error comes from independent roundings, of
    its probabilities (of p (dp - D)) and of the result, each u / sqrt(3) of
    its norm at most in the mean of squares: 0.82 u together; 2 u leaves room
    for 64 elements' chance. 64 keys left out would be 0.025, in bf16 2 u is
    0.0078. Log-sums: a score's bound and the sum's steps, which grow with the
    2000 additions of a lane at most."""
    import torch
    import paper_1806_06144_amd as ep
    n, d, scale = 100000, 64, 0.125
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k, v, go = (torch.randn((n, 1, d), device="cuda", generator=gen).to(_dtype(kind))
                   for _ in range(4))
    out, lse = torch.empty_like(q), torch.empty((n, 1), device="cuda")
    grads = [torch.empty_like(q) for _ in range(3)]
    s = _starts(n)
    ep.ep_attention(q, k, v, out, lse, s, s, scale)
    ep.ep_attention_backward(go, q, k, v, out, lse, *grads, s, s, scale)
    q64, k64, v64, g64 = (f64(x)[:, 0] for x in (q, k, v, go))
    u = oa.U[kind]
    low = 8 * 2.0 ** -25 if kind == "fp16" else 0.0      # 64 roundings below fp16's normal range
    for i in [n - 1, *np.random.default_rng(0).integers(n // 2, n, 10)]:
        args = q64[i:i + 1], k64[:i + 1], v64[:i + 1]
        o, l = oa.head_forward(*args, True, 0, scale)
        dq = oa.head_backward(*args, g64[i:i + 1], True, 0, scale)[0]
        for got, want, name in ((out, o, "out"), (grads[0], dq, "dq")):
            off = np.linalg.norm(f64(got[i, 0]) - want[0])
            assert off <= 2 * u * np.linalg.norm(want) + low, (name, i)
        room = 2 * oa.score_error(args[0], args[1], scale)[0, 0] + 2000 * oa.U32
        assert abs(f64(lse[i])[0] - l[0]) <= room
