"""Caches quantised elsewhere, whose scales are no powers of two; and many rows
over small pages, at products of every depth."""

import numpy as np
import pytest

from attention_common import f64, oracle_forward, rounded, starts, within

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()


def _table(rng, totals, page, spare=2):
    per = [-(-t // page) for t in totals]
    pages = sum(per) + spare
    order, table, at = rng.permutation(pages), np.zeros((len(totals), max(per)), dtype=np.int32), 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, table


def _eight(rng, kind, g, d, page, totals, scale_of):
    """A cache of random finite codes with scales scale_of(shape), and its rows
    as the 16-bit type holds them, float64."""
    import torch
    import paper_1806_06144_amd as ep
    pages, table = _table(rng, totals, page)
    dt = torch.bfloat16 if kind == "bf16" else torch.float16
    parts, rows = [], []
    for _ in range(2):
        code = rng.integers(0, 256, (pages, page, g, d)).astype(np.uint8)
        code[(code & 0x7f) == 0x7f] = 0x38                      # (NaN: 1 instead)
        scale = scale_of((pages, page, g)).astype(np.float32)
        value = torch.from_numpy(code).view(torch.float8_e4m3fn).float()
        value = (value * torch.from_numpy(scale)[..., None]).to(dt)
        parts.append((torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()))
        flat = value.reshape(pages * page, g, d)
        rows.append(torch.cat([flat[torch.from_numpy(table[b][np.arange(t) // page].astype(np.int64)) * page
                                    + torch.from_numpy(np.arange(t) % page)]
                               for b, t in enumerate(totals)]))
    (k, ks), (v, vs) = parts
    return ep.EpCache(k, v, ks, vs), _ints(table), rows, dt


def _amax_like(rng):
    """Scales as a division of rows' maxima by 448 leaves them, some powers of
    two, zeros and negative ones among them."""
    def make(shape):
        s = rng.uniform(0.5, 4.0, shape) / 448
        s[rng.random(shape) < 0.2] = 2.0 ** -8
        s[rng.random(shape) < 0.05] = 0.0
        s[rng.random(shape) < 0.05] *= -1
        return s
    return make


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("g,d,page,totals", [(2, 128, 16, [40, 129]), (1, 72, 4, [70]), (8, 8, 32, [33])])
def test_any_scale_is_read_as_it_is(kind, g, d, page, totals):
    """Values are code x scale, in float32, rounded to the 16-bit type."""
    import torch
    import paper_1806_06144_amd as ep
    rng = np.random.default_rng(d)
    cache, table, rows, dt = _eight(rng, kind, g, d, page, totals, _amax_like(rng))
    got = [torch.full((sum(totals), g, d), float("nan"), dtype=dt, device="cuda") for _ in range(2)]
    ep.ep_cache_read(cache, *got, table, _ints(totals), _ints(starts(totals)))
    for x, y in zip(got, rows):
        assert np.array_equal(f64(x), f64(y))


# new tokens, lengths, heads, kv_heads, dim, page, causal, window
MANY = [([1, 3], [300, 64], 8, 2, 128, 32, True, 0), ([2], [90], 4, 1, 64, 4, True, 0),
        ([100, 37], [300, 37], 4, 2, 128, 16, True, 0), ([90], [200], 4, 2, 64, 64, False, 0),
        ([130, 70], [130, 333], 4, 1, 96, 32, True, 0), ([70, 40], [150, 90], 6, 2, 128, 8, True, 50),
        ([65], [129], 4, 2, 64, 2, True, 0), ([90], [177], 3, 1, 80, 1, True, 0)]


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("case", MANY, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}.{c[3]}x{c[4]}-{c[5]}")
def test_attention_over_any_scale(kind, case):
    import torch
    import paper_1806_06144_amd as ep
    new, totals, h, g, d, page, causal, window = case
    rng = np.random.default_rng(d + page)
    cache, table, (k, v), dt = _eight(rng, kind, g, d, page, totals, _amax_like(rng))
    q = rounded(rng, (sum(new), h, d), kind)
    out, lse = torch.full_like(q.cuda(), float("nan")), torch.empty((sum(new), h), device="cuda")
    ep.ep_cache_attention(q.cuda(), cache, out, lse, table, _ints(totals), _ints(starts(new)), 0.1,
                          causal, window)
    want, l, b_out, b_lse = oracle_forward(f64(q), f64(k), f64(v), new, totals, causal, window,
                                           float(np.float32(0.1)), kind)
    within(f64(out), want, b_out, "out")
    within(f64(lse), l, b_lse, "lse")


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", MANY[2:], ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}.{c[3]}x{c[4]}-{c[5]}")
def test_many_rows_over_pages_of_any_size(kind, eight, case):
    """128-row workgroups over 16-bit and written 8-bit pages, those of fewer
    than 16 tokens among them, at products of depth 64, 96 and 128."""
    from test_gpu_cache import Cache
    new, totals, h, g, d, page, causal, window = case
    rng = np.random.default_rng(d)
    c = Cache(rng, kind, eight, g, d, page, totals)
    k, v = (rounded(rng, (sum(totals), g, d), kind) for _ in range(2))
    c.write(k.cuda(), v.cuda(), totals, totals)
    q = rounded(rng, (sum(new), h, d), kind)
    got = c.attend(q.cuda(), totals, new, 0.125, causal, window)
    out, lse, b_out, b_lse = oracle_forward(f64(q), c.values(k), c.values(v), new, totals, causal,
                                            window, 0.125, kind)
    within(f64(got[0]), out, b_out, "out")
    within(f64(got[1]), lse, b_lse, "lse")
    assert c.err.item() == 0
