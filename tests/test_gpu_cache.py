"""The paged cache: writing, 8-bit rows and reading back against the float64
oracle, and attention over it; pages that end inside a tile, stale slots, bad
page numbers, offsets past 32 bits; and a run of all calls together."""

import numpy as np
import pytest

import oracle.attention as oa
from attention_common import f64, oracle_forward, rounded, starts, within

pytestmark = pytest.mark.gpu


class Cache:
    """A cache of shuffled pages with stale slots of NaN."""

    def __init__(self, rng, kind, eight, kv_heads, dim, page, totals, spare=2, cols=None):
        import torch
        import paper_1806_06144_amd as ep
        self.ep, self.torch = ep, torch
        self.kind, self.eight, self.page = kind, eight, page
        self.dtype = torch.bfloat16 if kind == "bf16" else torch.float16
        per = [-(-t // page) for t in totals]
        pages = sum(per) + spare
        order = rng.permutation(pages)
        self.table_np = np.full((len(totals), cols or max(max(per), 1)), -7, dtype=np.int32)
        at = 0
        for b, n in enumerate(per):
            self.table_np[b, :n] = order[at:at + n]
            at += n
        shape = (pages, page, kv_heads, dim)
        if eight:
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda")
                              for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:3], float("nan"), device="cuda")
                                for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=self.dtype, device="cuda")
                              for _ in range(2))
            self.ks = self.vs = None
        self.c = ep.EpCache(self.k, self.v, self.ks, self.vs)
        self.table = torch.from_numpy(self.table_np).cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def ints(self, x):
        return self.torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()

    def write(self, k, v, lengths, new):
        self.ep.ep_cache_write(self.c, k, v, self.table, self.ints(lengths), self.ints(starts(new)),
                               self.err)

    def read(self, like, lengths):
        t = int(sum(lengths))
        out = [self.torch.full((t,) + tuple(like.shape[1:]), float("nan"), dtype=self.dtype,
                               device="cuda") for _ in range(2)]
        self.ep.ep_cache_read(self.c, *out, self.table, self.ints(lengths),
                              self.ints(starts(lengths)), self.err)
        return out

    def attend(self, q, lengths, new, scale=None, causal=True, window=0):
        out = self.torch.full(tuple(q.shape), float("nan"), dtype=q.dtype, device="cuda")
        lse = self.torch.full(tuple(q.shape[:2]), float("nan"), device="cuda")
        self.ep.ep_cache_attention(q, self.c, out, lse, self.table, self.ints(lengths),
                                   self.ints(starts(new)), scale, causal, window, self.err)
        return out, lse

    def values(self, x):
        """What the cache should give back for rows x, float64."""
        return oa.stored(f64(x), self.kind)[0] if self.eight else f64(x)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("kv_heads,dim,page,totals", [(2, 128, 16, [40, 1, 0, 129]),
                                                      (3, 64, 64, [64, 200]), (1, 72, 1, [5, 9]),
                                                      (8, 8, 32, [33]), (1, 120, 4096, [100])])
def test_write_and_read_back(kind, eight, kv_heads, dim, page, totals):
    rng = np.random.default_rng(dim + page)
    c = Cache(rng, kind, eight, kv_heads, dim, page, totals)
    # rows of very different sizes, zeros and single values among them
    shape = (sum(totals), kv_heads, dim)
    size = 2.0 ** rng.integers(-12, 12, shape[:2] + (1,)) * (rng.random(shape) < 0.7)
    size[:1] = 0.0
    k, v = (rounded(rng, shape, kind, size).cuda() for _ in range(2))
    c.write(k, v, totals, totals)
    got = c.read(k, totals)
    for x, y in zip(got, (k, v)):
        assert np.array_equal(f64(x), c.values(y))
    assert c.err.item() == 0
    # untouched slots stay stale
    written = sum(totals) * kv_heads * dim
    stale = (c.k == 0x7f).sum().item() if eight else c.k.isnan().sum().item()
    assert stale == c.k.numel() - written


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_every_8_bit_rounding(kind):
    """All finite values of a type's positive range, a row per power of two,
    both signs; the largest, the smallest and the ones that saturate."""
    import torch
    bits = torch.arange(0, 0x7c00 if kind == "fp16" else 0x7f80, dtype=torch.int32)
    x = bits.to(torch.int16).view(torch.float16 if kind == "fp16" else torch.bfloat16)
    x = torch.cat([x, -x])
    x = x[:x.numel() // 128 * 128].view(-1, 1, 128)
    rng = np.random.default_rng(0)
    rows = torch.cat([x, x.flatten()[torch.from_numpy(rng.permutation(x.numel()))].view(x.shape)])
    c = Cache(rng, kind, True, 1, 128, 256, [rows.shape[0]])
    rows = rows.cuda()
    c.write(rows, rows, [rows.shape[0]], [rows.shape[0]])
    k, v = c.read(rows, [rows.shape[0]])
    want, scales = oa.stored(f64(rows), kind)
    assert np.array_equal(f64(k), want) and np.array_equal(f64(v), want)
    pages = c.ks[c.table.long()[0]].view(-1)[:rows.shape[0]]
    assert np.array_equal(f64(pages), scales[:, 0])


def test_not_finite_values_become_nan():
    import torch
    rng = np.random.default_rng(0)
    c = Cache(rng, "bf16", True, 1, 64, 16, [3])
    k = torch.ones((3, 1, 64), dtype=torch.bfloat16)
    k[0, 0, 3], k[1, 0, 5], k[2] = float("inf"), float("nan"), float("-inf")
    k = k.cuda()
    c.write(k, k, [3], [3])
    got, _ = c.read(k, [3])
    assert got.isnan().sum().item() == 2 + 64 and got[0, 0, 3].isnan() and got[1, 0, 5].isnan()
    assert (got[0, 0, :3] == 1).all() and c.ks.isfinite().sum().item() == 3


# kind, 8-bit, heads, kv_heads, dim, page, new tokens, lengths, causal, window
ATTEND = [
    ("bf16", False, 4, 4, 128, 16, [1], [1], True, 0),
    ("bf16", False, 32, 8, 128, 16, [1], [511], True, 0),
    ("fp16", False, 8, 2, 64, 64, [1, 1, 1], [1000, 64, 65], True, 0),
    ("bf16", True, 8, 2, 128, 32, [1, 1], [700, 31], True, 0),
    ("fp16", True, 8, 1, 128, 32, [4, 1], [300, 2], True, 0),
    ("bf16", False, 6, 2, 72, 8, [1, 0, 5], [129, 40, 5], True, 0),     # no new tokens in one
    ("bf16", True, 3, 3, 40, 1, [2, 1], [70, 1], True, 0),
    ("fp16", False, 4, 2, 128, 16, [100, 37], [300, 37], True, 0),
    ("bf16", False, 4, 1, 64, 128, [200], [777], True, 0),
    ("bf16", True, 4, 2, 128, 64, [130], [401], True, 0),
    ("fp16", True, 4, 2, 64, 16, [65], [65], True, 0),
    ("bf16", False, 4, 2, 128, 16, [1, 9], [900, 400], True, 100),      # window
    ("bf16", True, 16, 2, 128, 256, [1], [2000], True, 1),
    ("bf16", False, 4, 2, 64, 16, [7, 20], [50, 33], False, 0),
    ("bf16", False, 4, 2, 64, 16, [5, 3], [0, 2], True, 0),             # fewer tokens than queries
    ("bf16", False, 40, 1, 128, 16, [1, 3], [600, 90], True, 0),        # a group of 40
    ("bf16", False, 2, 1, 64, 32, [1], [20000], True, 0),
    ("fp16", True, 2, 2, 128, 16, [2] * 70, [33] * 70, True, 0),
    ("bf16", False, 8, 8, 128, 16, [1] * 5, [3000, 1, 17, 1500, 256], True, 0),
]


def _fill(case, seed=1, spare=2, cols=None):
    kind, eight, h, g, d, page, new, totals, causal, window = case
    rng = np.random.default_rng(seed + d + len(new))
    c = Cache(rng, kind, eight, g, d, page, totals, spare, cols)
    k, v = (rounded(rng, (sum(totals), g, d), kind) for _ in range(2))
    if sum(totals):
        c.write(k.cuda(), v.cuda(), totals, totals)
    q = rounded(rng, (sum(new), h, d), kind)
    return c, q, c.values(k), c.values(v)


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}.{c[3]}x{c[4]}-{c[5]}-{c[6][:3]}-{c[7][:3]}-{c[8]}-{c[9]}")
def test_cache_attention(case):
    kind, eight, h, g, d, page, new, totals, causal, window = case
    c, q, k, v = _fill(case)
    scale = float(np.float32(d ** -0.5))
    got = c.attend(q.cuda(), totals, new, scale, causal, window)
    out, lse, b_out, b_lse = oracle_forward(f64(q), k, v, new, totals, causal, window, scale, kind)
    within(f64(got[0]), out, b_out, "out")
    within(f64(got[1]), lse, b_lse, "lse")
    assert c.err.item() == 0


@pytest.mark.parametrize("new,total", [(1, 5000), (140, 2000)])
def test_rows_of_no_sequence_stay_as_they_are(new, total):
    """Rows before the first and behind the last sequence, where the keys are
    cut and where they are not."""
    import torch
    for wide in (1, 60):
        case = ("bf16", False, 4, 2, 64, 16, [new], [total], True, 0)
        c, q, k, v = _fill(case, cols=wide * -(-total // 16))
        pad = rounded(np.random.default_rng(0), (20, 4, 64), "bf16")
        rows = torch.cat([pad[:9], q, pad[9:]]).cuda()
        out = torch.full_like(rows, 7.0)
        lse = torch.full(tuple(rows.shape[:2]), 7.0, device="cuda")
        c.ep.ep_cache_attention(rows, c.c, out, lse, c.table, c.ints([total]), c.ints([9, 9 + new]),
                                0.1, err=c.err)
        want, l, b_out, b_lse = oracle_forward(f64(q), k, v, [new], [total], True, 0, 0.1, "bf16")
        within(f64(out[9:9 + new]), want, b_out, "out")
        within(f64(lse[9:9 + new]), l, b_lse, "lse")
        for x in (out, lse):
            assert (x[:9] == 7).all() and (x[9 + new:] == 7).all()


def test_a_table_much_wider_than_the_sequences():
    case = ("bf16", False, 4, 2, 128, 16, [1, 1], [40, 700], True, 0)
    c, q, k, v = _fill(case, cols=60000)
    got = c.attend(q.cuda(), case[7], case[6], 0.1)
    out, lse, b_out, b_lse = oracle_forward(f64(q), k, v, case[6], case[7], True, 0, 0.1, "bf16")
    within(f64(got[0]), out, b_out, "out")
    within(f64(got[1]), lse, b_lse, "lse")


@pytest.mark.parametrize("new", [1, 90])
def test_bad_pages_and_lengths_are_reported_and_reach_nothing_else(new):
    """The other sequence's results are what they are without the bad one."""
    case = ("bf16", False, 4, 2, 64, 16, [new, new], [200, 100], True, 0)
    c, q, k, v = _fill(case)
    for x in (c.k, c.v):                             # (page 0 stands in for a bad one)
        x.nan_to_num_()
    want, _ = c.attend(q.cuda(), [200, 100], [new, new])
    assert c.err.item() == 0
    good = c.table.clone()
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table.copy_(good)
        c.table[0, 3] = bad
        c.err.zero_()
        out, _ = c.attend(q.cuda(), [200, 100], [new, new])
        assert c.err.item() == 1 and (out[new:] == want[new:]).all()
    c.table.copy_(good)
    for length in (2 ** 31 - 1, -3, 16 * c.table.shape[1] + 1):
        c.err.zero_()
        out, _ = c.attend(q.cuda(), [length, 100], [new, new])
        assert c.err.item() == 1 and (out[new:] == want[new:]).all()


def test_bad_places_are_not_written_or_read():
    import torch
    case = ("fp16", False, 2, 2, 64, 16, [1, 1], [40, 40], True, 0)
    c, _, _, _ = _fill(case)
    before = c.k.clone()
    k = torch.ones((2, 2, 64), dtype=torch.float16, device="cuda")
    good = c.table.clone()
    for bad, length in ((-1, 40), (c.k.shape[0], 40), (None, 0), (None, 10 ** 9), (None, -5)):
        c.table.copy_(good)
        if bad is not None:
            c.table[:, 2] = bad
        c.err.zero_()
        c.write(k, k, [length, length], [1, 1])
        assert c.err.item() == 1
        assert torch.equal(c.k.view(torch.int16), before.view(torch.int16))
    c.table.copy_(good)
    c.table[1, 1] = 99
    c.err.zero_()
    out = [torch.full((80, 2, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    c.ep.ep_cache_read(c.c, *out, c.table, c.ints([40, 40]), c.ints([0, 40, 80]), c.err)
    assert c.err.item() == 1 and (out[0][56:72] == 7).all()
    assert (out[0][:40] != 7).all() and (out[0][72:] != 7).all()


def test_offsets_past_32_bits():
    """A cache of 5 GB whose used pages are its last ones, and whose first 4 GB
    hold other values."""
    import torch
    import paper_1806_06144_amd as ep
    pages, page, g, d = 40000, 64, 8, 128            # 131072 bytes a page
    k, v = (torch.empty((pages, page, g, d), dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    rng = np.random.default_rng(0)
    n = 300
    used = torch.tensor([[39999, 39990, 35000, 33001, 32769]], dtype=torch.int32, device="cuda")
    for x in (k, v):
        x[used[0].long() - 32768] = float("nan")     # where a 32-bit byte offset would land
    kn, vn = (rounded(rng, (n, g, d), "bf16") for _ in range(2))
    c = ep.EpCache(k, v)
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    s = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ep.ep_cache_write(c, kn.cuda(), vn.cuda(), used, lengths, s)
    back = [torch.empty((n, g, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ep.ep_cache_read(c, *back, used, lengths, s)
    assert torch.equal(back[0].cpu(), kn) and torch.equal(back[1].cpu(), vn)
    for new in (1, 130):
        q = rounded(rng, (new, 16, d), "bf16")
        out = torch.empty((new, 16, d), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((new, 16), device="cuda")
        s1 = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        ep.ep_cache_attention(q.cuda(), c, out, lse, used, lengths, s1, 0.1)
        want, l, b_out, b_lse = oracle_forward(f64(q), f64(kn), f64(vn), [new], [n], True, 0, 0.1,
                                               "bf16")
        within(f64(out), want, b_out, "out")
        within(f64(lse), l, b_lse, "lse")


@pytest.mark.parametrize("eight", [False, True])
def test_prompt_chunks_and_tokens_together(eight):
    """Two sequences served as a program does: a prompt in two chunks, then
    single tokens, every step written and attended; each step's outputs are
    those of attention over everything so far."""
    import torch
    kind, h, g, d, page = "bf16", 8, 2, 128, 16
    steps = [[70, 21], [50, 0], [1, 1], [1, 1], [3, 1]]
    totals = np.sum(steps, 0)
    rng = np.random.default_rng(8)
    c = Cache(rng, kind, eight, g, d, page, totals)
    k, v = ([rounded(rng, (t, g, d), kind) for t in totals] for _ in range(2))
    q = [rounded(rng, (t, h, d), kind) for t in totals]
    done = np.zeros(2, dtype=int)
    for new in steps:
        rows = [slice(a, a + n) for a, n in zip(done, new)]
        done = done + new
        kn, vn, qn = (torch.cat([x[b][rows[b]] for b in range(2)]) for x in (k, v, q))
        c.write(kn.cuda(), vn.cuda(), done, new)
        out, lse = c.attend(qn.cuda(), done, new)
        kk, vv = (np.concatenate([c.values(x[b][:done[b]]) for b in range(2)]) for x in (k, v))
        want, l, b_out, b_lse = oracle_forward(f64(qn), kk, vv, new, done, True, 0, d ** -0.5, kind)
        within(f64(out), want, b_out, "out")
        within(f64(lse), l, b_lse, "lse")
    back = c.read(kn, done)
    for x, y in zip(back, (k, v)):
        assert np.array_equal(f64(x), np.concatenate([c.values(t) for t in y]))
    assert c.err.item() == 0


def test_decoding_in_a_captured_graph():
    """A step's write and attention, captured once; the lengths move on in
    device memory between replays."""
    import torch
    case = ("bf16", False, 8, 2, 128, 16, [1, 1], [300, 40], True, 0)
    kind, _, h, g, d, page, new, totals, _, _ = case
    c, _, _, _ = _fill(case, spare=40, cols=30)
    free = [p for p in range(c.k.shape[0]) if p not in set(c.table_np.flatten().tolist())]
    for b in range(2):                               # room to grow
        n = -(-totals[b] // page)
        c.table[b, n:n + 2] = c.ints(free[2 * b:2 * b + 2])
    k, v, q = (torch.randn(s, device="cuda").bfloat16() for s in ((2, g, d), (2, g, d), (2, h, d)))
    lengths, s = c.ints(totals), c.ints([0, 1, 2])
    out, lse = torch.empty_like(q), torch.empty((2, h), device="cuda")

    def step():
        c.ep.ep_cache_write(c.c, k, v, c.table, lengths, s)
        c.ep.ep_cache_attention(q, c.c, out, lse, c.table, lengths, s)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        lengths += 1
        for x in (k, v, q):
            x.normal_()
        step()
        want = out.clone(), lse.clone()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
