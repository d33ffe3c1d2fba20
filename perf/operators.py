"""Attention over packed sequences, its gradient, and a paged cache with the
attention that reads it, as measurable cases.

  forward   ``ep_attention`` on a packed batch of sequences
  backward  ``ep_attention_backward``, given the forward pass's results
  store     ``ep_cache_write`` of new tokens, then ``ep_cache_read`` of all
  cached    ``ep_cache_attention``: new tokens' queries over the paged cache

Sequences lie one after another in packed rows; sequence b holds rows
start[b] .. start[b+1] - 1. Query i of a sequence of n queries and m keys
stands at position i + m - n; causal queries see keys up to their position,
with a window w only the last w of these. Queries that see nothing give zeros
and a log-sum of minus infinity. Heads share keys in groups: head h reads key
head h // (heads // kv_heads). A cache with 8-bit values holds e4m3 numbers
with one power-of-two scale per token and key head.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, op, dtype, batch, heads, kv_heads, dim, new, total, ragged, causal=True,
          window=0, fused=False, page=0, store=""):
    """new: queries of the longest sequence (written tokens, for a store);
    total: its keys. fused: q, k and v are slices of one array, as a fused
    projection leaves them. page: tokens of a cache page; store: what it holds."""
    return dict(name=name, op=op, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads,
                dim=dim, new=new, total=total, ragged=ragged, causal=causal, window=window,
                fused=fused, page=page, store=store)


def listed():
    return [
        # one short sequence of a small model, nothing a multiple of anything: latency
        _case("forward tiny", "forward", "fp16", 1, 4, 1, 40, 37, 37, False, fused=True),
        # the training forward pass at a long context, grouped heads
        _case("forward 8k", "forward", "bf16", 2, 32, 8, 128, 8192, 8192, False, fused=True),
        # an encoder over a ragged batch: all keys visible, dim 64
        _case("forward encoder", "forward", "fp16", 24, 16, 16, 64, 1000, 1000, True, causal=False),
        # training steps: the usual one, a ragged one with a sliding window, a small one
        _case("backward 4k", "backward", "bf16", 2, 32, 8, 128, 4096, 4096, False, fused=True),
        _case("backward window", "backward", "fp16", 12, 12, 12, 64, 2047, 2047, True, window=512),
        _case("backward small", "backward", "bf16", 3, 6, 1, 80, 201, 201, True),
        # a prompt's tokens enter an 8-bit cache and are read back (prefix handed on)
        _case("store prompts", "store", "bf16", 4, 8, 8, 128, 4096, 16384, True, page=64,
              store="e4m3"),
        # one token for each of many sequences, 16-bit pages, short rows
        _case("store tokens", "store", "fp16", 48, 2, 2, 96, 1, 777, True, page=16, store="same"),
        # one user's next token: latency
        _case("cached 1 token", "cached", "bf16", 1, 32, 8, 128, 1, 511, False, page=16,
              store="same"),
        # a serving batch's next tokens
        _case("cached 64 users", "cached", "bf16", 64, 32, 8, 128, 1, 16000, True, page=64,
              store="same"),
        # next tokens (with a guess of three more) over long 8-bit caches
        _case("cached long 8-bit", "cached", "bf16", 8, 64, 8, 128, 4, 100000, True, page=256,
              store="e4m3"),
        # a chunk of a prompt that is taken in by pieces
        _case("cached chunk", "cached", "fp16", 4, 32, 4, 128, 1024, 12345, True, page=32,
              store="same"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ranges: 1 to 64 sequences of 1 to 8192 tokens (a
    cache: to 131072), 1 to 64 heads, dims 16 to 128."""
    while True:
        op = rng.choice(["forward", "backward", "store", "cached", "cached"])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
        heads = kv_heads if op == "store" else kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
        dim = rng.choice([64, 128, 128, 8 * rng.randint(2, 16)])
        batch = _log_int(rng, 1, 64)
        c = _case("", op, rng.choice(["bf16", "bf16", "fp16"]), batch, heads, kv_heads, dim, 1, 1,
                  batch > 1 and rng.random() < 0.7)
        del c["name"]
        if op in ("forward", "backward"):
            c["new"] = c["total"] = _log_int(rng, 1, 8192)
            if rng.random() < 0.2:                 # queries and keys of different lengths
                c["total"] = _log_int(rng, 1, 8192)
            else:
                c["fused"] = rng.random() < 0.5
            c["causal"] = rng.random() < 0.75
        else:
            c["total"] = _log_int(rng, 16, 131072)
            c["new"] = min(c["total"], 1 if rng.random() < 0.4 else _log_int(rng, 1, 2048))
            c["page"] = rng.choice([8, 16, 32, 64, 128, 256])
            c["store"] = rng.choice(["same", "e4m3"])
        if op != "store" and c["causal"] and rng.random() < 0.25:
            c["window"] = _log_int(rng, 1, 4096)
        w = work(c)
        area = batch * heads * c["new"] * c["total"]
        rows = batch * c["total"] * kv_heads * dim
        if w["flops"] > 1.0e12 or area > 4.0e9 or rows > 8.5e8 or heads > 64:
            continue
        return c


# ---- lengths: part of the case, not of its data ----


def _lengths(case):
    """(new, total) of each sequence. Of a ragged batch the first is whole,
    the third has no new tokens and, in a packed batch, is empty."""
    rng = random.Random("%(batch)d %(heads)d %(dim)d %(new)d %(total)d" % case)
    new, total = [], []
    for b in range(case["batch"]):
        n, t = case["new"], case["total"]
        if case["ragged"] and b > 0:
            f = rng.uniform(0.1, 1.0)
            if case["op"] in ("store", "cached"):
                t = max(1, int(t * f))
                n = 0 if b == 2 else rng.randint(min(t, (n + 1) // 2), min(n, t))
            elif b == 2:
                n = t = 0
            else:
                n, t = max(1, int(n * f)), max(1, int(t * f))
        new.append(n)
        total.append(t)
    return new, total


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _pairs(case):
    """Visible (query, key) pairs of one head, and rows of keys that some query sees."""
    pairs, seen = 0, 0
    for n, m in zip(*_lengths(case)):
        if n == 0 or m == 0:
            continue
        if not case["causal"]:
            pairs += n * m
            seen += m
            continue
        w = case["window"] or m
        # query i sees the keys max(0, p - w + 1) .. p, p = i + m - n >= 0
        lo, hi = max(0, m - n), m - 1              # positions of the queries that see any
        ramp = max(0, min(hi, w - 1) - lo + 1)     # of these, those that see p + 1 keys
        pairs += ramp * (lo + 1) + ramp * (ramp - 1) // 2 + (hi - lo + 1 - ramp) * w
        seen += hi + 1 - max(0, lo - w + 1)
    return pairs, seen


def work(case):
    new, total = _lengths(case)
    nq, nk = sum(new), sum(total)
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    pairs, seen = _pairs(case)
    row = d + 4 if case["store"] == "e4m3" else 2 * d     # a cached row and its scale
    if case["op"] == "forward":
        return {"bytes": 4.0 * nq * h * d + 4.0 * nk * g * d + 4.0 * nq * h,
                "flops": 4.0 * d * h * pairs}
    if case["op"] == "backward":
        return {"bytes": 8.0 * nq * h * d + 8.0 * nk * g * d + 4.0 * nq * h,
                "flops": 10.0 * d * h * pairs}
    if case["op"] == "store":
        return {"bytes": 2.0 * nq * g * (2 * d + row) + 2.0 * nk * g * (2 * d + row), "flops": 0.0}
    return {"bytes": 4.0 * nq * h * d + 2.0 * seen * g * row, "flops": 4.0 * d * h * pairs}


# ---- inputs ----


def _pow2_scale(x):
    """The smallest power of two that brings a row's largest value within 448,
    the largest e4m3 number (2^9 * 7/8). A power of two divides exactly, so
    a value is rounded once."""
    low = -15 if x.dtype == torch.float16 else -110
    m, e = torch.frexp(x.float().abs().amax(-1))
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp_min(low)
    return torch.where(m == 0, torch.ones_like(m), ((e + 127) << 23).view(torch.float32))


def _quantised(x):
    """(e4m3 values, scales) of rows along the last axis. Values that would
    round to the power of two past the type's largest number stay below it."""
    top = 1.875 * 2.0 ** (15 if x.dtype == torch.float16 else 127)
    x = x.float().clamp(-top, top).to(x.dtype)
    s = _pow2_scale(x)
    return (x.float() / s[..., None]).to(torch.float8_e4m3fn), s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    new, total = _lengths(case)
    nq, nk = sum(new), sum(total)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen).to(dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    u = {"start_q": ints(_starts(new)), "start_k": ints(_starts(total))}
    if case["op"] in ("forward", "backward"):
        if case["fused"]:
            a = normal(nq, h + 2 * g, d)
            u["q"], u["k"], u["v"] = a[:, :h], a[:, h:h + g], a[:, h + g:]
        else:
            u["q"], u["k"], u["v"] = normal(nq, h, d), normal(nk, g, d), normal(nk, g, d)
        if case["op"] == "backward":
            u["dout"] = normal(nq, h, d)
        return u
    ps = case["page"]
    per = [-(-t // ps) for t in total]
    pages = sum(per) + 3                            # some stay free
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros((case["batch"], max(per)), dtype=torch.int32, device="cuda")
    b = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"),
                                torch.tensor(per, device="cuda"))
    at = torch.arange(sum(per), device="cuda") - torch.tensor(_starts(per), device="cuda")[b]
    table[b, at] = order[:sum(per)]
    u["table"], u["lengths"] = table, ints(total)
    for x in ("k", "v"):
        p = normal(pages, ps, g, d)
        u[x + "_scale"] = None
        if case["store"] == "e4m3":
            p, u[x + "_scale"] = _quantised(p)
        u[x + "_pages"] = p
    if case["op"] == "store":
        a = normal(nq, 2 * g, d)
        u["k"], u["v"] = a[:, :g], a[:, g:]
    else:
        u["q"] = normal(nq, h, d)
    return u


def prepare(case, seed):
    u = _inputs(case, seed)
    u["case"] = case
    u["scale"] = 1.0 / math.sqrt(case["dim"])
    u["cached"] = sum(_lengths(case)[1])            # tokens, as a program that reads them back knows
    if case["op"] == "backward":                    # what the forward pass left
        u["out"], u["lse"] = _plain_forward(u)
    return u


# ---- plain forms ----


def _rows(start, n):
    """(sequence, place in it) of each of n packed rows."""
    at = torch.arange(n, device=start.device)
    b = torch.searchsorted(start[1:].long(), at, right=True)
    return b, at - start.long()[b]


def _padded(x, b, at, batch, length):
    out = torch.zeros((batch, length) + x.shape[1:], dtype=torch.float32, device=x.device)
    out[b, at] = x.float()
    return out


def _visible(case, new, total):
    """[batch, queries, keys]: which keys a query sees."""
    i = torch.arange(case["new"], device=new.device)[None, :, None]
    j = torch.arange(case["total"], device=new.device)[None, None, :]
    pos = i + (total - new)[:, None, None]
    vis = (i < new[:, None, None]) & (j < total[:, None, None])
    if case["causal"]:
        vis = vis & (j <= pos)
        if case["window"]:
            vis = vis & (j > pos - case["window"])
    return vis


def _grouped(x, g):
    """[batch, length, heads, dim] as [batch * g, heads / g * length, dim]."""
    b, n, h, d = x.shape
    return x.view(b, n, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(b * g, h // g * n, d)


def _ungrouped(x, b, g, n):
    """The reverse, [batch, length, heads, dim]."""
    return x.view(b, g, -1, n, x.shape[-1]).permute(0, 3, 1, 2, 4).reshape(b, n, -1, x.shape[-1])


def _probabilities(q, k, vis, scale):
    """p [batch * g, rows, keys] and lse [batch * g, rows], float32."""
    b, n, m = vis.shape
    g = k.shape[2]
    s = torch.bmm(_grouped(q, g), _grouped(k, g).transpose(1, 2).contiguous()).mul_(scale)
    s = s.view(b, g, -1, n, m).masked_fill_(~vis[:, None, None], -math.inf).view(b * g, -1, m)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, torch.ones_like(total), total))
    return p, (top + total.log())[..., 0]


def _attend(case, q, k, v, new, total, scale):
    """Padded float32 output and log-sums."""
    vis = _visible(case, new, total)
    b, n, _ = vis.shape
    g = k.shape[2]
    p, lse = _probabilities(q, k, vis, scale)
    out = _ungrouped(torch.bmm(p, _grouped(v, g)), b, g, n)
    return out, _ungrouped(lse[..., None], b, g, n)[..., 0]


def _plain_forward(st):
    case, q = st["case"], st["q"]
    new, total = (st[x].long().diff() for x in ("start_q", "start_k"))
    bq, iq = _rows(st["start_q"], q.shape[0])
    bk, ik = _rows(st["start_k"], st["k"].shape[0])
    n = case["batch"]
    out, lse = _attend(case, _padded(q, bq, iq, n, case["new"]),
                       _padded(st["k"], bk, ik, n, case["total"]),
                       _padded(st["v"], bk, ik, n, case["total"]), new, total, st["scale"])
    return out[bq, iq].to(q.dtype), lse[bq, iq]


def _plain_backward(st):
    case, q = st["case"], st["q"]
    new, total = (st[x].long().diff() for x in ("start_q", "start_k"))
    bq, iq = _rows(st["start_q"], q.shape[0])
    bk, ik = _rows(st["start_k"], st["k"].shape[0])
    b, n, m, g = case["batch"], case["new"], case["total"], case["kv_heads"]
    pq, pg = _padded(q, bq, iq, b, n), _padded(st["dout"], bq, iq, b, n)
    pk, pv = _padded(st["k"], bk, ik, b, m), _padded(st["v"], bk, ik, b, m)
    p, _ = _probabilities(pq, pk, _visible(case, new, total), st["scale"])
    go = _grouped(pg, g)
    dv = torch.bmm(p.transpose(1, 2), go)
    dp = torch.bmm(go, _grouped(pv, g).transpose(1, 2).contiguous())
    ds = dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).mul_(st["scale"])
    dq = torch.bmm(ds, _grouped(pk, g))
    dk = torch.bmm(ds.transpose(1, 2), _grouped(pq, g))
    dq, dk, dv = _ungrouped(dq, b, g, n), _ungrouped(dk, b, g, m), _ungrouped(dv, b, g, m)
    return dq[bq, iq].to(q.dtype), dk[bk, ik].to(q.dtype), dv[bk, ik].to(q.dtype)


def _from_pages(st, x, b, at):
    """Rows of the cache as float32: token at[i] of sequence b[i]."""
    ps = st["case"]["page"]
    page, slot = st["table"][b, at // ps].long(), at % ps
    if st[x + "_scale"] is None:
        return st[x + "_pages"][page, slot].float()
    rows = st[x + "_pages"].view(torch.uint8)[page, slot].view(torch.float8_e4m3fn).float()
    return rows * st[x + "_scale"][page, slot][..., None]


def _plain_store(st):
    case = st["case"]
    ps = case["page"]
    new = st["start_q"].long().diff()
    b, i = _rows(st["start_q"], st["k"].shape[0])
    at = i + (st["lengths"].long() - new)[b]
    page, slot = st["table"][b, at // ps].long(), at % ps
    for x in ("k", "v"):
        if case["store"] == "e4m3":
            rows, st[x + "_scale"][page, slot] = _quantised(st[x])
            st[x + "_pages"].view(torch.uint8)[page, slot] = rows.view(torch.uint8)
        else:
            st[x + "_pages"][page, slot] = st[x]
    total = sum(_lengths(case)[1])
    b, at = _rows(st["start_k"], total)
    return [_from_pages(st, x, b, at).to(DTYPES[case["dtype"]]) for x in ("k", "v")]


def _plain_cached(st):
    case, q = st["case"], st["q"]
    n, m = case["batch"], case["total"]
    new, total = st["start_q"].long().diff(), st["lengths"].long()
    bq, iq = _rows(st["start_q"], q.shape[0])
    bk = torch.arange(n, device=q.device)[:, None].expand(n, m)
    at = torch.arange(m, device=q.device)[None].expand(n, m)
    at = torch.minimum(at, total[:, None] - 1)      # (past the end: masked)
    out, lse = _attend(case, _padded(q, bq, iq, n, case["new"]), _from_pages(st, "k", bk, at),
                       _from_pages(st, "v", bk, at), new, total, st["scale"])
    return out[bq, iq].to(q.dtype), lse[bq, iq]


# ---- the framework's calls ----


def _own_run(st):
    import paper_1806_06144_amd as ep
    case, scale = st["case"], st["scale"]
    mask = dict(scale=scale, causal=case["causal"], window=case["window"])
    if case["op"] == "forward":
        q = st["q"]
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        ep.ep_attention(q, st["k"], st["v"], out, lse, st["start_q"], st["start_k"], **mask)
        return out, lse
    if case["op"] == "backward":
        q, k, v = st["q"], st["k"], st["v"]
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        ep.ep_attention_backward(st["dout"], q, k, v, st["out"], st["lse"], dq, dk, dv,
                                 st["start_q"], st["start_k"], **mask)
        return dq, dk, dv
    cache = ep.EpCache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    if case["op"] == "store":
        ep.ep_cache_write(cache, st["k"], st["v"], st["table"], st["lengths"], st["start_q"])
        total = st["cached"]
        out = [torch.empty((total, case["kv_heads"], case["dim"]), dtype=st["k"].dtype,
                           device="cuda") for _ in range(2)]
        ep.ep_cache_read(cache, out[0], out[1], st["table"], st["lengths"], st["start_k"])
        return out
    q = st["q"]
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    ep.ep_cache_attention(q, cache, out, lse, st["table"], st["lengths"], st["start_q"], **mask)
    return out, lse


def run(st):
    if own:
        return _own_run(st)
    return {"forward": _plain_forward, "backward": _plain_backward, "store": _plain_store,
            "cached": _plain_cached}[st["case"]["op"]](st)


# ---- the definition in 64 bits, one sequence and key head at a time ----


def _exact_head(case, q, k, v, scale):
    """q [n, group, d], k and v [m, d], float64: out and lse."""
    n, m = q.shape[0], k.shape[0]
    pos = torch.arange(n, device=q.device) + (m - n)
    j = torch.arange(m, device=q.device)
    hide = torch.zeros((n, m), dtype=torch.bool, device=q.device)
    if case["causal"]:
        hide |= j[None] > pos[:, None]
        if case["window"]:
            hide |= j[None] <= pos[:, None] - case["window"]
    s = torch.matmul(q.transpose(0, 1), k.T.contiguous()) * scale
    s = s.masked_fill(hide[None], -math.inf)
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = torch.where(lse == -math.inf, torch.zeros_like(s), torch.exp(s - lse))
    return torch.matmul(p, v).transpose(0, 1), lse[..., 0].T


def _e4m3_round64(x):
    """The nearest e4m3 number (ties to even), |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp_min(-6.0)
    step = torch.exp2(e - 3.0)
    return torch.round(x / step) * step


def _exact_stored(x, store):
    """Values that a cache gives back for rows x, float64."""
    half = x.dtype == torch.float16
    x = x.double()
    if store != "e4m3":
        return x
    top = 1.875 * 2.0 ** (15 if half else 127)
    x = x.clamp(-top, top)
    a = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(a.clamp_min(1e-300) / 448.0)) - 1.0
    for _ in range(3):                              # the smallest with a <= 448 2^e
        e = torch.where(a > 448.0 * torch.exp2(e), e + 1.0, e)
    s = torch.where(a == 0, torch.ones_like(a), torch.exp2(e.clamp_min(-15.0 if half else -110.0)))
    return _e4m3_round64(x / s) * s


def exact(case, seed):
    u = _inputs(case, seed)
    scale = 1.0 / math.sqrt(case["dim"])
    new, total = _lengths(case)
    sq, sk = _starts(new), _starts(total)
    h, g = case["heads"], case["kv_heads"]
    r = h // g

    def cached(x, b):
        ps = case["page"]
        t = torch.arange(total[b], device="cuda")
        page = u["table"][b].long()[t // ps]
        if case["store"] != "e4m3":
            return u[x + "_pages"][page, t % ps].double()
        rows = u[x + "_pages"].view(torch.uint8)[page, t % ps].view(torch.float8_e4m3fn)
        return rows.double() * u[x + "_scale"][page, t % ps].double()[..., None]

    if case["op"] == "store":
        got = []
        for x in ("k", "v"):
            fresh = _exact_stored(u[x], case["store"])
            got.append(torch.cat([torch.cat([cached(x, b)[:total[b] - new[b]],
                                             fresh[sq[b]:sq[b + 1]]])
                                  for b in range(case["batch"])]))
        return got
    q = u["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    if case["op"] == "backward":
        dq = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        dk = torch.zeros(u["k"].shape, dtype=torch.float64, device="cuda")
        dv = torch.zeros_like(dk)
    for b in range(case["batch"]):
        if not new[b] or not total[b]:
            continue
        rows, keys = slice(sq[b], sq[b + 1]), slice(sk[b], sk[b + 1])
        if case["op"] == "cached":
            kb, vb = cached("k", b), cached("v", b)
        else:
            kb, vb = u["k"][keys].double(), u["v"][keys].double()
        for c in range(g):
            mine = slice(c * r, c * r + r)
            qh, kh, vh = (x.contiguous() for x in (q[rows, mine], kb[:, c], vb[:, c]))
            if case["op"] != "backward":
                out[rows, mine], lse[rows, mine] = _exact_head(case, qh, kh, vh, scale)
                continue
            with torch.enable_grad():               # by differentiation, not by the formula
                leaves = [x.requires_grad_() for x in (qh, kh, vh)]
                o, _ = _exact_head(case, *leaves, scale)
                grads = torch.autograd.grad(o, leaves, u["dout"][rows, mine].double())
            dq[rows, mine], dk[keys, c], dv[keys, c] = grads
    return (dq, dk, dv) if case["op"] == "backward" else (out, lse)
