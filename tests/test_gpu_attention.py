"""ep_attention and ep_attention_backward against the float64 oracle, element
by element within bounds derived from the roundings made (oracle/attention.py),
over types, head layouts, lengths, strides and masks; what lies behind the
sequences; streams and captured graphs."""

import numpy as np
import pytest

from attention_common import (f64, oracle_backward, oracle_forward, rounded, starts, within)

pytestmark = pytest.mark.gpu

# kind, heads, kv_heads, dim, query lengths, key lengths, causal, window
CASES = [
    ("bf16", 1, 1, 128, [1], [1], True, 0),
    ("fp16", 2, 1, 64, [1], [300], True, 0),
    ("bf16", 4, 4, 64, [64, 128], [64, 128], True, 0),
    ("bf16", 4, 2, 128, [129], [129], True, 0),
    ("fp16", 6, 2, 128, [65, 0, 33, 1], [65, 0, 33, 1], True, 0),      # an empty sequence
    ("bf16", 3, 3, 8, [70], [70], True, 0),
    ("fp16", 4, 1, 40, [37], [37], True, 0),
    ("bf16", 5, 1, 80, [100, 41], [100, 41], False, 0),
    ("bf16", 8, 2, 72, [31], [200], True, 0),                          # more keys than queries
    ("fp16", 4, 2, 128, [200], [31], True, 0),                         # rows that see nothing
    ("bf16", 2, 2, 64, [90], [20], False, 0),
    ("bf16", 4, 2, 64, [50, 7, 20], [0, 9, 0], True, 0),               # no keys at all
    ("bf16", 4, 2, 64, [0, 7], [50, 0], False, 0),
    ("fp16", 4, 4, 128, [300], [300], True, 1),                        # itself only
    ("bf16", 4, 2, 128, [300], [300], True, 64),
    ("fp16", 7, 1, 64, [150, 260], [150, 260], True, 100),
    ("bf16", 2, 1, 64, [40], [500], True, 33),
    ("bf16", 2, 1, 64, [500], [40], True, 33),
    ("bf16", 12, 4, 112, [130, 2, 63, 64, 65], [130, 2, 63, 64, 65], True, 0),
    ("fp16", 64, 2, 64, [9, 33], [9, 33], True, 0),                    # a group of 32
    ("bf16", 100, 1, 16, [11], [77], True, 0),                         # 100 heads to one key head
    ("bf16", 2, 2, 128, [700], [700], True, 0),
    ("fp16", 2, 2, 128, [513], [1030], False, 0),
    ("bf16", 2, 1, 96, [3] * 70, [5] * 70, True, 0),                   # more than 64 sequences
]


def _make(case, seed=0, size=1.0):
    kind, h, g, d, nq, nk, causal, window = case
    rng = np.random.default_rng(seed + len(nq) + d)
    q = rounded(rng, (sum(nq), h, d), kind, size)
    k, v = (rounded(rng, (sum(nk), g, d), kind) for _ in range(2))
    return q, k, v, rounded(rng, q.shape, kind)


def _forward(q, k, v, nq, nk, scale=None, causal=True, window=0, stream=None, out=None, lse=None):
    import torch
    import paper_1806_06144_amd as ep
    sq, sk = (torch.from_numpy(starts(x)).cuda() for x in (nq, nk))
    if out is None:
        out = torch.full(tuple(q.shape), float("nan"), dtype=q.dtype, device="cuda")
    if lse is None:
        lse = torch.full(tuple(q.shape[:2]), float("nan"), device="cuda")
    ep.ep_attention(q, k, v, out, lse, sq, sk, scale, causal, window, stream)
    return out, lse


def _backward(g, q, k, v, out, lse, nq, nk, scale=None, causal=True, window=0, stream=None,
              into=None):
    import torch
    import paper_1806_06144_amd as ep
    sq, sk = (torch.from_numpy(starts(x)).cuda() for x in (nq, nk))
    grads = into or [torch.full(tuple(x.shape), float("nan"), dtype=x.dtype, device="cuda")
                     for x in (q, k, v)]
    ep.ep_attention_backward(g, q, k, v, out, lse, *grads, sq, sk, scale, causal, window, stream)
    return grads


def _check_forward(got, case, q, k, v, scale):
    kind, _, _, _, nq, nk, causal, window = case
    out, lse, b_out, b_lse = oracle_forward(f64(q), f64(k), f64(v), nq, nk, causal, window, scale,
                                            kind)
    within(f64(got[0]), out, b_out, "out")
    within(f64(got[1]), lse, b_lse, "lse")
    return out, lse


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}.{c[2]}x{c[3]}-{c[4][:3]}-{c[5][:3]}-{c[6]}-{c[7]}")
def test_forward(case):
    q, k, v, _ = _make(case)
    scale = float(np.float32(case[3] ** -0.5))
    got = _forward(q.cuda(), k.cuda(), v.cuda(), case[4], case[5], scale, case[6], case[7])
    _check_forward(got, case, q, k, v, scale)


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}.{c[2]}x{c[3]}-{c[4][:3]}-{c[5][:3]}-{c[6]}-{c[7]}")
def test_backward(case):
    import torch
    kind, _, _, _, nq, nk, causal, window = case
    q, k, v, g = _make(case, 5)
    scale = float(np.float32(case[3] ** -0.5))
    out, lse, _, _ = oracle_forward(f64(q), f64(k), f64(v), nq, nk, causal, window, scale, kind)
    grads = _backward(g.cuda(), q.cuda(), k.cuda(), v.cuda(),
                      torch.from_numpy(out).to(q.dtype).cuda(), torch.from_numpy(lse).float().cuda(),
                      nq, nk, scale, causal, window)
    want, bound = oracle_backward(f64(q), f64(k), f64(v), f64(g), out, nq, nk, causal, window,
                                  scale, kind)
    for x, w, b, name in zip(grads, want, bound, ("dq", "dk", "dv")):
        within(f64(x), w, b, name)


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_small_and_large_scores(size):
    """Scores near 0, and of several hundred: a softmax that one key takes."""
    case = ("bf16", 2, 1, 64, [150], [150], True, 0)
    q, k, v, _ = _make(case, 2, size)
    got = _forward(q.cuda(), k.cuda(), v.cuda(), [150], [150], 0.25)
    _check_forward(got, case, q, k, v, 0.25)


def test_scores_that_grow_with_every_tile():
    """The running maximum rises all along the keys, and falls."""
    import torch
    case = ("bf16", 1, 1, 64, [128], [640], False, 0)
    for order in (1, -1):
        q, k, v, _ = _make(case, 3)
        ramp = torch.linspace(0.1, 3.0, 640)[::1]
        k = (torch.ones_like(k) * (ramp if order > 0 else ramp.flip(0))[:, None, None]).to(k.dtype)
        q = torch.ones_like(q)
        got = _forward(q.cuda(), k.cuda(), v.cuda(), [128], [640], 1.0, False)
        _check_forward(got, case, q, k, v, 1.0)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_strided_slices_and_rows_behind_the_last_sequence(kind):
    """q, k, v and the gradients as slices of wider arrays; rows that belong
    to no sequence hold NaN, are not read into any result and stay as they are."""
    import torch
    h, g, d, nq = 6, 2, 64, [70, 33]
    extra = 40
    rng = np.random.default_rng(4)
    t = sum(nq)
    wide = rounded(rng, (t + extra, h + 2 * g + 1, d + 16), kind)
    wide[t:] = float("nan")
    wide = wide.cuda()
    q, k, v = (wide[:, a:b, 8:8 + d] for a, b in ((0, h), (h, h + g), (h + g, h + 2 * g)))
    out = torch.full((t + extra, h, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((t + extra, h), 7.0, device="cuda")
    scale = 0.125
    _forward(q, k, v, nq, nq, scale, out=out, lse=lse)
    assert (out[t:] == 7).all() and (lse[t:] == 7).all()
    case = (kind, h, g, d, nq, nq, True, 0)
    o64, l64 = _check_forward((out[:t], lse[:t]), case, q[:t], k[:t], v[:t], scale)
    go = rounded(rng, (t + extra, h, d), kind)
    go[t:] = float("nan")
    grads = torch.full((t + extra, h + 2 * g, d + 8), 7.0, dtype=q.dtype, device="cuda")
    into = [grads[:, a:b, :d] for a, b in ((0, h), (h, h + g), (h + g, h + 2 * g))]
    _backward(go.cuda(), q, k, v, out, lse, nq, nq, scale, into=into)
    assert (grads[t:] == 7).all() and (grads[:, :, d:] == 7).all()
    # (out as the kernel gave it: exact up to a rounding, as the bound assumes, and the
    # forward pass's own error on top)
    want, bound = oracle_backward(f64(q[:t]), f64(k[:t]), f64(v[:t]), f64(go[:t]),
                                  np.abs(f64(out[:t])) + np.abs(o64), nq, nq, True, 0, scale, kind)
    for x, w, b, name in zip(into, want, bound, ("dq", "dk", "dv")):
        within(f64(x[:t]), w, b, name)


def test_garbage_in_the_padding_of_starts():
    """start values outside the arrays are taken as the nearest inside."""
    import torch
    import paper_1806_06144_amd as ep
    case = ("bf16", 2, 2, 64, [50, 50], [50, 50], True, 0)
    q, k, v, _ = _make(case)
    out = torch.zeros_like(q).cuda()
    s = torch.tensor([-5, 50, 1 << 30], dtype=torch.int32, device="cuda")
    ep.ep_attention(q.cuda(), k.cuda(), v.cuda(), out, None, s, s)
    want, _ = _forward(q.cuda(), k.cuda(), v.cuda(), [50, 50], [50, 50])
    assert torch.equal(out, want)


def test_results_repeat_bit_by_bit_on_any_stream():
    import torch
    case = ("bf16", 8, 2, 128, [300, 77], [300, 77], True, 0)
    q, k, v, g = (x.cuda() for x in _make(case))
    nq = case[4]
    out, lse = _forward(q, k, v, nq, nq)
    grads = _backward(g, q, k, v, out, lse, nq, nq)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        out2, lse2 = _forward(q, k, v, nq, nq, stream=stream)
        grads2 = _backward(g, q, k, v, out2, lse2, nq, nq, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        assert all(torch.equal(a, b) for a, b in zip(grads, grads2))


def _captured_step(i, h, g, d, n):
    """A forward and backward pass, and the graph that holds it."""
    import torch
    import paper_1806_06144_amd as ep
    q, k, v, go = (x.cuda() for x in _make(("bf16", h, g, d, [n], [n], True, 0), i))
    s = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((n, h), device="cuda")
    grads = [torch.empty_like(x) for x in (q, k, v)]

    def step():
        ep.ep_attention(q, k, v, out, lse, s, s)
        ep.ep_attention_backward(go, q, k, v, out, lse, *grads, s, s)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    return graph, (step, (q, k, v, go), (out, lse, *grads))


def test_two_captured_graphs_replayed_in_turn():
    import torch
    made = [_captured_step(0, 4, 2, 64, 130), _captured_step(1, 8, 1, 128, 90)]
    graphs, state = [x[0] for x in made], [x[1] for x in made]
    for turn in range(4):
        for graph, (step, ins, outs) in zip(graphs, state):
            for x in ins:
                x.normal_()
            step()
            want = [x.clone() for x in outs]
            for x in outs:
                x.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


def test_gradients_match_differences():
    """The whole path against differences of the float64 forward pass along
    random directions: the tolerance is the bound of each gradient, summed over
    the direction's elements, and the difference's own error (step^2)."""
    import torch
    case = ("fp16", 4, 2, 64, [40, 9], [40, 9], True, 0)
    kind, h, g, d, nq, nk, causal, window = case
    q, k, v, go = _make(case, 9)
    scale = 0.125
    out, lse = _forward(q.cuda(), k.cuda(), v.cuda(), nq, nk, scale)
    grads = _backward(go.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, nq, nk, scale)
    args = [f64(x) for x in (q, k, v)]
    o64 = oracle_forward(*args, nq, nk, causal, window, scale, kind)[0]
    _, bound = oracle_backward(*args, f64(go), np.abs(f64(out)) + np.abs(o64), nq, nk, causal,
                               window, scale, kind)
    rng = np.random.default_rng(0)
    step = 1e-4

    def loss(x):
        return (oracle_forward(*x, nq, nk, causal, window, scale, kind)[0] * f64(go)).sum()
    for i, (x, b) in enumerate(zip(grads, bound)):
        way = rng.standard_normal(x.shape)
        up, down = list(args), list(args)
        up[i] = args[i] + step * way
        down[i] = args[i] - step * way
        want = (loss(up) - loss(down)) / (2 * step)
        room = (b * np.abs(way)).sum() + 1e-4
        assert abs((f64(x) * way).sum() - want) <= room


def test_binding_refusals():
    import torch
    import paper_1806_06144_amd as ep
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ep.ep_attention(q, q[:, :, :32], q, q.clone(), None, s, s)
    with pytest.raises(TypeError):
        ep.ep_attention(q, q.half(), q, q.clone(), None, s, s)
    with pytest.raises(TypeError):
        ep.ep_attention(q.float(), q, q, q.clone(), None, s, s)
    with pytest.raises(ValueError):
        ep.ep_attention(q, q.cpu(), q, q.clone(), None, s, s)
    with pytest.raises(TypeError):
        ep.ep_attention(q, q, q, q.clone(), None, s.long(), s)
    with pytest.raises(ValueError):
        ep.ep_attention(q, q, q, q.clone(), None, s, torch.zeros(5, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        ep.ep_attention(q, q, q, q.transpose(1, 2).contiguous().transpose(1, 2), None, s, s)
    with pytest.raises(ep.EigenProError) as e:       # 10 elements from the start: 20 bytes
        ep.ep_attention(torch.zeros(600, dtype=q.dtype, device="cuda")[10:522].view(4, 2, 64), q, q,
                        q.clone(), None, s, s)
    assert e.value.code == ep.EP_EINVAL
    with pytest.raises(ep.EigenProError):
        ep.ep_attention(q, q, q, q.clone(), None, s, s, causal=False, window=3)


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 64), ("bf16", 40)])
@pytest.mark.parametrize("lengths,window", [([1] * 20, 0), ([130, 7], 1)])
def test_a_query_of_one_key_has_no_gradient_to_either(kind, dim, lengths, window):
    """Its probability is 1 whatever q and k are: dq and dk are zero, exactly."""
    case = (kind, 6, 2, dim, lengths, lengths, True, window)
    q, k, v, g = (x.cuda() for x in _make(case, 3, 4.0))
    out, lse = _forward(q, k, v, lengths, lengths, window=window)
    dq, dk, dv = _backward(g, q, k, v, out, lse, lengths, lengths, window=window)
    assert (dq == 0).all() and (dk == 0).all()
    assert (out.view(-1, 2, 3, dim) == v[:, :, None]).all()


def test_thousands_of_sequences():
    """The search for a tile's sequence goes through several levels."""
    import torch
    rng = np.random.default_rng(1)
    lengths = rng.integers(0, 4, 9000)
    q, k, v = (torch.randn((lengths.sum(), 2, 16), device="cuda").half() for _ in range(3))
    out, lse = _forward(q, k, v, lengths, lengths, 0.25)
    # sequences 0 .. 3 long: row i of a sequence against the rows before it
    s = torch.from_numpy(starts(lengths)).long()
    b = torch.repeat_interleave(torch.arange(9000), torch.from_numpy(lengths))
    first = s[b].cuda()
    at = torch.arange(q.shape[0], device="cuda")
    x = torch.full((q.shape[0], 2, 3), -float("inf"), dtype=torch.float64, device="cuda")
    vals = torch.zeros((q.shape[0], 2, 3, 16), dtype=torch.float64, device="cuda")
    for j in range(3):
        ok = first + j <= at
        row = (first + j).clamp(max=q.shape[0] - 1)
        x[:, :, j] = torch.where(ok[:, None], 0.25 * (q.double() * k[row].double()).sum(-1), x[:, :, j])
        vals[:, :, j] = v[row].double()
    want = (x.softmax(-1)[..., None] * vals).sum(2)
    # (one rounding of the result and one of each probability, 2^-11 of sums of |v| < 16)
    assert (out.double() - want).abs().max() < 3 * 2.0 ** -11 * 6
    assert (lse.double() - x.logsumexp(-1)).abs().max() < 1e-5


@pytest.mark.parametrize("case", [("bf16", 2, 1, 64, [1], [6000], False, 0),
                                  ("fp16", 2, 2, 128, [3, 40], [2000, 2100], True, 0),
                                  ("bf16", 4, 1, 128, [2000], [30], False, 0),
                                  ("bf16", 2, 1, 72, [5, 700], [4000, 700], True, 0)],
                         ids=lambda c: f"{c[0]}-{c[4]}-{c[5]}")
def test_gradients_of_few_rows_or_few_keys(case):
    """Keys or rows cut over workgroups, their partial sums added."""
    test_forward(case)
    test_backward(case)


def test_gradients_without_queries_or_keys():
    import torch
    q, k = torch.zeros((0, 2, 64), dtype=torch.float16), torch.zeros((5, 2, 64), dtype=torch.float16)
    for nq, nk in (([0], [5]), ([5], [0])):
        a, b = (torch.ones((n, 2, 64), dtype=torch.float16, device="cuda") for n in (nq[0], nk[0]))
        out, lse = _forward(a, b, b, nq, nk)
        grads = _backward(a, a, b, b, out, lse, nq, nk)
        assert all((x == 0).all() for x in (out, *grads)) and (lse == -float("inf")).all()


def test_keys_shared_by_stride():
    """An input may be one head expanded over all (stride 0)."""
    import torch
    case = ("bf16", 6, 3, 64, [70], [70], True, 0)
    q, k, v, _ = _make(case)
    k, v = (x[:, :1].expand(-1, 3, -1) for x in (k, v))
    ke, ve = (x.cuda()[:, :1].expand(-1, 3, -1) for x in (k, v))
    got = _forward(q.cuda(), ke, ve, [70], [70], 0.125)
    assert ke.stride(1) == 0
    _check_forward(got, case, q, k, v, 0.125)


def test_offsets_past_32_bits():
    """Rows 16 MB apart: 300 of them span 5 GB, in every array of the calls."""
    import torch
    n, h, g, d = 300, 4, 2, 64
    case = ("bf16", h, g, d, [n], [n], True, 0)
    q, k, v, go = _make(case, 11)
    wide = torch.empty((n, 1 << 23), dtype=torch.bfloat16, device="cuda")
    views, at = [], 0
    for heads in (h, g, g, h, h, h, g, g):           # q, k, v, dout, out, dq, dk, dv
        views.append(wide[:, at:at + heads * d].view(n, heads, d))
        at += heads * d
    for x, y in zip(views, (q, k, v, go)):
        x.copy_(y)
    qw, kw, vw, gw, ow, *grads = views
    scale = 0.125
    out, lse = _forward(qw, kw, vw, [n], [n], scale, out=ow)
    o64, _ = _check_forward((out, lse), case, q, k, v, scale)
    _backward(gw, qw, kw, vw, out, lse, [n], [n], scale, into=grads)
    want, bound = oracle_backward(f64(q), f64(k), f64(v), f64(go), np.abs(f64(out)) + np.abs(o64),
                                  [n], [n], True, 0, scale, "bf16")
    for x, w, b, name in zip(grads, want, bound, ("dq", "dk", "dv")):
        within(f64(x), w, b, name)


def test_calls_at_once_on_two_streams():
    """Calls with work memory on two streams, not waiting for each other."""
    import torch
    problems = []
    for i, (nq, nk) in enumerate((([400, 30], [400, 30]), ([6], [3000]))):
        case = ("bf16", 8, 2, 128, nq, nk, True, 0)
        q, k, v, g = (x.cuda() for x in _make(case, i))
        out, lse = _forward(q, k, v, nq, nk)
        grads = _backward(g, q, k, v, out, lse, nq, nk)
        problems.append((q, k, v, g, nq, nk, [out, lse, *grads]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    got = [[], []]
    for _ in range(5):
        for i, (s, (q, k, v, g, nq, nk, _)) in enumerate(zip(streams, problems)):
            with torch.cuda.stream(s):
                out, lse = _forward(q, k, v, nq, nk)
                got[i].append([out, lse, *_backward(g, q, k, v, out, lse, nq, nk)])
    torch.cuda.synchronize()
    for i, p in enumerate(problems):
        assert all(torch.equal(a, b) for run in got[i] for a, b in zip(run, p[-1]))


def test_a_padded_batch():
    """Each sequence's padding is a sequence of its own; it holds NaN, which
    reaches no row of the sequences, nor their gradients."""
    import torch
    h, g, d, length, lengths = 4, 2, 64, 100, [100, 37, 0, 64]
    case = ("bf16", h, g, d, lengths, lengths, True, 0)
    q, k, v, go = _make(case, 4)
    parts = [x for n in lengths for x in (n, length - n)]
    keep = torch.cat([torch.arange(length) < n for n in lengths]).cuda()

    def padded(x):
        y = torch.full((len(lengths) * length,) + tuple(x.shape[1:]), float("nan"), dtype=x.dtype,
                       device="cuda")
        y[keep] = x.cuda()
        return y
    qp, kp, vp, gp = (padded(x) for x in (q, k, v, go))
    out, lse = _forward(qp, kp, vp, parts, parts, 0.125)
    o64, _ = _check_forward((out[keep], lse[keep]), case, q, k, v, 0.125)
    grads = _backward(gp, qp, kp, vp, out, lse, parts, parts, 0.125)
    want, bound = oracle_backward(f64(q), f64(k), f64(v), f64(go), np.abs(f64(out[keep])) + np.abs(o64),
                                  lengths, lengths, True, 0, 0.125, "bf16")
    for x, w, b, name in zip(grads, want, bound, ("dq", "dk", "dv")):
        within(f64(x[keep]), w, b, name)


def test_a_long_sequence():
    """100000 tokens: some rows, and the gradients of some rows and of the last
    keys, which few rows see."""
    import torch
    import oracle.attention as oa
    n, h, d, scale, kind = 100000, 2, 64, 0.125, "bf16"
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, go = (torch.randn((n, h, d), device="cuda", generator=gen).bfloat16() for _ in range(2))
    k, v = (torch.randn((n, 1, d), device="cuda", generator=gen).bfloat16() for _ in range(2))
    out, lse = _forward(q, k, v, [n], [n], scale)
    dq, dk, dv = _backward(go, q, k, v, out, lse, [n], [n], scale)
    q64, g64, k64, v64 = f64(q), f64(go), f64(k)[:, 0], f64(v)[:, 0]
    rng = np.random.default_rng(0)
    tail = n - 40
    for i in [0, 1, 63, 64, n - 1, *rng.integers(100, n, 8)]:
        for j in range(h):
            args = q64[i:i + 1, j], k64[:i + 1], v64[:i + 1]
            o, l = oa.head_forward(*args, True, 0, scale)
            within(f64(out[i, j])[None], o, oa.forward_bound(*args, True, 0, scale, kind), "out")
            within(f64(lse[i:i + 1, j]), l, oa.lse_bound(args[0], args[1], l, scale), "lse")
            g = oa.head_backward(*args, g64[i:i + 1, j], True, 0, scale)[0]
            b = oa.backward_bound(*args, g64[i:i + 1, j], np.abs(o) + np.abs(f64(out[i, j])), True, 0,
                                  scale, kind)[0]
            within(f64(dq[i, j])[None], g, b, "dq")
    want, bound = np.zeros((2, 40, d)), np.zeros((2, 40, d))
    for j in range(h):                               # rows tail .. n - 1 over all keys
        args = q64[tail:, j], k64, v64, g64[tail:, j]
        o = oa.head_forward(*args[:3], True, 0, scale)[0]
        _, a, b = oa.head_backward(*args, True, 0, scale)
        _, ea, eb = oa.backward_bound(*args, np.abs(o) + np.abs(f64(out[tail:, j])), True, 0, scale, kind)
        want += [a[tail:], b[tail:]]
        bound += [ea[tail:], eb[tail:]]
    u = oa.U[kind]
    for x, w, e, name in zip((dk, dv), want, bound, ("dk", "dv")):
        within(f64(x[tail:, 0]), w, e * (1 + u) + u * np.abs(w), name)
