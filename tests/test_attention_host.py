"""Attention without a GPU: the oracle's gradients against differences, its
8-bit rounding against all codes, the kernels' index arithmetic on the host
(bad starts, lengths and page numbers among it), and refusals."""

import ctypes
import os
import subprocess

import numpy as np
import pytest

import oracle.attention as oa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1806_06144_amd", "csrc")


@pytest.mark.parametrize("n,m,causal,window", [(5, 5, True, 0), (3, 7, True, 0), (7, 3, True, 0),
                                               (6, 6, True, 2), (4, 6, False, 0), (1, 1, True, 1)])
def test_oracle_gradients_match_differences(n, m, causal, window):
    rng = np.random.default_rng(n * 10 + m)
    q, k, v, g = (rng.standard_normal(s) for s in ((n, 8), (m, 8), (m, 8), (n, 8)))

    def loss(q, k, v):
        return (oa.head_forward(q, k, v, causal, window, 0.3)[0] * g).sum()
    grads = oa.head_backward(q, k, v, g, causal, window, 0.3)
    step = 1e-5           # central differences: error of the order step^2, rounding 1e-16 / step
    for i, (x, got) in enumerate(zip((q, k, v), grads)):
        for at in np.ndindex(x.shape):
            a, b = x.copy(), x.copy()
            a[at] += step
            b[at] -= step
            args = [q, k, v]
            args[i] = a
            up = loss(*args)
            args[i] = b
            assert abs((up - loss(*args)) / (2 * step) - got[at]) < 1e-8


def test_oracle_empty_rows():
    q, k, v = np.ones((4, 8)), np.ones((2, 8)), np.ones((2, 8))
    out, lse = oa.head_forward(q, k, v, True, 0, 1.0)
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all()
    assert (out[2:] == 1).all() and lse[2] == 8.0
    out, lse = oa.head_forward(q, k[:0], v[:0], False, 0, 1.0)
    assert (out == 0).all() and (lse == -np.inf).all()


def test_oracle_e4m3_rounding_matches_torch():
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = np.unique(codes[np.isfinite(codes)])
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 1e9), np.nextafter(mid, -1e9)])
    # (through float32, which torch converts from; the midpoints are exact in it)
    x = x.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oa.e4m3_round(x), want)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_oracle_scales(kind):
    big = 65504.0 if kind == "fp16" else float.fromhex("0x1.fep127")
    for most in (448.0, 448.5, 1.0, 0.875, 0.9, big, 6e-8, 1e-3):
        got, s = oa.stored(np.array([[most, -most / 3]]), kind)
        top = 1.875 * 2.0 ** (15 if kind == "fp16" else 127)
        low = 2.0 ** (-15 if kind == "fp16" else -110)
        assert min(most, top) <= 448 * s[0] and (s[0] == low or min(most, top) > 224 * s[0])
        assert abs(got[0, 0]) <= top


PROGRAM = r"""
#include "attn_index.h"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace ep;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
    // token of a row: every row below the documented bound, at its edges
    for (int group = 1; group <= 1024; ++group) {
        const unsigned magic = group_magic(group);
        const int64_t rows = ((int64_t(1) << 32) - 1) / group;      // r group < 2^32
        const int64_t top = rows < 0x7fffffff ? rows : 0x7fffffff;
        for (int64_t r = 0; r < 5000 && r <= top; ++r) CHECK(row_token((int)r, group, magic) == r / group);
        for (int64_t r = top; r > top - 5000 && r >= 0; --r) CHECK(row_token((int)r, group, magic) == r / group);
    }
    // starts and lengths of any value give ranges inside
    const int odd[] = {-2147483647 - 1, -5, 0, 1, 99, 100, 101, 2147483647};
    for (int a : odd) for (int b : odd) {
        int first, count;
        held_range(a, b, 100, first, count);
        CHECK(first >= 0 && count >= 0 && first + count <= 100);
        if (a >= 0 && b >= a && b <= 100) CHECK(first == a && count == b - a);
    }
    for (int l : odd) {
        const int m = held_length(l, 7, 4);
        CHECK(m >= 0 && m <= 112 && (l < 0 || l > 112 || m == l));
    }
    // tiles: every row of every sequence lies in a tile of its own sequence
    unsigned seed = 1;
    auto next = [&](unsigned n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; };
    for (int trial = 0; trial < 2000; ++trial) {
        const int batch = 1 + next(9), per = 1 + next(5), size = 32 << next(3);
        std::vector<int> start(batch + 1, 0);
        for (int b = 0; b < batch; ++b) start[b + 1] = start[b] + next(3) * next(300);
        const int tokens = start[batch] + next(50);
        const int64_t tiles = (int64_t)tokens * per / size + batch;
        for (int b = 0; b < batch; ++b) {
            const int64_t need = ((int64_t)(start[b + 1] - start[b]) * per + size - 1) / size;
            const int64_t f = first_tile(start[b], tokens, b, per, size);
            const int64_t g = b + 1 < batch ? first_tile(start[b + 1], tokens, b + 1, per, size) : tiles;
            CHECK(f + need <= g && g <= tiles);
        }
    }
    // pages: only numbers of the cache, only inside the table
    const int table[8] = {3, -1, 8, 2147483647, 7, 0, -2147483647 - 1, 5};
    for (int shift = 0; shift <= 4; ++shift)
        for (int j = 0; j < 4 << shift; ++j)
            for (int b = 0; b < 2; ++b) {
                const int want = table[4 * b + (j >> shift)], page = page_of(table, 4, b, 8, shift, j);
                CHECK(page == (want >= 0 && want < 8 ? want : -1));
                if (page >= 0) CHECK(page_slot(page, shift, j) == ((int64_t)page << shift) + j % (1 << shift));
            }
    CHECK(page_slot(2000000000, 8, 255) == 2000000000LL * 256 + 255);
    // masks: the two sides agree, at every pair
    for (int n = 0; n < 9; ++n) for (int m = 0; m < 9; ++m) for (int causal = 0; causal < 2; ++causal)
        for (int window = 0; window <= (causal ? 9 : 0); ++window) for (int group = 1; group < 4; ++group)
            for (int t = 0; t < n; ++t) for (int j = 0; j < m; ++j) {
                const int p = t + m - n;
                const bool sees = !causal || (j <= p && (!window || j > p - window));
                CHECK(sees == (j >= visible_lo(t, m - n, window) && j < visible_hi(t, m - n, m, causal)));
                for (int r = t * group; r < (t + 1) * group; ++r)
                    CHECK(sees == (r >= seen_from(j, m - n, n, group, causal) &&
                                   r < seen_to(j, m - n, n, group, window)));
            }
    std::printf("ok\n");
    return 0;
}
"""


def test_index_arithmetic(tmp_path):
    src, exe = tmp_path / "i.cpp", tmp_path / "i"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.stdout == "ok\n", r.stdout + r.stderr


# ---- refusals: before any device work, so addresses are only numbers ----

import paper_1806_06144_amd as ep  # noqa: E402

A = 4096                                            # an aligned address, never read


def _attn(**kw):
    d = dict(type=ep.EP_BF16, causal=1, batch=2, heads=8, kv_heads=2, dim=64, tokens_q=100,
             tokens_k=100, window=0, start_q=A, start_k=A, scale=0.1)
    d.update(kw)
    return ep.EpAttn(**d)


def _rows(data=A, row=512, head=64):
    return ep.EpRows(data, row, head)


def _forward(a, **kw):
    r = {n: _rows() for n in ("q", "k", "v", "out")}
    r.update(kw)
    return ep.raw_call("ep_attention", None if a is None else ctypes.byref(a), r["q"], r["k"],
                       r["v"], r["out"], A, A, 1 << 30, None)


BAD = [dict(type=2), dict(type=-1), dict(causal=2), dict(batch=0), dict(batch=1 << 24),
       dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(heads=4096, kv_heads=2), dict(dim=0),
       dict(dim=4), dict(dim=60), dict(dim=136), dict(dim=256), dict(tokens_q=-1),
       dict(tokens_q=1 << 30), dict(tokens_k=-1), dict(tokens_k=1 << 30), dict(window=-1),
       dict(window=1 << 30), dict(window=5, causal=0), dict(start_q=None), dict(start_k=None),
       dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
       dict(heads=2048, kv_heads=2, tokens_q=5000), dict(heads=65534, kv_heads=65534, tokens_q=1 << 20),
       dict(heads=65534, kv_heads=65534, batch=1 << 10)]


@pytest.mark.parametrize("kw", BAD)
def test_attention_refuses(kw):
    a = _attn(**kw)
    assert _forward(a) == ep.EP_EINVAL
    assert ep.ep_last_error() != ""
    assert ep.raw_call("ep_attention_backward_bytes", ctypes.byref(a)) == ep.EP_EINVAL


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
@pytest.mark.parametrize("bad", [dict(data=None), dict(data=A + 2), dict(data=A + 8),
                                 dict(row=100), dict(head=4), dict(row=-8),
                                 dict(head=-64), dict(row=1 << 24)])
def test_attention_refuses_rows(name, bad):
    assert _forward(_attn(), **{name: _rows(**bad)}) == ep.EP_EINVAL
    assert name in ep.ep_last_error()


def test_outputs_that_overlap_themselves():
    for bad in (dict(row=0), dict(row=56), dict(head=0), dict(head=8)):
        assert _forward(_attn(), out=_rows(**bad)) == ep.EP_EINVAL
        for name in ("dq", "dk", "dv"):
            assert _backward(_attn(), **{name: _rows(**bad)}) == ep.EP_EINVAL
        assert ep.raw_call("ep_cache_read", ctypes.byref(_cache()), ctypes.byref(_table()),
                           ep.EP_BF16, _rows(**bad), _rows(), 10, A, None) == ep.EP_EINVAL


def test_attention_null():
    assert _forward(None) == ep.EP_EINVAL


def test_no_queries_is_no_work():
    assert _forward(_attn(tokens_q=0), q=_rows(None), out=_rows(None)) == ep.EP_OK


def _backward(a, work=A, work_bytes=1 << 20, lse=A, **kw):
    names = ("dout", "q", "k", "v", "out", "dq", "dk", "dv")
    r = {n: kw.get(n, _rows()) for n in names}
    return ep.raw_call("ep_attention_backward", ctypes.byref(a), r["dout"], r["q"], r["k"], r["v"],
                       r["out"], lse, r["dq"], r["dk"], r["dv"], work, work_bytes, None)


@pytest.mark.parametrize("kw", [dict(lse=None), dict(work=None), dict(work=A + 4),
                                dict(work_bytes=8)] +
                         [{n: _rows(data=None)} for n in ("dout", "q", "k", "v", "out", "dq", "dk",
                                                          "dv")] +
                         [{n: _rows(row=12)} for n in ("dout", "dq", "dk", "dv")])
def test_backward_refuses(kw):
    assert _backward(_attn(), **kw) == ep.EP_EINVAL


def _cache(**kw):
    d = dict(type=ep.EP_BF16, pages=10, page_size=16, kv_heads=2, dim=64, k=A, v=A, k_scale=A,
             v_scale=A)
    d.update(kw)
    return ep.EpCacheDesc(**d)


def _table(**kw):
    d = dict(batch=2, table=A, cols=5, lengths=A, err=None)
    d.update(kw)
    return ep.EpPages(**d)


BAD_CACHE = [(dict(type=3), {}), (dict(type=ep.EP_FP16), {}), (dict(pages=0), {}),
             (dict(pages=1 << 31), {}), (dict(page_size=0), {}), (dict(page_size=24), {}),
             (dict(page_size=1 << 17), {}), (dict(dim=12), {}), (dict(dim=0), {}),
             (dict(kv_heads=0), {}), (dict(k=None), {}), (dict(v=A + 8), {}),
             (dict(type=ep.EP_E4M3, k_scale=None), {}), (dict(type=ep.EP_E4M3, v_scale=None), {}),
             ({}, dict(batch=0)), ({}, dict(cols=0)), ({}, dict(cols=1 << 26)),
             ({}, dict(table=None)), ({}, dict(lengths=None))]


@pytest.mark.parametrize("c,p", BAD_CACHE)
def test_cache_refuses(c, p):
    cache, pages = _cache(**c), _table(**p)
    for name in ("ep_cache_write", "ep_cache_read"):
        assert ep.raw_call(name, ctypes.byref(cache), ctypes.byref(pages), ep.EP_BF16, _rows(),
                           _rows(), 10, A, None) == ep.EP_EINVAL
    a = _attn()
    assert ep.raw_call("ep_cache_attention", ctypes.byref(a), ctypes.byref(cache),
                       ctypes.byref(pages), _rows(), _rows(), A, A, 1 << 30, None) == ep.EP_EINVAL
    assert ep.raw_call("ep_cache_attention_bytes", ctypes.byref(a), ctypes.byref(cache),
                       ctypes.byref(pages)) == ep.EP_EINVAL


@pytest.mark.parametrize("kw", [dict(kv_heads=4), dict(dim=128), dict(batch=3),
                                dict(type=ep.EP_FP16), dict(start_q=None), dict(scale=0.0)])
def test_cache_attention_refuses(kw):
    a = _attn(**kw)
    assert ep.raw_call("ep_cache_attention", ctypes.byref(a), ctypes.byref(_cache()),
                       ctypes.byref(_table()), _rows(), _rows(), A, A, 1 << 30,
                       None) == ep.EP_EINVAL


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(tokens=1 << 30), dict(start=None),
                                dict(k=_rows(data=None)), dict(v=_rows(row=4)), dict(type=2)])
def test_cache_moves_refuse(kw):
    d = dict(type=ep.EP_BF16, k=_rows(), v=_rows(), tokens=10, start=A)
    d.update(kw)
    for name in ("ep_cache_write", "ep_cache_read"):
        assert ep.raw_call(name, ctypes.byref(_cache()), ctypes.byref(_table()), d["type"], d["k"],
                           d["v"], d["tokens"], d["start"], None) == ep.EP_EINVAL


def test_null_cache():
    assert ep.raw_call("ep_cache_write", None, None, 0, _rows(), _rows(), 1, A, None) == ep.EP_EINVAL


def test_binding_refuses_host_tensors():
    import torch
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    s = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        ep.ep_attention(q, q, q, q.clone(), None, s, s)
    with pytest.raises((TypeError, ValueError)):
        ep.ep_attention(q.float(), q, q, q.clone(), None, s, s)
    with pytest.raises(ValueError):
        ep.EpCache(torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 16, 2, 64)))
    with pytest.raises(ValueError):
        ep.EpCache(*[torch.zeros((2, 16, 2, 64), dtype=torch.uint8)] * 2)
