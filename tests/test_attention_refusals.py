"""More refusals of the attention calls, without a GPU."""

import ctypes
import os
import subprocess
import sys

import pytest

import paper_1806_06144_amd as ep
from test_attention_host import A, _attn, _backward, _cache, _rows, _table


def _forward(a, out):
    """(with a bad address for work: what passes the checks of rows stops there)"""
    return ep.raw_call("ep_attention", ctypes.byref(a), _rows(), _rows(), _rows(), out, A, A + 4,
                       1 << 30, None)


def _overlap(row, head, tokens, heads, dim):
    """By the definition: does any pair of rows share an element?"""
    at = sorted(t * row + h * head for t in range(tokens) for h in range(heads))
    return any(b - a < dim for a, b in zip(at, at[1:]))


LAYOUTS = [(64, 64), (512, 64), (64, 6400), (64, 448), (128, 192), (192, 128), (72, 64), (64, 72),
           (520, 64), (504, 64), (64, 6336), (64, 6392), (128, 64), (256, 64), (320, 128),
           (1 << 23, 64), (64, 1 << 40), (640, 192), (136, 408), (64, 1 << 62)]


@pytest.mark.parametrize("row,head", LAYOUTS)
@pytest.mark.parametrize("name,heads", [("out", 8), ("dq", 8), ("dk", 2), ("dv", 2), ("read", 2)])
def test_outputs_whose_rows_overlap(name, heads, row, head):
    """100 tokens of 8 heads, 2 key heads, of 64 elements."""
    rows, cache, pages = _rows(row=row, head=head), _cache(), _table()
    if name == "out":
        rc = _forward(_attn(), rows)
    elif name == "read":                             # (start, checked before v, is left out)
        rc = ep.raw_call("ep_cache_read", ctypes.byref(cache), ctypes.byref(pages), ep.EP_BF16,
                         rows, _rows(data=A + 2), 100, A, None)
        name = "k"
    else:
        rc = _backward(_attn(), work=A + 4, **{name: rows})
    assert rc == ep.EP_EINVAL
    refused = ep.ep_last_error().startswith(name + ":")
    assert refused == _overlap(row, head, 100, heads, 64), ep.ep_last_error()


def test_one_token_or_one_head_needs_no_stride():
    """The stride of an axis of one element is not looked at."""
    for a, out in ((_attn(tokens_q=1), _rows(row=0)), (_attn(heads=1, kv_heads=1), _rows(head=0))):
        assert _forward(a, out) == ep.EP_EINVAL and "work" in ep.ep_last_error()


def test_a_scale_that_overflows_in_units_of_log_2():
    """scale log2(e) has to be finite as well."""
    for scale, fine in ((2.3e38, True), (2.4e38, False), (3.4e38, False), (1e-45, True)):
        a = _attn(scale=scale)
        rc = ep.raw_call("ep_attention_bytes", ctypes.byref(a))
        assert (rc >= 0) == fine
        assert fine or "scale" in ep.ep_last_error()


class _Stream:
    def __init__(self, device):
        self.device = device


def test_a_stream_of_another_device():
    """Work on one device's tensors does not go to another device's stream."""
    import torch
    called = []
    with pytest.raises(ValueError, match="stream"):
        ep._on_stream(torch.device("cuda", 0), _Stream(torch.device("cuda", 1)),
                      lambda *a: called.append(a))
    assert not called


def test_rows_of_no_elements():
    """dim = 0 has no scale of its own; it is refused like any other bad dim."""
    import torch
    q, s = torch.zeros((4, 2, 0), dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    a = ep._attn(q, 2, 4, s, s, None, True, 0, q.device)
    assert ep.raw_call("ep_attention_bytes", ctypes.byref(a)) == ep.EP_EINVAL


def test_the_binding_loads_beside_a_torch_without_devices():
    """As it did before it had attention."""
    program = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_1806_06144_amd as ep
print(ep.raw_call("ep_sync", None) == ep.EP_EINVAL)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", program], cwd=root, capture_output=True, text=True)
    assert r.stdout == "True\n", r.stderr
