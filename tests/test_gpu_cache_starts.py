"""What only the device sees of a cache move's arguments."""

import numpy as np
import pytest

from attention_common import rounded
from test_gpu_cache import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [False, True])
def test_starts_outside_the_rows_are_the_nearest_inside(eight):
    """As everywhere with packed rows."""
    import torch
    rng = np.random.default_rng(3)
    totals, g, d = [40, 25], 2, 64
    k, v = (rounded(rng, (30, g, d), "bf16").cuda() for _ in range(2))
    got = []
    for s in ([0, 18, 30], [-7, 18, 1 << 30], [-(2 ** 31), 18, 2 ** 31 - 1]):
        c = Cache(np.random.default_rng(5), "bf16", eight, g, d, 16, totals)
        c.ep.ep_cache_write(c.c, k, v, c.table, c.ints(totals), c.ints(s), c.err)
        back = [torch.full((30, g, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        c.ep.ep_cache_read(c.c, *back, c.table, c.ints([18, 12]), c.ints(s), c.err)
        assert c.err.item() == 0
        got.append([x.view(torch.uint8) for x in (c.k, c.v, *back)])
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


def test_lengths_past_the_table_are_reported():
    import torch
    rng = np.random.default_rng(3)
    c = Cache(rng, "fp16", False, 2, 64, 16, [48, 48])
    k, v = (rounded(rng, (96, 2, 64), "fp16").cuda() for _ in range(2))
    c.write(k, v, [48, 48], [48, 48])
    for length in (49, 2 ** 31 - 1):
        c.err.zero_()
        back = [torch.full((20, 2, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
        c.ep.ep_cache_read(c.c, *back, c.table, c.ints([length, 48]), c.ints([0, 8, 20]), c.err)
        assert c.err.item() == 1 and torch.equal(back[0][8:], k[48:60])
    c.err.zero_()
    c.ep.ep_cache_read(c.c, *back, c.table, c.ints([48, 48]), c.ints([0, 8, 20]), c.err)
    assert c.err.item() == 0
