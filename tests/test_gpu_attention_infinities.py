"""Infinite values that only some rows of a chunk see, against the oracle: which columns are +inf, -inf or NaN, and that the others are what they are.
The contexts are long enough to be cut into parts, and the values stand on both sides of a border between tiles of 128 positions."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2511_22972_b200 import ChunkAttention
from tests._cache import HALF, rows
from tests.test_gpu_attention import held, stream

pytestmark = pytest.mark.gpu
COLUMN = 5


def put(pool, b, p, sign):
    """Position p of sequence b gets an infinite value in one column."""
    page, slot = int(pool.table[b, p // pool.page]), p % pool.page
    if pool.fmt == "bf16":
        pool.v_pages[page, slot, 0, COLUMN] = sign * math.inf
    else:                                                          # code 448 times 2^127
        pool.v_pages.view(torch.uint8)[page, slot, 0] = 0
        pool.v_pages.view(torch.uint8)[page, slot, 0, COLUMN] = 0x7e if sign > 0 else 0xfe
        pool.v_scales[page, 0, slot] = 254


def check(pool, q, out, lse, window, sinks):
    """Tolerances of finite columns as in check_attention: two roundings to bf16, scores and sums in fp32."""
    scale = 1 / math.sqrt(pool.D)
    vals = [torch.tensor(x).to(torch.bfloat16).double().numpy() for x in pool.values()]    # what is held is a bf16 number
    seen_infinite = 0
    for b in range(q.shape[0]):
        L = int(pool.lengths[b])
        k, v, _ = pool.sequence(vals, b, L + q.shape[1])
        for i in range(q.shape[1]):
            see = np.array(O.visible(L + i, window, sinks))
            for h in range(q.shape[2]):
                x = q[b, i, h].double().cpu().numpy()
                with np.errstate(invalid="ignore"):
                    want, want_lse = O.attend_row(x, k[see, 0], v[see, 0], scale)
                got = out[b, i, h].double().cpu().numpy()
                d = pool.D * 2.0 ** -23 * scale * (np.abs(k[see, 0]) @ np.abs(x)).max() + 2.0 ** -21 + len(see) * 2.0 ** -24
                size, _ = O.attend_row(x, k[see, 0], np.abs(v[see, 0]), scale)
                fin = np.isfinite(want)
                seen_infinite += int((~fin).any())
                assert np.array_equal(got[~fin], want[~fin], equal_nan=True), (b, i, h, got[~fin], want[~fin])
                got, want, size = got[fin], want[fin], size[fin]
                assert (np.abs(got - want) <= size * (HALF + 2 * d) + np.abs(want) * HALF).all(), (b, i, h)
                assert abs(float(lse[b, i, h]) - want_lse) <= 2 * d + abs(want_lse) * 2.0 ** -22
    assert seen_infinite


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads", [4, 16])             # 80 rows: one row tile; 16 heads: pairs of tiles of eight tokens
@pytest.mark.parametrize("L,window,sinks,at", [
    (500, 0, 0, ((507, 1), (513, 1))),                 # later tokens of the chunk
    (500, 0, 0, ((507, 1), (513, -1))),
    (500, 0, 0, ((507, -1), (509, -1), (515, 1))),
    (500, 0, 0, ((513, 1),)),
    (700, 326, 0, ((380, 1), (390, 1))),               # positions that leave the window, tiles 2 and 3
    (700, 326, 10, ((380, 1), (390, -1), (3, 1))),
    (1020, 0, 0, ((1022, 1), (1023, 1), (1024, 1), (1037, -1))),
])
def test_infinite_values_that_some_rows_see(fmt, heads, L, window, sinks, at):
    n = 20
    pool = held([L, 90], n, 1, 64, 16, fmt, seed=L + heads)
    for p, sign in at:
        put(pool, 0, p, sign)
    q = rows(2, n, heads, 64, torch.Generator(device="cuda").manual_seed(3))
    out, lse = torch.zeros_like(q), torch.zeros(2, n, heads, device="cuda")
    ChunkAttention(2, n, heads, 1, 64).run(pool.cache, q, out, window=window, sinks=sinks, lse=lse, stream=stream())
    torch.cuda.synchronize()
    check(pool, q, out, lse, window, sinks)
