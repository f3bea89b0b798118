"""Rows whose largest magnitude is next to the end of bf16: written, read back and attended to as finite values."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2511_22972_b200 import cache_read
from tests._cache import Pool, rows
from tests.test_gpu_cache import check_append, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
def test_the_largest_finite_values_read_back_finite(dim):
    H, g = 2, torch.Generator(device="cuda").manual_seed(2)
    tops = torch.arange(0x7f40, 0x7f80, dtype=torch.int16, device="cuda").view(torch.bfloat16)      # the last 64 numbers: 1.5 * 2^127 and more
    n = len(tops)
    pool = Pool([5], n, H, dim, 16, "e4m3")
    k, v = rows(1, n, H, dim, g), rows(1, n, H, dim, g)
    k[0, :, 0, 3] = tops
    k[0, :, 0, dim - 1] = -tops
    v[0, :, 1, :] = -tops[:, None]
    v[0, :, 1, 1::2] = tops.flip(0)[:, None]
    check_append(pool, k, v)
    pool.lengths += n
    pool.refresh()
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    cache_read(pool.cache, ko, vo, starts=pool.d_lengths - n, stream=stream())
    for x, y in ((k, ko), (v, vo)):
        assert bool(y.isfinite().all())
        for i in range(n):
            for h in range(H):
                want = O.row_values(*O.quantise_row(x[0, i, h].float().cpu().double().numpy()))
                assert (y[0, i, h].float().cpu().double().numpy() == want).all(), (i, h)
