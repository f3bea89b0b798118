"""Lengths and tables that a cache is given after it was made."""
import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, PagedCache, cache_append, cache_read
from tests._cache import Pool, check_attention, rows
from tests.test_gpu_cache import check_append, stream

pytestmark = pytest.mark.gpu


def test_calls_use_the_lengths_and_the_table_that_the_cache_has_now():
    n = 6
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = Pool([10, 20], 40, 2, 64, 16)
    old = pool.d_lengths
    pool.cache.lengths = pool.cache.lengths + 7
    pool.lengths = pool.lengths + 7
    assert pool.cache.lengths.data_ptr() != old.data_ptr()
    check_append(pool, rows(2, n, 2, 64, g), rows(2, n, 2, 64, g))
    # a longer table, whose rows stand elsewhere
    more = torch.zeros(2, pool.table.shape[1] + 3, dtype=torch.int32)
    more[:, :-3] = pool.table.flip(1)
    pool.table = more
    pool.cache.block_table = more.to("cuda")
    k, v = rows(2, n, 2, 64, g), rows(2, n, 2, 64, g)
    check_append(pool, k, v)
    att, q = ChunkAttention(2, n, 8, 2, 64), rows(2, n, 8, 64, g)
    out, lse = torch.zeros_like(q), torch.zeros(2, n, 8, device="cuda")
    pool.k_pages[pool.k_pages != pool.k_pages] = 0.5               # (slots that nobody held before the table was turned round)
    pool.v_pages[pool.v_pages != pool.v_pages] = 0.5
    att.run(pool.cache, q, out, lse=lse, stream=stream())
    check_attention(pool, q, out, lse)
    pool.cache.lengths = pool.cache.lengths + n
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    cache_read(pool.cache, ko, vo, starts=pool.cache.lengths - n, stream=stream())
    assert torch.equal(ko, k) and torch.equal(vo, v)


def test_what_a_cache_refuses_to_be_given():
    pool = Pool([10, 20], 4, 2, 64, 16, "e4m3")
    c = pool.cache
    for bad in (pool.d_lengths[:1], pool.d_lengths.long(), pool.lengths, torch.zeros(2, 2, dtype=torch.int32, device="cuda")[:, 0], None):
        with pytest.raises(ValueError):
            c.lengths = bad
    for bad in (pool.d_table[:1], pool.d_table.long(), pool.table, pool.d_table[:1].expand(2, -1), None):
        with pytest.raises(ValueError):
            c.block_table = bad
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name).clone())
    assert c.lengths is pool.d_lengths and c.block_table is pool.d_table
    g = torch.Generator(device="cuda").manual_seed(1)
    check_append(pool, rows(2, 4, 2, 64, g), rows(2, 4, 2, 64, g))
