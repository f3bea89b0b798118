"""Over e4m3 a query is taken as the sum of an e4m3 and an e5m2 part.  How far that is off, one value at a time: a sequence of one position whose key
is 1 in one dimension and 0 in the others has that value, times the scale, for its logarithm of the sum."""
import math

import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, PagedCache, binding as Bd
from tests._cache import rows
from tests.test_gpu_attention import held, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 12])                       # 16 heads: one row tile, and a pair of them
@pytest.mark.parametrize("top", [1.0, 1.75, 1.984375, 448.0 * 2.0 ** 60, 2.0 ** -100])
def test_values_of_a_query_row_are_as_exact_as_the_header_says(tokens, top):
    D, heads, big = 64, 16, 2.0 ** 20
    pages = torch.zeros(D, 16, 1, D, device="cuda")
    pages[torch.arange(D), :, 0, torch.arange(D)] = 1.0           # page d: keys that are 1 in dimension d
    v = torch.zeros_like(pages).to(torch.float8_e4m3fn)
    s = [torch.full((D, 1, 16), 127, dtype=torch.uint8, device="cuda") for _ in "kv"]
    cache = PagedCache(pages.to(torch.float8_e4m3fn), v, torch.arange(D, dtype=torch.int32, device="cuda").view(D, 1),
                       torch.zeros(D, dtype=torch.int32, device="cuda"), *s)
    g = torch.Generator(device="cuda").manual_seed(3)
    # every mantissa, over 32 binades below the row's largest value; sequence d looks at dimension d
    q = (1 + torch.randint(0, 128, (D, tokens, heads, D), generator=g, device="cuda") / 128.0) * torch.exp2(-torch.randint(1, 33, (D, tokens, heads, D), generator=g, device="cuda").float())
    q = q * torch.where(torch.rand(q.shape, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    q = (q * top).bfloat16()
    d = torch.arange(D, device="cuda")
    q[d, :, :, (d + 1) % D] = top                                 # the largest, which nobody looks at
    att, lse = ChunkAttention(D, tokens, heads, 1, D), torch.zeros(D, tokens, heads, device="cuda")
    att.run(cache, q, torch.zeros_like(q), lse=lse, scale=big / top, stream=stream())
    x = q[d, :, :, d].double() / top                              # row i of a chunk sees i + 1 positions, all alike
    many = torch.log(torch.arange(1, tokens + 1, device="cuda", dtype=torch.float64))[None, :, None]
    got = (lse.double() - many) / big
    # fp32: the scale and two products (2^-22 of the value), a logarithm and its exponential (2^-20 of 1, here 2^-40 of the largest)
    fp32 = x.abs() * 2.0 ** -22 + 2.0 ** -39
    off = (got - x).abs()
    split = torch.where(x.abs() >= 2.0 ** -13.8, 0.0, 2.0 ** -21.8)
    assert bool((off <= fp32 + split).all()), float((off - fp32 - split).max())
    assert bool((off > fp32).any())                               # (the second figure is not idle)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [5, 40])
def test_queries_behind_the_chunks_end_have_no_influence(fmt, n):
    counts = [2, n - 1, 0, n]
    pool = held([300, 20, 5, 0], n, 2, 64, 16, fmt, seed=8)
    q = rows(4, n, 16, 64, torch.Generator(device="cuda").manual_seed(2))
    c, att = torch.tensor(counts, dtype=torch.int32, device="cuda"), ChunkAttention(4, n, 16, 2, 64)
    res = []
    for bad in (0.0, math.nan, math.inf):
        p = q.clone()
        for b, m in enumerate(counts):
            p[b, m:] = bad
        out, lse = torch.full_like(q, 3.0), torch.full((4, n, 16), 3.0, device="cuda")
        att.run(pool.cache, p, out, counts=c, lse=lse, stream=stream())
        res.append((out, lse))
    assert att.device_status(stream()) == Bd.FLY_OK
    for out, lse in res[1:]:
        assert torch.equal(out, res[0][0]) and torch.equal(lse, res[0][1]) and bool(out.isfinite().all())
