"""Writing rows into a paged cache and reading them back, against the fp64 oracle: bit-exact."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2511_22972_b200 import binding as Bd, cache as C, cache_append, cache_read
from tests._cache import Pool, rows

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def raw(pool):
    """Everything that a cache holds, as bytes."""
    return [t.contiguous().view(torch.uint8).cpu().clone() for t in (pool.k_pages, pool.v_pages, pool.k_scales, pool.v_scales) if t is not None]


def check_append(pool, k, v, counts=None, flags=None):
    """The pool after an append of k, v against the oracle applied to the pool before it (`before`: its bytes)."""
    before = [t.clone() for t in (pool.k_pages, pool.v_pages, pool.k_scales, pool.v_scales) if t is not None]
    fl = None if flags is None else torch.full((pool.B, k.shape[1]), 77, dtype=torch.int32, device="cuda")
    cache_append(pool.cache, k, v, counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"), row_flags=fl,
                 stream=stream())
    torch.cuda.synchronize()
    after = [t.clone() for t in (pool.k_pages, pool.v_pages, pool.k_scales, pool.v_scales) if t is not None]
    total = pool.k_pages.shape[0]
    src = [x.float().cpu().double().numpy() for x in (k, v)]
    want_flags = np.full((pool.B, k.shape[1]), 77)
    touched = torch.zeros(total, pool.page, dtype=torch.bool)
    for b in range(pool.B):
        L = O.held_length(int(pool.lengths[b]), pool.table[b].tolist(), pool.page)
        for i in range(O.held_count(counts, b, k.shape[1])):
            at = O.place(pool.table[b].tolist(), L + i, pool.page, total) if L >= 0 else None
            want_flags[b, i] = 0 if at else C.FLAG_NOT_WRITTEN
            if at is None:
                continue
            touched[at] = True
            for t in range(2):
                for h in range(pool.H):
                    got = after[t][at[0], at[1], h].float().cpu().double().numpy()
                    if pool.fmt == "bf16":
                        assert torch.equal(after[t][at[0], at[1], h].view(torch.int16), (k, v)[t][b, i, h].view(torch.int16))
                        continue
                    codes, s = O.quantise_row(src[t][b, i, h])
                    assert int(after[2 + t][at[0], h, at[1]]) == s, (b, i, h, t)
                    assert (got == codes).all() and (np.signbit(got) == np.signbit(codes))[codes != 0].all(), (b, i, h, t)
    for x, y in zip(before, after):          # nothing else moved
        rest = ~touched.to("cuda")
        x, y = (x, y) if x.dim() == 4 and x.shape[1] == pool.page else (x.transpose(1, 2), y.transpose(1, 2))
        assert torch.equal(x.contiguous().view(torch.uint8)[rest], y.contiguous().view(torch.uint8)[rest])
    if flags is not None:
        assert fl.cpu().numpy().tolist() == want_flags.tolist()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim,kv_heads,page,layout,n,lengths", [
    (128, 8, 16, "nhd", 16, [1000]),
    (128, 8, 16, "nhd", 9, [0, 7, 15, 16, 31, 100]),
    (64, 2, 8, "hnd", 5, [0, 3, 8]),
    (64, 5, 64, "pair", 70, [60, 0, 64]),
    (128, 1, 256, "hnd", 1, [255, 256, 0]),
    (128, 3, 32, "pair", 33, [31, 32]),
])
def test_append(fmt, dim, kv_heads, page, layout, n, lengths):
    g = torch.Generator(device="cuda").manual_seed(5)
    pool = Pool(lengths, n, kv_heads, dim, page, fmt, layout)
    for strided in (False, True):
        k, v = rows(pool.B, n, kv_heads, dim, g, strided), rows(pool.B, n, kv_heads, dim, g, not strided, std=30.0)
        check_append(pool, k, v, flags=True)
    counts = [(3 * b) % (n + 1) for b in range(pool.B)]
    check_append(pool, rows(pool.B, n, kv_heads, dim, g), rows(pool.B, n, kv_heads, dim, g), counts, flags=True)


def test_values_at_the_borders_of_the_format():
    n, H, D = 40, 2, 64
    pool = Pool([5], n, H, D, 16, "e4m3")
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = rows(1, n, H, D, g), rows(1, n, H, D, g)
    grid = torch.tensor(O.GRID, device="cuda")
    mid = ((grid[1:] + grid[:-1]) / 2)
    mid = mid[mid.bfloat16().double() == mid]                      # the ties that bf16 can hold
    k[0, :10, 0] = torch.cat([mid, -mid])[torch.randint(0, 2 * len(mid), (10, D), device="cuda")].bfloat16()
    k[0, :10, 0, 0] = 448.0                                        # scale 127: codes are the values
    k[0, 10] = 0.0
    k[0, 11] = -0.0
    k[0, 12, 0] = torch.full((D,), 3.3895e38).bfloat16()           # the largest finite
    k[0, 13, 0] = 1e-38
    k[0, 14, 0] = 9.2e-41                                          # the smallest subnormal
    k[0, 15, 0, 3] = float("inf")
    k[0, 16, 0, 63] = float("nan")
    k[0, 17, 1, 9] = float("-inf")
    k[0, 18, 0] = 2.0 ** -112
    k[0, 18, 0, 5] = 448 * 2.0 ** -120
    k[0, 19, 0, 5] = 450.0
    for e in range(-16, 20):
        v[0, e + 16] = (torch.randn(H, D, device="cuda", generator=g) * 2.0 ** (6 * e)).bfloat16()
    check_append(pool, k, v)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_rows_at_every_alignment(fmt):
    n, H, D = 6, 3, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    for off in range(8):
        pool = Pool([10, 20], n, H, D, 16, fmt, seed=off)
        flat = torch.randn(2, 2 * n * (H * D + 1) + 16, device="cuda", generator=g).bfloat16()
        k, v = (flat[t][off + t:].as_strided((2, n, H, D), (n * (H * D + 1), H * D + 1, D, 1)) for t in range(2))
        check_append(pool, k, v)
        pool.lengths += n
        pool.refresh()
        back = torch.zeros(2, 2 * n * (H * D + 1) + 16, device="cuda", dtype=torch.bfloat16)
        ko, vo = (back[t][off + t:].as_strided((2, n, H, D), (n * (H * D + 1), H * D + 1, D, 1)) for t in range(2))
        cache_read(pool.cache, ko, vo, starts=(pool.d_lengths - n), stream=stream())
        vals = pool.values()
        for b in range(2):
            for t, out in enumerate((ko, vo)):
                seq = pool.sequence(vals, b, int(pool.lengths[b]))[t][-n:]
                assert (out[b].float().cpu().double().numpy() == seq).all()
        assert not back[0][:off].any() and int((back[0] != 0).sum()) <= 2 * n * H * D


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_bad_lengths_counts_and_pages_write_nothing_outside(fmt):
    n = 12
    pool = Pool([20, 30, 5, 16, 40, 9, 9], n, 2, 64, 16, fmt)      # 4 pages each: positions 0 .. 63
    total = pool.k_pages.shape[0]
    pool.lengths = torch.tensor([-1, 2 ** 31 - 1, 60, 64, 65, 20, 30], dtype=torch.int32)
    pool.table[5, 1] = total
    pool.table[6, 2] = -5
    pool.table[2, 0] = 2 ** 31 - 1
    pool.refresh()
    g = torch.Generator(device="cuda").manual_seed(1)
    check_append(pool, rows(7, n, 2, 64, g), rows(7, n, 2, 64, g), flags=True)
    check_append(pool, rows(7, n, 2, 64, g), rows(7, n, 2, 64, g), [12, 12, 13, -1, 12, 2 ** 31 - 1, 0], flags=True)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim,kv_heads,page,layout,n,lengths,starts", [
    (128, 8, 16, "nhd", 1003, [1003], None),
    (64, 3, 8, "pair", 50, [0, 1, 7, 49, 50, 51, 200], None),
    (128, 2, 64, "hnd", 77, [0, 64, 128, 300, 90, 20], [0, 60, -20, 250, 2 ** 31 - 1, -2 ** 31]),
])
def test_read(fmt, dim, kv_heads, page, layout, n, lengths, starts):
    pool = Pool(lengths, n, kv_heads, dim, page, fmt, layout, seed=3)
    if pool.B > 3:
        pool.table[3, 1] = -1
        pool.lengths[2] = pool.table.shape[1] * page + 1           # not a length: nothing is held
        pool.refresh()
    vals = pool.values()
    ko, vo = (torch.full((pool.B, n, kv_heads + t, dim), 7.5, dtype=torch.bfloat16, device="cuda")[:, :, t:] for t in range(2))
    cache_read(pool.cache, ko, vo, starts=None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda"), stream=stream())
    for b in range(pool.B):
        L, s = O.held_length(int(pool.lengths[b]), pool.table[b].tolist(), page), 0 if starts is None else starts[b]
        seq = pool.sequence(vals, b, max(L, 0))
        for i in range(n):
            for t, out in enumerate((ko, vo)):
                want = seq[t][s + i] if 0 <= s + i < L and seq[2][s + i] else np.full((kv_heads, dim), 7.5)
                assert (out[b, i].float().cpu().double().numpy() == want).all(), (b, i, t)


def test_a_page_past_32_bits():
    # 40000 pages of 64 tokens x 8 heads x 128: 2.6e9 elements in a tensor
    pages, page, H, D = 40000, 64, 8, 128
    kp = torch.zeros(pages, page, H, D, dtype=torch.float8_e4m3fn, device="cuda")
    vp = torch.zeros_like(kp)
    ks, vs = (torch.full((pages, H, page), 127, dtype=torch.uint8, device="cuda") for _ in "kv")
    table = torch.tensor([[39999, 33333]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([60], dtype=torch.int32, device="cuda")
    cache = C.PagedCache(kp, vp, table, lengths, ks, vs)
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = rows(1, 10, H, D, g), rows(1, 10, H, D, g)
    cache_append(cache, k, v, stream=stream())
    lengths += 10
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    cache_read(cache, ko, vo, starts=lengths - 10, stream=stream())
    for x, y in ((k, ko), (v, vo)):
        for i in range(10):
            for h in range(H):
                codes, s = O.quantise_row(x[0, i, h].float().cpu().double().numpy())
                assert (y[0, i, h].float().cpu().double().numpy() == O.row_values(codes, s)).all()
    assert bool(kp[39999, 60:].float().any()) and bool(kp[33333, :6].float().any()) and not bool(kp[39999 - 2 ** 31 // (page * H * D)].float().any())


def test_captured_and_replayed_between_plain_calls():
    n, H, D = 9, 8, 128
    g = torch.Generator(device="cuda").manual_seed(8)
    pool = Pool([10, 100], 4 * n, H, D, 16, "e4m3")
    k, v = rows(2, n, H, D, g), rows(2, n, H, D, g)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        cache_append(pool.cache, k, v, stream=side.cuda_stream)
        pool.d_lengths.add_(n)
        cache_read(pool.cache, ko, vo, starts=pool.d_lengths - n, stream=side.cuda_stream)
    for _ in range(3):
        k.copy_(rows(2, n, H, D, g))
        v.copy_(rows(2, n, H, D, g))
        graph.replay()
        torch.cuda.synchronize()
        pool.lengths = pool.d_lengths.cpu()
        for x, y in ((k, ko), (v, vo)):
            codes, s = O.quantise_row(x[1, 3, 5].float().cpu().double().numpy())
            assert (y[1, 3, 5].float().cpu().double().numpy() == O.row_values(codes, s)).all()
    assert pool.lengths.tolist() == [10 + 3 * n, 100 + 3 * n]


def test_refusals():
    pool = Pool([10, 20], 4, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(8)
    k = rows(2, 4, 2, 64, g)
    for bad in (rows(3, 4, 2, 64, g),):                              # more sequences than the cache has
        with pytest.raises(Bd.FlyError) as e:
            cache_append(pool.cache, bad, bad)
        assert e.value.status == Bd.FLY_ERR_INVALID_ARG
    for bad in (k.cpu(), k.float(), k[0], rows(2, 4, 3, 64, g), rows(2, 4, 2, 128, g), k.transpose(2, 3), k[:, :0], k[:0]):
        with pytest.raises((ValueError, Bd.FlyError)):
            cache_append(pool.cache, bad, bad)
        with pytest.raises((ValueError, Bd.FlyError)):
            cache_read(pool.cache, bad, bad)
    for kw in (dict(counts=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(counts=torch.zeros(2, device="cuda")),
               dict(counts=torch.zeros(2, dtype=torch.int32)), dict(row_flags=torch.zeros(2, 3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            cache_append(pool.cache, k, k, **kw)
    for bad in (lambda p: (p.k_pages, p.v_pages[:, :, :1], p.d_table, p.d_lengths), lambda p: (p.k_pages.float(), p.v_pages.float(), p.d_table, p.d_lengths),
                lambda p: (p.k_pages, p.v_pages, p.d_table.long(), p.d_lengths), lambda p: (p.k_pages, p.v_pages, p.d_table, p.d_lengths[:1]),
                lambda p: (p.k_pages, p.v_pages, p.d_table.cpu(), p.d_lengths), lambda p: (p.k_pages.cpu(), p.v_pages.cpu(), p.table, p.lengths),
                lambda p: (p.k_pages, p.v_pages, p.d_table, p.d_lengths, torch.zeros(1, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            C.PagedCache(*bad(pool))
