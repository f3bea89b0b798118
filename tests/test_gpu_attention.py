"""Attention of a chunk over a paged cache against the fp64 oracle."""
import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, PagedCache, binding as Bd
from tests._cache import Pool, check_attention, rows

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def run(pool, n, heads, window=0, sinks=0, scale=0.0, counts=None, strided=False, seed=0, handle=None, rows_of=None, std=2.0, q=None):
    """One step over the first n positions behind pool.lengths (which the pool already holds), checked."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = rows(pool.B, n, heads, pool.D, g, False, std) if q is None else q
    if strided:
        wide = torch.zeros(pool.B, n, heads + 3, pool.D + 8, dtype=torch.bfloat16, device="cuda")
        wide[:, :, 1:1 + heads, :pool.D] = q
        q = wide[:, :, 1:1 + heads, :pool.D]
    out = torch.full((pool.B, heads, n, pool.D), 3.25, dtype=torch.bfloat16, device="cuda").transpose(1, 2) if strided else torch.full(
        (pool.B, n, heads, pool.D), 3.25, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((pool.B, n, heads), 5.5, device="cuda")
    before = out.clone(), lse.clone()
    att = handle or ChunkAttention(pool.B, n, heads, pool.H, pool.D)
    att.run(pool.cache, q, out, window=window, sinks=sinks, scale=scale,
            counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"), lse=lse, stream=stream())
    torch.cuda.synchronize()
    assert att.last_launch_count >= 1
    check_attention(pool, q, out, lse, window, sinks, scale, counts, before, rows_of)
    if handle is None:
        att.close()
    return q, out, lse


def held(lengths, n, *a, **kw):
    """A pool that also holds the n positions of the chunk, with lengths as they were before it."""
    pool = Pool([L + n for L in lengths], 0, *a, **kw)
    pool.lengths = torch.tensor(lengths, dtype=torch.int32)
    pool.refresh()
    return pool


FORMATS = ["bf16", "e4m3"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 1, 128), (4, 2, 64), (7, 1, 64), (3, 3, 128), (16, 1, 128), (40, 2, 64)])
@pytest.mark.parametrize("n", [1, 2, 9, 17])
def test_head_layouts_and_chunks(fmt, heads, kv_heads, dim, n):
    run(held([0, 1, 60, 127, 128, 129, 300], n, kv_heads, dim, 16, fmt, seed=n), n, heads, seed=n)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_pages_and_layouts(fmt, page, layout):
    run(held([0, 5, 200, 255, 256, 511], 4, 2, 64, page, fmt, layout, seed=page), 4, 6, strided=True, seed=page)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("L", [0, 1, 7, 15, 16, 119, 120, 121, 126, 127, 128, 136, 248, 255, 256, 257, 383, 384, 640, 1000])
def test_lengths_around_a_tile(fmt, L):
    run(held([L], 8, 1, 128, 16, fmt, seed=L), 8, 8, seed=L)
    run(held([L, L + 1, 2 * L], 1, 1, 64, 32, fmt, seed=L), 1, 4, seed=L)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 4), (16, 0), (100, 4), (128, 128), (129, 200), (400, 3), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(fmt, window, sinks):
    run(held([0, 3, 130, 255, 700, 1300], 9, 2, 64, 16, fmt, seed=window % 97), 9, 8, window, sinks, seed=sinks % 97)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 0), (150, 20)])
def test_chunks_of_several_row_tiles(fmt, window, sinks):
    # 16 heads to a key/value head: eight tokens to a tile of 128 rows, 16 to a pair of tiles
    for n in (8, 16, 17, 24, 33, 70):
        run(held([0, 100, 333], n, 1, 64, 16, fmt, seed=n), n, 16, window, sinks, seed=n)
    run(held([40], 300, 1, 128, 64, fmt, seed=3), 300, 1, window, sinks, rows_of=set(range(0, 300, 7)) | {127, 128, 255, 256, 299})
    run(held([11, 64], 130, 2, 128, 64, fmt, seed=3), 130, 14, window, sinks, rows_of={0, 1, 17, 18, 35, 36, 37, 71, 72, 128, 129})


@pytest.mark.parametrize("fmt", FORMATS)
def test_counts_leave_rows_as_they_were(fmt):
    n = 20
    pool = held([0, 50, 128, 200, 77, 300, 13, 400], n, 2, 64, 16, fmt)
    run(pool, n, 16, counts=[0, 1, 20, 21, -1, 7, 16, 2 ** 31 - 1], strided=True)
    run(pool, n, 16, 30, 3, counts=[3, 1, 20, 0, 9, 8, 16, 17])


@pytest.mark.parametrize("fmt", FORMATS)
def test_lengths_and_pages_out_of_range(fmt):
    n = 3
    pool = held([40, 40, 40, 40, 45, 150, 200], n, 2, 64, 16, fmt, spare=0)
    total, cap = pool.k_pages.shape[0], pool.table.shape[1] * 16
    pool.lengths = torch.tensor([-1, cap + 1, 2 ** 31 - 1, -2 ** 31, 45, 150, 200], dtype=torch.int32)
    pool.table[4] = -1                                          # no page at all: the rows see nothing
    pool.table[5, 3] = total
    pool.table[5, 9] = 2 ** 31 - 1                              # the page of the chunk itself
    pool.table[6, 0] = -2 ** 31
    pool.refresh()
    run(pool, n, 8)
    run(pool, n, 8, 60, 20)
    full = Pool([cap] * 7, 0, 2, 64, 16, fmt, spare=0, seed=9)  # chunks that run past the table: only what is there is seen
    full.lengths = torch.tensor([cap, cap - 1, cap - 2, cap - 3, cap, cap, cap], dtype=torch.int32)
    full.refresh()
    run(full, n, 8)
    run(full, n, 8, 2, 1)                                       # (windows that hold nothing any more)


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_and_uneven_sequences(fmt):
    lengths = [(37 * b * b) % 900 for b in range(70)] + [6000]
    pool = held(lengths, 2, 2, 64, 16, fmt, seed=4)
    run(pool, 2, 4, rows_of={1})
    run(pool, 2, 4, 300, 5, rows_of={0})


def test_long_contexts_are_cut_into_parts():
    run(held([30000], 16, 1, 128, 16, "bf16", seed=1), 16, 8, rows_of={0, 15})
    run(held([20000, 10], 5, 2, 64, 64, "e4m3", seed=1), 5, 4, rows_of={0, 4})


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("std,scale", [(30.0, 0.0), (0.01, 0.0), (2.0, 0.7), (2.0, 1e-4)])
def test_sharp_and_flat_softmax(fmt, std, scale):
    run(held([500, 1000], 4, 1, 64, 16, fmt, seed=5, std=3.0), 4, 4, scale=scale, std=std)


@pytest.mark.parametrize("heads", [4, 16])
@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (140, 10)])
def test_what_a_row_does_not_see_has_no_influence(what, heads, window, sinks):
    # values and keys of later tokens of the chunk, of positions that have left the window of some rows, and behind the end
    n, L = 20, 500
    pool = held([L], n, 1, 64, 16, "bf16", seed=6)
    bad = float(what)
    at = lambda p: (int(pool.table[0, p // 16]), p % 16)  # noqa: E731
    bads = (L + 7, L + 13, L + n - 1) if not window else (L + 13, L + n - 1, L - 138, L - 139, 12)
    for p in bads:
        pool.v_pages[at(p)][0, 5] = bad
        pool.k_pages[at(p)][0, 9] = bad
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(1, n, heads, 64, g).abs()
    out, lse = torch.zeros_like(q), torch.zeros(1, n, heads, device="cuda")
    att = ChunkAttention(1, n, heads, 1, 64)
    att.run(pool.cache, q, out, window=window, sinks=sinks, lse=lse, stream=stream())
    # (with the window, L - 138 is seen by rows 0 and 1, L - 139 by row 0)
    clean = {i for i in range(n) if not any(p <= L + i and (not window or p > L + i - window or p < sinks) for p in bads)}
    check_attention(pool, q, out, lse, window, sinks, rows_of=clean)
    for i in set(range(n)) - clean:
        assert not bool(out[0, i].isfinite().all()) or not bool(lse[0, i].isfinite().all())
    # only values: the other columns of a row that sees one stay what they are
    pool2 = held([L], n, 1, 64, 16, "bf16", seed=6)
    pool2.v_pages[at(L + 7)][0, 5] = bad
    out2 = torch.zeros_like(q)
    att.run(pool2.cache, q, out2, window=window, sinks=sinks, stream=stream())
    assert bool(out2[0, :7].isfinite().all()) and not bool(out2[0, 7:, :, 5].isfinite().any())
    assert bool(out2[0, :, :, :5].isfinite().all()) and bool(out2[0, :, :, 6:].isfinite().all())


def test_e4m3_rows_that_hold_nan():
    n, L = 10, 300
    pool = held([L], n, 1, 64, 16, "e4m3", seed=6)
    p = L + 4
    pool.v_scales[int(pool.table[0, p // 16]), 0, p % 16] = 255
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(1, n, 8, 64, g)
    out, lse = torch.zeros_like(q), torch.zeros(1, n, 8, device="cuda")
    ChunkAttention(1, n, 8, 1, 64).run(pool.cache, q, out, lse=lse, stream=stream())
    check_attention(pool, q, out, lse, rows_of={0, 1, 2, 3})
    assert bool(out[0, 4:].isnan().all())


def test_scores_of_minus_infinity():
    n, L = 2, 200
    pool = held([L], n, 1, 64, 16, "bf16", seed=6)
    for p in range(L + 1):
        pool.k_pages[int(pool.table[0, p // 16]), p % 16, 0, 0] = float("-inf")
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(1, n, 8, 64, g).abs() + 1
    run(pool, n, 8, q=q)


def test_one_handle_many_shapes():
    att = ChunkAttention(6, 40, 16, 2, 64)
    for seed, (lengths, n, fmt, window, sinks) in enumerate([([5], 1, "bf16", 0, 0), ([700, 3, 90], 9, "e4m3", 0, 0), ([1, 2, 3, 4, 5, 600], 40, "bf16", 64, 4),
                                                           ([2000], 8, "e4m3", 0, 0), ([0], 40, "bf16", 0, 0)]):
        run(held(lengths, n, 2, 64, 16, fmt, seed=seed), n, 16, window, sinks, handle=att, seed=seed, rows_of=set(range(0, n, 3)))
    att.close()


def test_the_same_call_gives_the_same_bits():
    pool = held([3000, 100, 900], 9, 2, 128, 16, "e4m3", seed=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(3, 9, 16, 128, g)
    att = ChunkAttention(3, 9, 16, 2, 128)
    outs = [torch.zeros_like(q) for _ in range(30)]
    for o in outs:
        att.run(pool.cache, q, o, stream=stream())
    torch.cuda.synchronize()
    assert all(torch.equal(o.view(torch.int16), outs[0].view(torch.int16)) for o in outs)


def test_captured_and_replayed_between_plain_calls_and_on_other_streams():
    n = 9
    pool = held([500, 60], n, 2, 64, 16, "bf16", seed=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, out, lse = rows(2, n, 8, 64, g), None, torch.zeros(2, n, 8, device="cuda")
    out = torch.zeros_like(q)
    att = ChunkAttention(2, n, 8, 2, 64)
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for window in (0, 100):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            att.run(pool.cache, q, out, window=window, lse=lse, stream=side.cuda_stream)
        graphs.append(graph)
    for turn in range(4):
        q.copy_(rows(2, n, 8, 64, g))
        pool.lengths = torch.tensor([400 + turn, 17 * turn], dtype=torch.int32)
        pool.refresh()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        check_attention(pool, q, out, lse, window=100 * (turn % 2))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            att.run(pool.cache, q, out, window=7, lse=lse, stream=side.cuda_stream)
        torch.cuda.synchronize()
        check_attention(pool, q, out, lse, window=7)


def test_a_wait_that_runs_out_is_reported_once_and_shows_in_the_rows():
    n = 3
    pool = held([700, 20], n, 1, 64, 16, "bf16", seed=3)
    att = ChunkAttention(2, n, 8, 1, 64)
    run(pool, n, 8, handle=att)
    assert att.device_status(stream()) == Bd.FLY_OK
    assert att.selftest_wait(stream()) == Bd.FLY_OK
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(2, n, 8, 64, g)
    out, lse = torch.zeros_like(q), torch.zeros(2, n, 8, device="cuda")
    att.run(pool.cache, q, out, lse=lse, stream=stream())            # while the record is pending
    assert att.device_status(stream()) == Bd.FLY_ERR_TIMEOUT
    assert bool(out.isnan().all()) and bool(lse.isnan().all())
    assert att.device_status(stream()) == Bd.FLY_OK
    run(pool, n, 8, handle=att)


def test_refusals():
    pool = held([10, 20], 4, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(8)
    q = rows(2, 4, 8, 64, g)
    att = ChunkAttention(2, 4, 8, 2, 64)
    ok = dict(stream=stream())
    att.run(pool.cache, q, torch.zeros_like(q), **ok)
    for kw, error in ((dict(window=-1), ValueError), (dict(sinks=-1), ValueError), (dict(sinks=1), Bd.FlyError), (dict(scale=-1.0), Bd.FlyError),
                      (dict(scale=float("nan")), Bd.FlyError), (dict(scale=float("inf")), Bd.FlyError),
                      (dict(counts=torch.zeros(3, dtype=torch.int32, device="cuda")), ValueError), (dict(lse=torch.zeros(2, 4, 7, device="cuda")), ValueError)):
        with pytest.raises(error):
            att.run(pool.cache, q, torch.zeros_like(q), **kw, **ok)
    for bad in (rows(2, 5, 8, 64, g), rows(3, 4, 8, 64, g), rows(2, 4, 6, 64, g), q.cpu(), q.float(), q.transpose(2, 3)):
        with pytest.raises((ValueError, Bd.FlyError)):
            att.run(pool.cache, bad, torch.zeros_like(bad), **ok)
    flat = torch.zeros(2 * 4 * 8 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for bad in (flat[1:-7].view(2, 4, 8, 64), flat[:4 * 8 * 64].view(1, 4, 8, 64).expand(2, 4, 8, 64)):
        with pytest.raises(Bd.FlyError) as e:                     # not on 16 bytes; a stride of 0
            att.run(pool.cache, bad, torch.zeros_like(q), **ok)
        assert e.value.status == Bd.FLY_ERR_UNSUPPORTED
    with pytest.raises(Bd.FlyError):
        ChunkAttention(2, 4, 8, 4, 64).run(pool.cache, q, torch.zeros_like(q), **ok)   # another shape than the cache's


# ---- row tiles without work, windows behind the table's end, waits that run out in every form of the kernel ------------------

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (43, 20)])
def test_pairs_of_row_tiles_of_which_one_is_empty(fmt, window, sinks):
    # two heads to a key/value head: 64 tokens to a row tile.  Many chunks end in the first tile of a pair, eight heads one after the other,
    # several items to an SM.
    n, lengths = 130, [5 * b for b in range(40)]
    counts = [(30, 130, 64, 129, 1)[b % 5] for b in range(40)]
    pool = held(lengths, n, 8, 64, 128, fmt, seed=6)
    att = ChunkAttention(40, n, 16, 8, 64)
    for _ in range(3):
        run(pool, n, 16, window, sinks, counts=counts, handle=att, rows_of={0, 63, 64, 128, 129})
    assert att.device_status(stream()) == Bd.FLY_OK


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [12, 70])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (5, 3), (5, 300), (300, 40)])
def test_windows_that_end_behind_the_table(fmt, n, window, sinks):
    # what is behind the table does not exist: later rows see less and less of the window, then the first tokens only, or nothing
    full = Pool([304, 304, 304, 304], 0, 2, 64, 16, fmt, seed=n)
    full.lengths = torch.tensor([304, 300, 250, 304 - n], dtype=torch.int32)
    full.refresh()
    run(full, n, 16, window, sinks, rows_of=set(range(0, n, 5)) | {n - 1})


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [3, 40])
def test_every_form_gives_nan_while_a_wait_that_ran_out_is_pending(fmt, dim, n):
    pool = held([700, 20], n, 2, dim, 16, fmt, seed=3)
    att = ChunkAttention(2, n, 16, 2, dim)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = rows(2, n, 16, dim, g)
    out, lse = torch.zeros_like(q), torch.zeros(2, n, 16, device="cuda")
    assert att.selftest_wait(stream()) == Bd.FLY_OK
    for _ in range(2):
        att.run(pool.cache, q, out, lse=lse, stream=stream())
    assert att.device_status(stream()) == Bd.FLY_ERR_TIMEOUT
    assert bool(out.isnan().all()) and bool(lse.isnan().all())
    run(pool, n, 16, handle=att, rows_of={0, n - 1})


# ---- values and sizes at the edges ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,kv_heads,n,dim", [(128, 1, 1, 128), (127, 1, 2, 64), (128, 1, 3, 64), (65, 1, 3, 128), (3, 1, 50, 64), (15, 5, 9, 128), (100, 2, 2, 64)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_groups_of_all_sizes(fmt, heads, kv_heads, n, dim):
    run(held([0, 130, 300], n, kv_heads, dim, 32, fmt, seed=heads), n, heads, seed=n, rows_of={0, n // 2, n - 1})


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lengths", [[500], [511], [512], [513], [480, 0, 100, 505], [300] * 32, [300] * 33, [500] * 80, [600] + [10] * 60])
def test_whole_items_and_cut_ones(fmt, lengths):
    # around four tiles of positions, 32 groups, one item to an SM
    pool = held(lengths, 3, 2, 64, 16, fmt, seed=len(lengths))
    run(pool, 3, 4, rows_of={2})
    run(pool, 3, 4, 200, 20, rows_of={0})


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [5, 50])
@pytest.mark.parametrize("window,sinks", [(10, 5), (40, 60), (3, 130), (200, 1)])
def test_first_tokens_and_window_in_one_tile(fmt, n, window, sinks):
    run(held([0, 20, 90, 100, 126, 140, 250, 270], n, 1, 64, 16, fmt, seed=window), n, 8, window, sinks, rows_of=set(range(0, n, 7)) | {n - 1})


@pytest.mark.parametrize("n", [4, 40])
def test_scales_and_codes_that_append_does_not_write(n):
    # values' scales over the whole range, NaN codes where nobody looks (a page's slots past the end are full of them already)
    pool = held([200, 333], n, 2, 64, 16, "e4m3", seed=3)
    s = pool.v_scales.cpu()
    g = torch.Generator().manual_seed(3)
    live = s != 255
    s[live] = torch.tensor([0, 1, 6, 7, 100, 133, 134, 135, 136, 180, 220], dtype=torch.uint8)[torch.randint(11, (int(live.sum()),), generator=g)]
    pool.v_scales.copy_(s)
    run(pool, n, 8, rows_of={0, n - 1})
    run(pool, n, 8, 50, 20, rows_of={0, n - 1})


def test_e4m3_queries_of_a_wide_range():
    # what is far below the largest value of a query row is kept to 2^-22 of that value
    n = 9
    pool = held([300, 20], n, 2, 64, 16, "e4m3", seed=8)
    g = torch.Generator(device="cuda").manual_seed(8)
    q = rows(2, n, 8, 64, g)
    q *= torch.exp2(torch.randint(-30, 3, q.shape, generator=g, device="cuda").float()).bfloat16()
    q[0, 0] = 0
    q[1, 2] *= 2.0 ** -100
    q[1, 3, 1] = torch.finfo(torch.bfloat16).tiny
    run(pool, n, 8, q=q)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_that_are_not_finite_stay_in_their_rows(fmt, n, bad):
    pool = held([300, 20], n, 2, 64, 16, fmt, seed=8)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = rows(2, n, 8, 64, g)
    _, good, good_lse = run(pool, n, 8, q=q, rows_of={0})
    q = q.clone()
    q[0, 1, 3, 17] = bad
    q[1, n - 1, 0] = bad
    out, lse, att = torch.zeros_like(q), torch.zeros_like(good_lse), ChunkAttention(2, n, 8, 2, 64)
    att.run(pool.cache, q, out, lse=lse, stream=stream())
    hit = torch.zeros(2, n, 8, dtype=torch.bool, device="cuda")
    hit[0, 1, 3] = hit[1, n - 1, 0] = True
    assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(out[~hit], good[~hit]) and torch.equal(lse[~hit], good_lse[~hit])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lengths,n", [([700, 20], 4), ([5000], 3), ([300, 100], 60)])
def test_the_output_may_be_the_queries(fmt, lengths, n):
    pool = held(lengths, n, 2, 64, 16, fmt, seed=4)
    q, want, _ = run(pool, n, 16, 0, 0, rows_of={0})
    both, att = q.clone(), ChunkAttention(len(lengths), n, 16, 2, 64)
    att.run(pool.cache, both, both, stream=stream())
    assert torch.equal(both, want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_past_32_bits(fmt):
    # three pages 2^30 elements (bf16) or 2^31 (e4m3) apart
    n, H, D, page, step = 3, 2, 64, 64, 2 ** (30 if fmt == "bf16" else 31)
    small = held([150], n, H, D, page, fmt, spare=0, seed=7)
    flat = [torch.zeros(2 * step + page * H * D, dtype=small.k_pages.dtype, device="cuda") for _ in "kv"]
    for t, x in zip(flat, (small.k_pages, small.v_pages)):
        big = t.as_strided((3, page, H, D), (step, H * D, D, 1))
        (big.view(torch.uint8) if fmt == "e4m3" else big).copy_(x.view(torch.uint8) if fmt == "e4m3" else x)
    k, v = (t.as_strided((3, page, H, D), (step, H * D, D, 1)) for t in flat)
    small.k_pages, small.v_pages = k, v
    small.cache = PagedCache(k, v, small.d_table, small.d_lengths, small.k_scales, small.v_scales)
    run(small, n, 8)


def test_two_handles_on_two_streams():
    pools = [held([3000, 100], 5, 2, 64, 16, f, seed=3) for f in FORMATS]
    g = torch.Generator(device="cuda").manual_seed(1)
    qs, atts, side = [rows(2, 5, 16, 64, g) for _ in pools], [ChunkAttention(2, 5, 16, 2, 64) for _ in pools], [torch.cuda.Stream() for _ in pools]
    outs, lses = [[torch.zeros_like(qs[0]) for _ in range(20)] for _ in pools], [torch.zeros(2, 5, 16, device="cuda") for _ in pools]
    torch.cuda.synchronize()
    for i in range(20):
        for k in range(2):
            atts[k].run(pools[k].cache, qs[k], outs[k][i], lse=lses[k], stream=side[k].cuda_stream)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, outs[k][0]) for o in outs[k])
        check_attention(pools[k], qs[k], outs[k][0], lses[k], rows_of={0, 4})


def test_tables_of_too_many_tiles_are_refused():
    # 2^30 positions in each of 200 sequences: more tiles than the schedule counts
    pages = torch.zeros(1, 65536, 2, 64, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(200, 16384, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(200, dtype=torch.int32, device="cuda")
    cache = PagedCache(pages, pages, table, lengths)
    q = torch.zeros(200, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    att = ChunkAttention(200, 1, 2, 2, 64)
    with pytest.raises(Bd.FlyError) as e:
        att.run(cache, q, torch.zeros_like(q), stream=stream())
    assert e.value.status == Bd.FLY_ERR_UNSUPPORTED
    for bad in (q[:, :, :1].expand(200, 1, 2, 64), q[:1].expand(200, 1, 2, 64)):     # an output of which several rows are one
        with pytest.raises(Bd.FlyError) as e:
            att.run(cache, q, bad, stream=stream())
        assert e.value.status == Bd.FLY_ERR_UNSUPPORTED


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scale", [2.0 ** 16, 2.0 ** 20, 2.0 ** 22])
def test_scores_whose_ulps_are_large(fmt, scale):
    # (up to 2^30, beyond which the header promises nothing)
    for n, heads in ((9, 4), (70, 4)):
        pool = held([300, 20], n, 1, 64, 16, fmt, seed=8)
        run(pool, n, heads, scale=scale, rows_of={0, n - 1})
        run(pool, n, heads, 50, 3, scale=scale, rows_of={0, n - 1})


def test_pointers_off_their_alignment_are_refused():
    import ctypes as C
    from paper_2511_22972_b200 import cache as M
    pool = held([10, 20], 4, 2, 64)
    att, g = ChunkAttention(2, 4, 8, 2, 64), torch.Generator(device="cuda").manual_seed(8)
    q, lse = rows(2, 4, 8, 64, g), torch.zeros(2 * 4 * 8 + 1, device="cuda")
    r = M.fly_rows_t(q.data_ptr(), *q.stride()[:3])
    for counts, at, want in ((None, 0, Bd.FLY_OK), (None, 2, Bd.FLY_ERR_UNSUPPORTED), (pool.d_lengths.data_ptr() + 1, 0, Bd.FLY_ERR_UNSUPPORTED)):
        a = M.fly_attention_args_t(2, 4, r, r, lse.data_ptr() + at, counts, 0, 0, 0.0)
        assert M.lib().fly_attention_run(att._h, C.byref(pool.cache.struct), C.byref(a), C.c_void_p(stream())) == want
    torch.cuda.synchronize()
