"""Attention of a chunk over a paged cache against the fp64 oracle."""
import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, binding as Bd
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
