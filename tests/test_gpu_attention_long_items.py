"""Contexts so long that one item keeps a block busy for longer than a wait's limit (200 ms), while other warps wait for its end."""
import math

import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, PagedCache, binding as Bd
from tests.test_gpu_attention import stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,counts", [(16, (16, 16)), (16, (4, 16)), (8, (8, 8))])
def test_waits_for_the_end_of_a_long_item_do_not_run_out(fmt, n, counts):
    # 16 heads to one key/value head: eight tokens to a row tile.  (16, 16): pairs whose next queries come when the item ends.  (4, 16): the second
    # tile of every other pair has no rows.  (8, 8): single row tiles.  160 items for 148 SMs or fewer: blocks go on to a second one.
    # All positions are on one page of 65536, so 32 million of them take 8 MB.
    B, heads, D, page, L = 160, 16, 64, 65536, 32_000_000
    kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
    signs = torch.tensor([1.0, -1.0], device="cuda").repeat(D // 2) * torch.exp2(torch.arange(D, device="cuda") % 5)
    k = torch.zeros(1, page, 1, D, device="cuda").to(kind)
    v = signs.expand(1, page, 1, D).contiguous().to(kind)
    scales = [torch.full((1, 1, page), 127, dtype=torch.uint8, device="cuda") for _ in "kv"] if fmt == "e4m3" else []
    table = torch.zeros(B, -(-(L + n) // page), dtype=torch.int32, device="cuda")
    cache = PagedCache(k, v, table, torch.full((B,), L, dtype=torch.int32, device="cuda"), *scales)
    held = torch.tensor([counts[b % 2] for b in range(B)], dtype=torch.int32, device="cuda")
    q = torch.zeros(B, n, heads, D, dtype=torch.bfloat16, device="cuda")
    out, lse, att = torch.full_like(q, 7.0), torch.full((B, n, heads), 7.0, device="cuda"), ChunkAttention(B, n, heads, 1, D)
    att.run(cache, q, out, counts=held, lse=lse, stream=stream())
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    att.run(cache, q, out, counts=held, lse=lse, stream=stream())
    end.record()
    assert att.device_status(stream()) == Bd.FLY_OK
    assert begin.elapsed_time(end) > 230                       # (else the case would not show anything)
    live = torch.arange(n, device="cuda") < held[:, None]
    assert bool((out[~live] == 7).all()) and bool((lse[~live] == 7).all())
    # Scores are 0: every weight is 1, and sums of weights are exact in fp32 up to the last tile.  (Sums of weighted values are not: so
    # many equal terms may each lose what the sum has no place for.  They only have to be of the right sign and not too large.)
    want = torch.log(L + 1.0 + torch.arange(n, device="cuda", dtype=torch.float64))
    assert bool(((lse.double() - want[None, :, None])[live].abs() <= 2.0 ** -22 * math.log(L) + 2.0 ** -20).all())
    ratio = out[live].float() / signs
    print(fmt, n, counts, begin.elapsed_time(end), float(ratio.min()), float(ratio.max()))
    assert bool((ratio > 0).all()) and bool((ratio <= 1 + 2.0 ** -7).all())
