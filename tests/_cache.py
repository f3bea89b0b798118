"""Helpers of the cache tests: a pool of pages with a chosen layout, the same contents in fp64, and the oracle over it."""
import math

import numpy as np
import torch

from oracle import cache_oracle as O
from paper_2511_22972_b200 import PagedCache

HALF = torch.finfo(torch.bfloat16).eps / 2


class Pool:
    """A cache of `lengths` random positions per sequence; layout: 'nhd', 'hnd' (heads before tokens) or 'pair' (keys and values of
    a page side by side).  Pages are dealt in random order; slots that nobody holds are full of NaN."""

    def __init__(self, lengths, n, kv_heads, dim, page=16, fmt="bf16", layout="nhd", seed=0, device="cuda", spare=3, std=1.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.n, self.H, self.D, self.page, self.fmt = len(lengths), n, kv_heads, dim, page, fmt
        width = max(1, -(-(max(lengths) + n) // page))
        total = self.B * width + spare
        self.table = torch.randperm(total, generator=g)[:self.B * width].view(self.B, width).int()
        self.lengths = torch.tensor(lengths, dtype=torch.int32)
        dtype = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn

        def pages(k):
            if layout == "hnd":
                return torch.empty(total, kv_heads, page, dim, dtype=dtype).transpose(1, 2)
            if layout == "pair":
                return both[:, k]
            return torch.empty(total, page, kv_heads, dim, dtype=dtype)
        both = torch.empty(total, 2, page, kv_heads, dim, dtype=dtype) if layout == "pair" else None
        self.k_pages, self.v_pages = pages(0), pages(1)
        x = torch.randn(2, total, page, kv_heads, dim, generator=g) * std
        x[0] += torch.randn(kv_heads, dim, generator=g)
        x = x.bfloat16()
        live = torch.zeros(total, page, dtype=torch.bool)
        for b, L in enumerate(lengths):
            for p in range(min(max(L, 0), width * page)):
                live[self.table[b, p // page].long(), p % page] = True
        self.k_scales = self.v_scales = None
        if fmt == "bf16":
            x[:, ~live] = float("nan")
            self.k_pages.copy_(x[0])
            self.v_pages.copy_(x[1])
        else:
            m, e = torch.frexp(x.float().abs().amax(-1))
            e = torch.where(m > 0.875, e - 8, e - 9)
            codes = torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn)
            codes.view(torch.uint8)[:, ~live] = 0x7f
            scales = (e + 127).to(torch.uint8).transpose(2, 3).contiguous()
            scales.transpose(2, 3)[:, ~live] = 255
            self.k_pages.view(torch.uint8).copy_(codes[0].view(torch.uint8))
            self.v_pages.view(torch.uint8).copy_(codes[1].view(torch.uint8))
            self.k_scales, self.v_scales = scales[0].contiguous(), scales[1].contiguous()
        if device != "cpu":
            self.to(device, both)

    def to(self, device, both):
        if both is not None:
            both = both.to(device)
            self.k_pages, self.v_pages = both[:, 0], both[:, 1]
        else:
            k, v = self.k_pages.to(device), self.v_pages.to(device)   # (strides of a transposed tensor are kept)
            assert k.stride() == self.k_pages.stride()
            self.k_pages, self.v_pages = k, v
        self.d_table, self.d_lengths = self.table.to(device), self.lengths.to(device)
        if self.fmt == "e4m3":
            self.k_scales, self.v_scales = self.k_scales.to(device), self.v_scales.to(device)
        self.cache = PagedCache(self.k_pages, self.v_pages, self.d_table, self.d_lengths, self.k_scales, self.v_scales)

    def refresh(self):
        """The table and lengths as the host copies are now."""
        self.d_table.copy_(self.table)
        self.d_lengths.copy_(self.lengths)

    def values(self):
        """All pages in fp64: [2, total, page, H, D] (numpy)."""
        out = []
        for pages, scales in ((self.k_pages, self.k_scales), (self.v_pages, self.v_scales)):
            x = pages.float().cpu().double()
            if scales is not None:
                s = scales.cpu().transpose(1, 2).double()
                x = torch.where((s == 255)[..., None], torch.full_like(x, float("nan")), x * torch.exp2(s - 127)[..., None])
            out.append(x.numpy())
        return out

    def sequence(self, vals, b, upto):
        """Keys and values of positions 0 .. upto - 1 and which of them exist."""
        k, v = np.zeros((upto, self.H, self.D)), np.zeros((upto, self.H, self.D))
        there = np.zeros(upto, dtype=bool)
        for p in range(upto):
            at = O.place(self.table[b].tolist(), p, self.page, vals[0].shape[0])
            if at is not None:
                k[p], v[p], there[p] = vals[0][at], vals[1][at], True
        return k, v, there


def rows(B, n, heads, dim, g, strided=False, std=1.0):
    """bf16 [B, n, heads, dim] on the GPU; strided: a slice of a wider tensor, as of a fused projection's output."""
    if strided:
        return (torch.randn(B, n, heads + 5, dim, generator=g, device="cuda") * std).bfloat16()[:, :, 2:2 + heads]
    return (torch.randn(B, n, heads, dim, generator=g, device="cuda") * std).bfloat16()


def check_attention(pool, q, out, lse, window=0, sinks=0, scale=0.0, counts=None, untouched=None, rows_of=None):
    """out and lse against the oracle.  The tolerance, all in units of what the formula sums: a weight is rounded to bf16 before it
    meets its value (2^-8 of it), the result once more (2^-8 of it); a score is a sum of D products in fp32 (D * 2^-23 of the sum of
    their magnitudes, which shifts a weight by as much) and its exponential is good to 2^-21; sums over P positions in fp32 are off
    by at most P * 2^-24 of the sum of magnitudes."""
    scale = scale or 1 / math.sqrt(pool.D)
    vals = pool.values()
    B, n, heads, D = q.shape
    G = heads // pool.H
    qd, od = q.float().cpu().double().numpy(), out.float().cpu().double().numpy()
    ld = None if lse is None else lse.cpu().double().numpy()
    for b in range(B):
        L = O.held_length(int(pool.lengths[b]), pool.table[b].tolist(), pool.page)
        m = O.held_count(counts, b, n)
        k, v, there = pool.sequence(vals, b, max(0, L + m))
        for i in range(n):
            if i >= m:
                if untouched is not None:
                    assert torch.equal(out[b, i].cpu(), untouched[0][b, i].cpu()), ("written", b, i)
                    assert ld is None or torch.equal(lse[b, i].cpu(), untouched[1][b, i].cpu()), ("written", b, i)
                continue
            if rows_of is not None and i not in rows_of:
                continue
            see = np.array([p for p in O.visible(L + i, window, sinks) if there[p]] if L >= 0 else [], dtype=int)
            for h in range(heads):
                kk, vv = k[see, h // G], v[see, h // G]
                want, want_lse = O.attend_row(qd[b, i, h], kk, vv, scale)
                if not np.isfinite(want_lse) or not np.isfinite(want).all():
                    assert want_lse == -math.inf and not want.any()
                    assert not od[b, i, h].any() and (ld is None or ld[b, i, h] == -math.inf), (b, i, h, od[b, i, h][:4])
                    continue
                reach = scale * (np.abs(kk) @ np.abs(qd[b, i, h])).max()
                d = D * 2.0 ** -23 * reach + 2.0 ** -21 + len(see) * 2.0 ** -24
                size, _ = O.attend_row(qd[b, i, h], kk, np.abs(vv), scale)
                tol = size * (HALF + 2 * d) + np.abs(want) * HALF
                err = np.abs(od[b, i, h] - want)
                assert (err <= tol).all(), (b, i, h, float((err / tol).max()), len(see))
                if ld is not None:
                    assert abs(ld[b, i, h] - want_lse) <= 2 * d + abs(want_lse) * 2.0 ** -22, (b, i, h, ld[b, i, h], want_lse)
