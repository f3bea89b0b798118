"""Timing cases of the operators on a paged key/value cache, with their plain forms.

A round of speculative decoding runs a chunk of n = K+1 new tokens per sequence through the target: their keys and values
are appended to a paged cache (as bf16, or quantised to e4m3 as they are written), the chunk attends to everything that is
visible to it there, and the cache is now and then read back (to move a sequence, or for code that wants plain tensors).

  append   positions lengths[b] + i of sequence b take the chunk's keys and values
  read     positions starts[b] + i come back as bf16
  attend   row i of the chunk sees positions 0 .. lengths[b] + i
  window   the same with a sliding window: the last `window` of them and the first `sinks` positions

An e4m3 row (one token of one head, `dim` values) is held as codes c and one byte s: value = c * 2^(s - 127), with the
smallest s >= 7 for which no code exceeds 448.
"""
import math

import torch

own = False

HEADS = [(64, 8, 128), (32, 8, 128), (128, 8, 128), (28, 4, 128), (40, 8, 128), (8, 8, 64), (12, 2, 64), (16, 1, 128),
         (14, 2, 64), (8, 8, 128)]


def _case(name, op, fmt, B, n, lo, hi, page=16, heads=64, kv_heads=8, dim=128, window=0, sinks=0, ragged=False):
    return dict(name=name, op=op, fmt=fmt, B=B, n=n, lo=lo, hi=hi, page=page, heads=heads, kv_heads=kv_heads, dim=dim,
                window=window, sinks=sinks, ragged=ragged)


def listed():
    return [
        # One sequence's 15 drafts and the token before them: the paper's setting for one user.  Latency.
        _case("append_one_sequence", "append", "e4m3", 1, 16, 1000, 1000),
        # A serving batch of 256 sequences with 8 drafts each, some of them with fewer.
        _case("append_round", "append", "e4m3", 256, 9, 100, 1000, ragged=True),
        # Prompts of three sequences, written in one go behind what is there.
        _case("append_prompt", "append", "e4m3", 3, 4099, 0, 50, page=64),
        # One short context read back.  Latency.
        _case("read_short", "read", "e4m3", 1, 1003, 1003, 1003),
        # Eight contexts read back, as to move them to another cache.
        _case("read_batch", "read", "e4m3", 8, 16000, 4000, 16000, page=32),
        # A short context and one round of 8 drafts for one user.  Latency.
        _case("attend_short", "attend", "bf16", 1, 9, 300, 300),
        # The paper's setting for one user (K = 15) over a long context.
        _case("attend_one_sequence", "attend", "bf16", 1, 16, 30000, 30000),
        # A serving batch without drafts: one token per sequence.
        _case("attend_token", "attend", "bf16", 64, 1, 500, 8000),
        # A serving batch with 8 drafts per sequence over a quantised cache.
        _case("attend_round_e4m3", "attend", "e4m3", 16, 9, 2000, 16000),
        # Chunks of two prompts behind what is in the cache already.
        _case("attend_prompt", "attend", "bf16", 2, 2000, 4000, 8000, page=64),
        # A drafter that reads very long quantised contexts through a window and the first tokens.
        _case("window_token", "window", "e4m3", 4, 1, 90000, 100000, window=4096, sinks=4),
        # A model with windowed attention in a serving batch with 8 drafts, small heads in an odd group.
        _case("window_round", "window", "bf16", 48, 9, 1000, 32000, page=64, heads=28, kv_heads=4, dim=64, window=2048, sinks=100,
              ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "read", "attend", "attend", "window", "window"])
        heads, kv_heads, dim = rng.choice(HEADS)
        c = dict(op=op, fmt=rng.choice(["bf16", "e4m3"]), page=rng.choice([8, 16, 32, 64, 128, 256]), heads=heads, kv_heads=kv_heads,
                 dim=dim, window=0, sinks=0, ragged=rng.random() < 0.5)
        if op == "append":
            c["B"] = _log(rng, 1, 256)
            c["n"] = _log(rng, 1, max(1, 12000 // c["B"]))
            c["lo"] = rng.randint(0, 500)
            c["hi"] = c["lo"] + rng.randint(0, 500)
        elif op == "read":
            c["B"] = _log(rng, 1, 64)
            c["hi"] = _log(rng, 1, 16000)
            c["lo"] = rng.randint(0, c["hi"])
            c["n"] = c["hi"]
            c["ragged"] = False
        else:
            c["B"] = _log(rng, 1, 64)
            c["n"] = rng.choice([1, rng.randint(2, 64), rng.randint(2, 64), _log(rng, 65, 2000)])
            c["hi"] = _log(rng, 1, 100000)
            c["lo"] = rng.randint(0, c["hi"])
            if op == "window":
                c["window"] = _log(rng, 1, 8192)
                c["sinks"] = rng.choice([0, 1, 4, rng.randint(5, 300)])
        tokens = c["B"] * (c["hi"] + c["n"])  # of the cache
        seen = c["B"] * c["n"] * (_span(c) if op in ("attend", "window") else 1)
        if tokens * kv_heads * dim <= 280e6 and seen * heads <= 2.5e9:
            return c


def _lengths(c):
    """The sequences' lengths before the call: spread evenly over lo .. hi.  In what order they come goes by the seed."""
    return [c["lo"] + (c["hi"] - c["lo"]) * i // max(1, c["B"] - 1) for i in range(c["B"])] if c["B"] > 1 else [c["hi"]]


def _counts(c):
    """Tokens of the chunk that each sequence really has."""
    return [1 + (7 * i + c["n"] - 1) % c["n"] if c["ragged"] else c["n"] for i in range(c["B"])]


def _span(c):
    """Positions that the rows of a chunk can see together, at most."""
    return min(c["hi"] + c["n"], c["sinks"] + c["window"] + c["n"] - 1) if c["window"] else c["hi"] + c["n"]


def work(case):
    c = case
    lens, counts = _lengths(c), _counts(c)
    row = c["kv_heads"] * c["dim"] * 2                     # values of a token in the cache, keys and values
    held = row * 2 if c["fmt"] == "bf16" else row + 2 * c["kv_heads"]
    if c["op"] == "append":
        t = sum(counts)
        return dict(bytes=t * (row * 2 + held), flops=0)
    if c["op"] == "read":
        t = sum(lens)
        return dict(bytes=t * (row * 2 + held), flops=0)
    tokens = pairs = 0
    for L, m in zip(lens, counts):
        w, s = c["window"] or L + m, c["sinks"]
        first = max(0, L - w + 1)                          # the lowest position in the first row's window
        tokens += L + m - first + min(s, first)
        low = [max(0, L + i - w + 1) for i in range(m)]
        pairs += sum(L + i + 1 - a + min(s, a) for i, a in enumerate(low))
    q = sum(counts) * c["heads"] * c["dim"]
    return dict(bytes=tokens * held + q * 4 + sum(counts) * c["heads"] * 4, flops=4 * pairs * c["heads"] * c["dim"])


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _quantise(x):
    """Codes and scale bytes of rows x [..., dim] (fp32)."""
    m, k = torch.frexp(x.abs().amax(-1))                   # amax = m * 2^k with 0.5 <= m < 1, and 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, k - 8, k - 9)
    e = torch.where(m == 0, torch.full_like(e, -120), e).clamp(min=-120)
    codes = torch.ldexp(x, -e.unsqueeze(-1)).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def _values(pages, scales, page, slot):
    """The rows [..., kv_heads, dim] of tokens at `slot` of `page`, in fp32."""
    x = pages[page, slot].float()
    if scales is None:
        return x
    return torch.ldexp(x, scales[page, :, slot].unsqueeze(-1).int() - 127)


def _where(s, pos):
    """Page and slot of positions pos [B, P] (clamped to the table)."""
    size = s["case"]["page"]
    at = (pos // size).clamp(0, s["table"].shape[1] - 1)
    return s["table"].gather(1, at).long(), pos % size


def _append(s):
    c = s["case"]
    i = torch.arange(c["n"], device="cuda")
    page, slot = _where(s, s["lengths"].unsqueeze(1) + i)
    live = i < s["counts"].unsqueeze(1)
    page, slot = page[live], slot[live]
    for x, pages, scales in ((s["k"], s["k_pages"], s["k_scales"]), (s["v"], s["v_pages"], s["v_scales"])):
        x = x[live]
        if scales is None:
            pages[page, slot] = x
        else:
            codes, e = _quantise(x.float())
            pages.view(torch.uint8)[page, slot] = codes.view(torch.uint8)
            scales.transpose(1, 2)[page, slot] = e
    return _pages(s)


def _pages(s):
    return [t for t in (s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]) if t is not None]


def _read(s):
    c = s["case"]
    pos = torch.arange(c["n"], device="cuda").expand(c["B"], -1)
    page, slot = _where(s, pos)
    live = (pos < s["lengths"].unsqueeze(1))[..., None, None]
    for out, pages, scales in ((s["k_out"], s["k_pages"], s["k_scales"]), (s["v_out"], s["v_pages"], s["v_scales"])):
        out.copy_(torch.where(live, _values(pages, scales, page, slot).bfloat16(), out))
    return s["k_out"], s["v_out"]


def _attend(s):
    c = s["case"]
    B, n, G, D = c["B"], c["n"], c["heads"] // c["kv_heads"], c["dim"]
    L = s["lengths"].long().unsqueeze(1)
    if c["window"]:                                        # the first tokens, and everything from the first row's window on
        first = (L - c["window"] + 1).clamp(min=0)
        a, b = torch.arange(c["sinks"], device="cuda").expand(B, -1), first + torch.arange(c["window"] + n - 1, device="cuda")
        pos, once = torch.cat([a, b], 1), torch.cat([a < first, b >= 0], 1)
    else:
        pos = torch.arange(c["hi"] + n, device="cuda").expand(B, -1)
        once = pos >= 0
    page, slot = _where(s, pos)
    k = _values(s["k_pages"], s["k_scales"], page, slot).transpose(1, 2)      # [B, kv_heads, P, D]
    v = _values(s["v_pages"], s["v_scales"], page, slot).transpose(1, 2)
    q = s["q"].float().view(B, n, -1, G, D).permute(0, 2, 1, 3, 4).reshape(B, -1, n * G, D)
    score = torch.matmul(q, k.transpose(2, 3)).view(B, -1, n, G, pos.shape[1]) * (1 / math.sqrt(D))
    at = L + torch.arange(n, device="cuda")                # a row's own position
    seen = (pos.unsqueeze(1) <= at.unsqueeze(2)) & once.unsqueeze(1)
    if c["window"]:
        seen &= (pos.unsqueeze(1) > at.unsqueeze(2) - c["window"]) | (pos < c["sinks"]).unsqueeze(1)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, -1, n * G, pos.shape[1]), v).view(B, -1, n, G, D) / total
    lse = (total.log() + top).squeeze(-1)
    live = torch.arange(n, device="cuda") < s["counts"].unsqueeze(1)
    s["out"].copy_(torch.where(live[..., None, None], o.permute(0, 2, 1, 3, 4).reshape(B, n, -1, D).bfloat16(), s["out"]))
    s["lse"].copy_(torch.where(live[..., None], lse.permute(0, 2, 1, 3).reshape(B, n, -1), s["lse"]))
    return s["out"], s["lse"]


# ---- the interface -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed)
    order = torch.randperm(c["B"], generator=h)
    lens, counts = torch.tensor(_lengths(c))[order], torch.tensor(_counts(c))
    width = -(-(c["hi"] + c["n"]) // c["page"])
    used = -(-(lens + c["n"]) // c["page"])                # pages of each sequence, in no order in the pool
    total = int(used.sum()) + 1
    pool = torch.randperm(total, generator=h).int()
    table = torch.zeros(c["B"], width, dtype=torch.int32)
    table[torch.arange(width) < used.unsqueeze(1)] = pool[:total - 1]
    i32 = lambda t: t.to("cuda", torch.int32)  # noqa: E731
    s = dict(case=c, lengths=i32(lens), counts=i32(counts), table=i32(table), k_scales=None, v_scales=None)
    shape = (total, c["page"], c["kv_heads"], c["dim"])
    bias = torch.randn(c["kv_heads"], c["dim"], generator=g, device="cuda")   # keys have channels of their own size

    def rows(shape, keys):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
        return x + bias.bfloat16() if keys else x

    for name in ("k", "v"):
        if c["op"] == "append":
            s[name] = rows((c["B"], c["n"], c["kv_heads"], c["dim"]), name == "k")
            pages = torch.zeros(shape, device="cuda", dtype=torch.bfloat16 if c["fmt"] == "bf16" else torch.float8_e4m3fn)
            scales = torch.full((total, c["kv_heads"], c["page"]), 127, dtype=torch.uint8, device="cuda")
        else:
            pages = rows(shape, name == "k")
            if c["fmt"] == "e4m3":
                pages, scales = _quantise(pages.float())
                scales = scales.transpose(1, 2).contiguous()
        s[name + "_pages"] = pages
        if c["fmt"] == "e4m3":
            s[name + "_scales"] = scales
    if c["op"] == "read":
        s["k_out"], s["v_out"] = (torch.zeros(c["B"], c["n"], c["kv_heads"], c["dim"], device="cuda", dtype=torch.bfloat16) for _ in "kv")
    if c["op"] in ("attend", "window"):
        s["q"] = 2 * torch.randn(c["B"], c["n"], c["heads"], c["dim"], generator=g, device="cuda", dtype=torch.bfloat16)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(c["B"], c["n"], c["heads"], device="cuda")
    if own:
        from paper_2511_22972_b200 import ChunkAttention, PagedCache
        s["cache"] = PagedCache(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["k_scales"], s["v_scales"])
        if c["op"] in ("attend", "window"):
            s["attention"] = ChunkAttention(c["B"], c["n"], c["heads"], c["kv_heads"], c["dim"])
    return s


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _append, "read": _read, "attend": _attend, "window": _attend}[c["op"]](s)
    from paper_2511_22972_b200 import cache_append, cache_read
    stream = torch.cuda.current_stream().cuda_stream
    counts = s["counts"] if c["ragged"] else None
    if c["op"] == "append":
        cache_append(s["cache"], s["k"], s["v"], counts=counts, stream=stream)
        return _pages(s)
    if c["op"] == "read":
        cache_read(s["cache"], s["k_out"], s["v_out"], stream=stream)
        return s["k_out"], s["v_out"]
    s["attention"].run(s["cache"], s["q"], s["out"], window=c["window"], sinks=c["sinks"], counts=counts, lse=s["lse"], stream=stream)
    return s["out"], s["lse"]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    lens, counts = s["lengths"].tolist(), s["counts"].tolist()

    def held(which, b, pos):
        """Rows [P, kv_heads, dim] of a sequence's positions, in 64 bits."""
        t, slot = s["table"][b, pos // c["page"]].long(), pos % c["page"]
        x = s[which + "_pages"][t, slot].double()
        return x if c["fmt"] == "bf16" else x * torch.exp2(s[which + "_scales"][t, :, slot].double() - 127)[..., None]

    if c["op"] == "append":
        for which in "kv":
            pages, scales = s[which + "_pages"], s[which + "_scales"]
            for b in range(c["B"]):
                pos = lens[b] + torch.arange(counts[b], device="cuda")
                t, slot = s["table"][b, pos // c["page"]].long(), pos % c["page"]
                x = s[which][b, :counts[b]].double()
                if c["fmt"] == "bf16":
                    pages[t, slot] = x.bfloat16()
                    continue
                top = x.abs().amax(-1)
                e = torch.ceil(torch.log2(top / 448)).clamp(min=-120)      # (the logarithm of a power of two may be a bit off)
                e = torch.where(top > 448 * torch.exp2(e), e + 1, torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)).clamp(min=-120)
                y = x / torch.exp2(e)[..., None]
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)   # distance of neighbouring codes
                pages.view(torch.uint8)[t, slot] = (torch.round(y / step) * step).to(torch.float8_e4m3fn).view(torch.uint8)
                scales.transpose(1, 2)[t, slot] = (e + 127).to(torch.uint8)
        return [t.double() if t.dtype != torch.uint8 else t for t in _pages(s)]
    if c["op"] == "read":
        k, v = s["k_out"].double(), s["v_out"].double()
        for b in range(c["B"]):
            pos = torch.arange(min(c["n"], lens[b]), device="cuda")
            k[b, :len(pos)], v[b, :len(pos)] = held("k", b, pos), held("v", b, pos)
        return k, v
    out, lse = s["out"].double(), s["lse"].double()
    G = c["heads"] // c["kv_heads"]
    for b in range(c["B"]):
        m, L = counts[b], lens[b]
        w = c["window"] or L + m
        first = max(0, L + 1 - w)
        pos = torch.cat([torch.arange(min(c["sinks"], first)), torch.arange(first, L + m)]).cuda()
        k, v = held("k", b, pos), held("v", b, pos)
        own_pos = (L + torch.arange(m, device="cuda")).repeat_interleave(G)[:, None]
        seen = (pos <= own_pos) & ((own_pos - pos < w) | (pos < c["sinks"]))
        for j in range(c["kv_heads"]):
            x = s["q"][b, :m, j * G:(j + 1) * G].double().reshape(m * G, -1) @ k[:, j].T / math.sqrt(c["dim"])
            x = torch.where(seen, x, -math.inf)
            lse[b, :m, j * G:(j + 1) * G] = torch.logsumexp(x, 1).view(m, G)
            out[b, :m, j * G:(j + 1) * G] = (torch.softmax(x, 1) @ v[:, j]).view(m, G, -1)
    return out, lse
