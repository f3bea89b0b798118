"""Rounds of speculative decoding with all of it in one stream: drafts by prompt lookup, the chunk's keys and values into the cache,
its queries over the cache, the LM head with the verification, and the cache's lengths moved on by what was kept."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO, fly_oracle as O
from paper_2511_22972_b200 import (ChunkAttention, FlyVerify, PagedCache, VerifyBuffers, binding as Bd, cache_append, cache_read,
                                   verify_fused)
from tests._cache import Pool, check_attention

pytestmark = pytest.mark.gpu
VOCAB, HEADS, KV, DIM, K, B, PAGE = 512, 8, 2, 64, 5, 4, 16
WIDTH = HEADS * DIM


class Layer:
    """One attention layer and an LM head: q, k, v are products of the tokens' embeddings, the hidden state is what attention gives."""

    def __init__(self, fmt):
        g = torch.Generator(device="cuda").manual_seed(5)
        mat = lambda *s: (torch.randn(*s, generator=g, device="cuda") / np.sqrt(s[0])).bfloat16()  # noqa: E731
        self.embed, self.q, self.kv, self.head = mat(VOCAB, 256) * 22, mat(256, WIDTH) * 2, mat(256, 2 * KV * DIM), mat(WIDTH, VOCAB) * 24

    def rows(self, tokens):
        x = self.embed[tokens.long()]
        kv = (x @ self.kv).view(*tokens.shape, 2, KV, DIM)
        return (x @ self.q).view(*tokens.shape, HEADS, DIM), kv[..., 0, :, :], kv[..., 1, :, :]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_rounds(fmt, window, sinks):
    layer, pool = Layer(fmt), Pool([0] * B, 256, KV, DIM, PAGE, fmt, seed=1)
    st = torch.cuda.current_stream().cuda_stream
    prompts = [[(7 * i + b) % 13 for i in range(20 + 11 * b)] for b in range(B)]       # they repeat: lookup finds drafts
    width = 256
    tokens = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    for b, t in enumerate(prompts):
        tokens[b, :len(t)] = torch.tensor(t, dtype=torch.int32)
    held = torch.tensor([len(t) for t in prompts], dtype=torch.int32, device="cuda")   # tokens so far; the last one's keys come with the round
    n0 = max(len(t) for t in prompts)
    attention = ChunkAttention(B, max(n0, K + 1), HEADS, KV, DIM)
    fv, buffers = FlyVerify(B, K, VOCAB, "bf16", hidden=WIDTH), VerifyBuffers(B, K, "cuda")
    cache, lengths = pool.cache, pool.d_lengths
    # the prompts but for their last tokens, in one chunk of ragged rows
    q, k, v = layer.rows(tokens[:, :n0])
    counts = held - 1
    cache_append(cache, k, v, counts=counts, stream=st)
    out = torch.zeros(B, n0, HEADS, DIM, dtype=torch.bfloat16, device="cuda")
    attention.run(cache, q, out, window=window, sinks=sinks, counts=counts, stream=st)
    lengths.add_(counts)
    kept = [[(k[b, i].clone(), v[b, i].clone()) for i in range(len(t) - 1)] for b, t in enumerate(prompts)]
    for _ in range(6):
        draft, count, _, _ = Bd.pld_draft(tokens, held, K, 3, 1, stream=st)
        last = tokens.gather(1, (held - 1).long().unsqueeze(1))
        chunk = torch.cat([last, draft.clamp(min=0)], 1)
        q, k, v = layer.rows(chunk)
        cache_append(cache, k, v, stream=st)
        out, lse = torch.zeros(B, K + 1, HEADS, DIM, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, K + 1, HEADS, device="cuda")
        attention.run(cache, q, out, window=window, sinks=sinks, lse=lse, stream=st)
        hidden = out.view(B * (K + 1), WIDTH)
        verify_fused(fv, hidden, layer.head, draft, buffers, theta=0.5, W=2, boundary="reject", stream=st)
        # ... against the definitions, from what the round itself produced
        torch.cuda.synchronize()
        pool.lengths = lengths.cpu()
        check_attention(pool, q, out, lse, window, sinks)
        logits = O.lm_head_logits(hidden.cpu().double().numpy(), layer.head.cpu().double().numpy())
        ref = O.verify_batch(logits.reshape(B, K + 1, VOCAB), draft.cpu().numpy(), 0.5, 2, boundary="reject")
        near = np.sort(logits, 1)
        for b in range(B):                                    # (a draw of the two largest logits may go either way)
            if (near[b * (K + 1):(b + 1) * (K + 1), -1] - near[b * (K + 1):(b + 1) * (K + 1), -2]).min() > 1e-2:
                s = int(buffers.accept_len[b])
                assert s == int(ref.accept_len[b]) and buffers.out_tokens[b, :s].tolist() == list(ref.out_tokens[b][:s])
        # what is kept: accept_len tokens, whose keys (but for the newest token's) are in the cache
        for b in range(B):
            s = int(buffers.accept_len[b])
            tokens[b, int(held[b]):int(held[b]) + s] = buffers.out_tokens[b, :s]
            kept[b] += [(k[b, i].clone(), v[b, i].clone()) for i in range(s - int(buffers.rollback[b]))]
        held.add_(buffers.accept_len).sub_(buffers.rollback)
        lengths.add_(buffers.accept_len).sub_(buffers.rollback)
        assert torch.equal(lengths, held - 1)
    # the cache holds the rows of the tokens that were kept, in order, and of no draft that was not
    m = int(lengths.max())
    k_out, v_out = (torch.zeros(B, m, KV, DIM, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    cache_read(cache, k_out, v_out, stream=st)
    torch.cuda.synchronize()
    for b in range(B):
        assert len(kept[b]) == int(lengths[b])
        for p, row in enumerate(kept[b]):
            for x, y in zip(row, (k_out, v_out)):
                want = x.float().cpu().double().numpy()
                if fmt == "e4m3":
                    want = np.stack([CO.row_values(*CO.quantise_row(r)) for r in want])
                assert (y[b, p].float().cpu().double().numpy() == want).all(), (b, p)
