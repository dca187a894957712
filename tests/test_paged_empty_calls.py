"""Calls of the paged cache on no sequences or no tokens: every entry point returns an empty result, on any device."""
import torch

from paper_2407_12820_amd import paged


def test_every_call_takes_nothing():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = paged.PagedCache(k, k.clone(), None, None, n_q_heads=4)
    table, lengths = torch.zeros((0, 3), dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    q, x, idx = torch.zeros((0, 4, 64), dtype=torch.bfloat16), torch.zeros((0, 2, 64), dtype=torch.bfloat16), torch.zeros((0, 2, 5), dtype=torch.int32)
    assert cache.append(x, x, table, lengths) is None
    assert cache.append(x, x, table, lengths, q=q).shape == (0, 4, 64)
    for got in (cache.attn(q, table, lengths), cache.gather_attn(q, idx, table, lengths)):
        assert got.shape == (0, 4, 64) and got.dtype is torch.float32
    out = torch.zeros((0, 4, 64))
    assert cache.attn(q, table, lengths, out=out) is out and cache.gather_attn(q, idx, table, lengths, out=out) is out
    # sequences, but no tokens for them
    off = torch.zeros(3, dtype=torch.int32)
    table, lengths = torch.zeros((2, 3), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    assert cache.append(x, x, table, lengths, new_offsets=off) is None
    assert cache.attn(q, table, lengths, q_offsets=off).shape == (0, 4, 64)
