"""Outputs that overlap inputs of the paged cache's calls: refused on the host, to the byte."""
import ctypes as C

import pytest
import torch

from paper_2407_12820_amd import paged

MB = 1 << 20  # addresses below are never read: every call is refused first


@pytest.fixture(scope="module")
def lib():
    return paged._load()


def config(**kw):
    # two tokens, 4 query heads on 2 KV heads of 64 dimensions, bf16: rows of 512 and 256 bytes
    c = paged.Config(2, 4, 2, 64, 16, 10, 4, 1, 1, 0, 0.0, 0, 0, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


PAGES = paged.Pages(64 * MB, 80 * MB, None, None, 96 * MB, 97 * MB, None)  # pools of 10 * 2 * 16 * 64 bf16: 40960 bytes
POOL = 40960


def append(lib, q=1 * MB, q_stride=256, k=2 * MB, k_stride=128, v=3 * MB, v_stride=128, n=2, q_out=4 * MB, k_out=5 * MB, **cfg):
    c = config(**cfg)
    return lib.pqc_paged_append(C.byref(c), C.byref(PAGES), q, q_stride, k, k_stride, v, v_stride, n, 6 * MB, None, None, q_out, k_out, None)


def test_append(lib):
    for bad in (
        dict(q_out=1 * MB), dict(q_out=1 * MB + 16), dict(q_out=1 * MB - 1008), dict(q_out=1 * MB + 1008),           # the queries
        dict(q_out=2 * MB), dict(q_out=2 * MB + 496), dict(q_out=2 * MB - 1008),                                      # the keys
        dict(q_out=3 * MB), dict(q_out=3 * MB - 512), dict(k_out=3 * MB + 496), dict(k_out=2 * MB - 496),             # the values
        dict(k_out=1 * MB + 1008), dict(k_out=4 * MB + 1008), dict(k_out=4 * MB - 496),                               # queries, the other output
        dict(q_out=64 * MB + POOL - 16), dict(k_out=80 * MB - 16), dict(k_out=64 * MB),                               # the pools
        # rows of one projection of 1024 bytes; the second token's
        dict(q=1 * MB, k=1 * MB + 512, v=1 * MB + 768, q_stride=512, k_stride=512, v_stride=512, k_out=1 * MB + 1024 + 1008),
        dict(q=1 * MB, k=1 * MB + 512, v=1 * MB + 768, q_stride=512, k_stride=512, v_stride=512, q_out=1 * MB + 1024 + 768 - 1008),
        # the last of many tokens, far away
        dict(n=1000, k_stride=1 << 30, k_out=2 * MB + (999 << 31) - 16),
    ):
        assert append(lib, **bad) == -1, bad


def test_attention(lib):
    c = config()
    need = max(lib.pqc_paged_workspace_bytes(C.byref(c), 2, n) for n in (0, 3))

    def attn(out, q=1 * MB, n=2):
        return lib.pqc_paged_attn(C.byref(c), C.byref(PAGES), q, n, 6 * MB, out, 1024 * MB, need, None)

    def gather(out, q=1 * MB, idx=7 * MB):
        return lib.pqc_paged_gather_attn(C.byref(c), C.byref(PAGES), q, idx, 3, out, 1024 * MB, need, None)

    # queries of 1024 bytes, outputs of 2048 (fp32)
    for at in (1 * MB, 1 * MB + 1008, 1 * MB - 2032, 64 * MB + POOL - 16, 80 * MB - 16, 1024 * MB - 16, 1024 * MB + need - 16):
        assert attn(at) == -1, at
    for at in (1 * MB, 1 * MB + 1008, 1 * MB - 2032, 64 * MB + POOL - 16, 80 * MB - 16, 7 * MB - 2032, 7 * MB + 32):
        assert gather(at) == -1, at


def test_the_binding_names_partial_overlaps():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = paged.PagedCache(k, k.clone(), None, None, n_q_heads=4, out_dtype="bf16")
    table, lengths = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    rows = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    idx = torch.zeros((2, 2, 5), dtype=torch.int32)
    for q, out in ((rows[:2], rows[1:]), (rows[1:], rows[:2])):
        for call in (lambda: cache.attn(q, table, lengths, out=out), lambda: cache.gather_attn(q, idx, table, lengths, out=out)):
            with pytest.raises(ValueError, match="overlap"):
                call()
