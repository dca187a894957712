"""GPU tests of where the operands of calls on the paged cache may lie, and of the forms of append that long calls take."""
import pytest
import torch

import paged_reference as ref
import test_gpu_paged as base
from test_gpu_paged import DEV, close, dev, paged, place  # noqa: F401  (paged: fixture)

pytestmark = pytest.mark.gpu


def test_outputs_between_the_rows_of_their_inputs(paged):
    # one buffer: the rows of two tokens' projections far apart, the outputs directly behind the first, and directly behind the last
    gen = torch.Generator().manual_seed(2)
    heads, G, D, P = 2, 2, 64, 16
    q_row, kv_row = heads * G * D, heads * D
    row = q_row + 2 * kv_row
    gap = 2 * q_row + 2 * kv_row
    buf = torch.randn((2 * row + gap + 2 * q_row,), generator=gen).to(torch.bfloat16)
    on = dev(buf)
    stride = row + gap

    qkv = [torch.as_strided(on, (2, h, D), (stride, D, 1), at) for h, at in ((heads * G, 0), (heads, q_row), (heads, q_row + kv_row))]
    qo = torch.as_strided(on, (2, heads * G, D), (q_row, D, 1), row)
    ko = torch.as_strided(on, (2, heads, D), (kv_row, D, 1), row + 2 * q_row)
    before = [t.clone().cpu() for t in qkv]
    rotation = paged.rotation_table(32, D, device="cpu")
    c = paged.PagedCache.empty(2, heads * G, heads, D, P, "bf16", device=DEV, rotation=dev(rotation), out_dtype="bf16")
    table, lens = torch.tensor([[1]], dtype=torch.int32, device=DEV), torch.tensor([2], dtype=torch.int32, device=DEV)
    off = torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    c.append(qkv[1], qkv[2], table, lens, new_offsets=off, q=qkv[0], q_out=qo, k_out=ko)
    out = torch.as_strided(on, (2, heads * G, D), (q_row, D, 1), stride + row)  # behind the second token's row
    c.attn(qo, table, lens, q_offsets=off, out=out)
    torch.cuda.synchronize()
    for t, b in zip(qkv, before):
        assert torch.equal(t.cpu(), b)
    for got, x in ((qo, before[0]), (ko, before[1])):
        want = ref.rotated(x.double(), torch.arange(2), rotation, "halves")
        close(got, want, 2.0 ** -8 * want.abs() + 3 * ref.U * want.abs().amax(-1, keepdim=True))
    pages = (c.k_pages.cpu(), c.v_pages.cpu(), None, None)
    assert torch.equal(pages[0][1, :, :2].transpose(0, 1), ko.cpu()) and torch.equal(pages[1][1, :, :2].transpose(0, 1), before[2])
    close(out, *ref.attention(qo.cpu(), pages, table.cpu(), lens.cpu(), off.cpu(), D ** -0.5, "bf16"))
    for bad in (dict(q_out=torch.as_strided(on, (2, heads * G, D), (q_row, D, 1), row - 8)), dict(k_out=torch.as_strided(on, (2, heads, D), (kv_row, D, 1), row + 2 * q_row + 8))):
        with pytest.raises(paged.PQCacheError):
            c.append(qkv[1], qkv[2], table, lens, new_offsets=off, q=qkv[0], **{**dict(q_out=qo, k_out=ko), **bad})


# ------------------------------------------------------------------ forms of long calls
def ragged(n, seed, most, longer=()):
    """n lengths with their new tokens, a few of none; `longer`: (sequence, length, new) that differ."""
    gen = torch.Generator().manual_seed(seed)
    new = [int(x) for x in torch.randint(0, most + 1, (n,), generator=gen)]
    lengths = [w + int(x) for w, x in zip(new, torch.randint(0, 40, (n,), generator=gen))]
    for b, t, w in longer:
        lengths[b], new[b] = t, w
    return lengths, new


LONG_APPENDS = {  # lengths with the new tokens, new, P, heads, G, D, cache, dtype, rot, style
    # from 64 pages on the workgroups of eight pages lie side by side: numbers of pages that eight does not divide, calls that begin inside a page;
    # from 1024 tokens on two queries share a workgroup
    "94 pages": ([1507], [1500], 16, 2, 2, 128, "fp8", "bf16", 128, "halves"),
    "four prompts": ([900, 37, 1205, 64], [880, 37, 1200, 1], 16, 3, 1, 64, "bf16", "bf16", 64, "halves"),
    "fp32, pairs": ([2200, 300], [2111, 299], 32, 1, 3, 128, "fp8", "f32", 64, "pairs"),
    "fp32, bf16 pages": ([1301, 40], [1301, 22], 16, 2, 1, 128, "bf16", "f32", 128, "pairs"),
    "64 dimensions, 8 bits": ([1100], [1033], 16, 1, 16, 64, "fp8", "bf16", 32, "halves"),
    "odd tokens, many heads": ([1025, 70], [1025, 0], 16, 5, 2, 64, "fp8", "bf16", 0, "halves"),
    # more sequences than a wave has lanes, pages of several calls' lengths in the second and third group of 64
    "70 of one token": ([5 + 7 * b for b in range(70)], [1] * 70, 16, 2, 4, 128, "fp8", "bf16", 128, "halves"),
    "150, ragged": (*ragged(150, 4, 12, ((70, 300, 290), (149, 120, 77))), 16, 2, 2, 64, "fp8", "bf16", 64, "halves"),
    "90, ragged, bf16 pages": (*ragged(90, 5, 30, ((88, 200, 170),)), 32, 1, 2, 128, "bf16", "bf16", 128, "pairs"),
}


@pytest.mark.parametrize("case", LONG_APPENDS)
def test_long_appends(paged, case):
    base.test_append(paged, *LONG_APPENDS[case])


def test_one_token_of_each_of_many_sequences_with_and_without_offsets(paged):
    gen = torch.Generator().manual_seed(6)
    B, heads, G, D, P = 131, 2, 3, 128, 16
    lengths = [int(x) for x in torch.randint(1, 90, (B,), generator=gen)]
    table, n_pages = place(lengths, P, gen)
    k, ks = ref.fill_pool(n_pages, heads, P, D, "fp8", gen)
    v, vs = ref.fill_pool(n_pages, heads, P, D, "fp8", gen)
    rotation = dev(paged.rotation_table(90, D, device="cpu"))
    x = dev(torch.randn((B, heads * (G + 2), D), generator=gen).to(torch.bfloat16) * 30.0)
    table, lens = dev(table), dev(torch.tensor(lengths, dtype=torch.int32))
    got = []
    for off in (None, torch.arange(B + 1, dtype=torch.int32, device=DEV)):
        c = paged.PagedCache(*(dev(t).clone() for t in (k, v, ks, vs)), n_q_heads=heads * G, rotation=rotation)
        ko = torch.empty((B, heads, D), dtype=torch.bfloat16, device=DEV)
        qo = c.append(x[:, heads * G:heads * (G + 1)], x[:, heads * (G + 1):], table, lens, new_offsets=off, q=x[:, :heads * G], k_out=ko)
        got.append((c.k_pages.view(torch.uint8), c.v_pages.view(torch.uint8), c.k_scale, c.v_scale, qo, ko))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


MANY_SEQUENCES = {  # lengths, queries, P, heads, G, D, cache, dtype, out
    "tiles of 128 rows": (*ragged(70, 7, 40, ((3, 2500, 60), (66, 4000, 64), (69, 700, 33))), 16, 1, 4, 128, "fp8", "bf16", "f32"),
    "tiles of 128 rows, bf16 out": (*ragged(140, 8, 60, ((64, 1800, 40), (139, 3000, 45))), 64, 2, 3, 64, "bf16", "bf16", "bf16"),
    "tiles of 16 rows": (*ragged(70, 9, 6, ((1, 900, 5), (67, 5000, 7))), 32, 2, 4, 128, "fp8", "bf16", "f32"),
    "tiles of 16 rows, no queries for many": ([40] * 130, [0] * 65 + [3] + [0] * 63 + [9], 16, 1, 5, 128, "bf16", "f32", "f32"),
}


@pytest.mark.parametrize("case", MANY_SEQUENCES)
def test_several_tokens_of_many_sequences(paged, case):
    base.test_attention_of_several_tokens(paged, *MANY_SEQUENCES[case])
