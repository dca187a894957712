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


# ------------------------------------------------------------------ what the documentation allows beside the ordinary
def test_offsets_that_begin_behind_the_first_row(paged):
    gen = torch.Generator().manual_seed(12)
    P, heads, G, D, n = 16, 2, 2, 64, 80
    off = torch.tensor([3, 3, 40, 71], dtype=torch.int32)  # rows 0 .. 2 and from 71 on are nobody's, the first sequence has none
    lens = torch.tensor([5, 60, 31], dtype=torch.int32)
    table, n_pages = place(lens.tolist(), P, gen)
    rotation = paged.rotation_table(64, D, device="cpu")
    k, v = (ref.fill_pool(n_pages, heads, P, D, "bf16", gen)[0] for _ in range(2))
    q0, k0, v0 = (torch.randn((n, h, D), generator=gen).to(torch.bfloat16) for h in (heads * G, heads, heads))
    for t in (q0, k0, v0):
        t[:3], t[71:] = float("nan"), float("nan")
    c = paged.PagedCache(dev(k), dev(v), None, None, n_q_heads=heads * G, rotation=dev(rotation))
    qo, ko = (torch.full_like(dev(t), 7.0) for t in (q0, k0))
    c.append(dev(k0), dev(v0), dev(table), dev(lens), new_offsets=dev(off), q=dev(q0), q_out=qo, k_out=ko)
    pos = torch.cat([torch.arange(60 - 37, 60), torch.arange(31)])
    for got, x in ((qo, q0), (ko, k0)):
        want = ref.rotated(x[3:71].double(), pos, rotation, "halves")
        close(got[3:71], want, 2.0 ** -8 * want.abs() + 3 * ref.U * want.abs().amax(-1, keepdim=True))
        assert bool((got[:3] == 7.0).all()) and bool((got[71:] == 7.0).all())
    pages = (c.k_pages.cpu(), c.v_pages.cpu(), None, None)
    want_k, _, tol = ref.append(ref.rotated(torch.cat([torch.zeros(3, heads, D), k0[3:71].float()]).double(), torch.cat([torch.zeros(3).long(), pos]), rotation, "halves"), k, None, table, lens, off)
    assert bool(((ref.dequantised(pages[0], None) - want_k).abs() <= tol).all())
    # the wide tiles, and those of 16 rows with queries for the last places only
    for several in (off, torch.tensor([2, 2, 5, 9], dtype=torch.int32)):
        rows = int(several[-1]) + 4
        q = torch.randn((rows, heads * G, D), generator=gen).to(torch.bfloat16)
        q[:int(several[0])], q[int(several[-1]):] = float("nan"), float("nan")
        out = torch.full((rows, heads * G, D), 7.0, device=DEV)
        c.attn(dev(q), dev(table), dev(lens), q_offsets=dev(several), out=out)
        want, tol = ref.attention(q, pages, table, lens, several, D ** -0.5, "f32")
        close(out, want, tol)
        lo, hi = int(several[0]), int(several[-1])
        assert bool((out[:lo] == 7.0).all()) and bool((out[hi:] == 7.0).all())


def test_tokens_taken_back(paged):
    """A program that drafts tokens and rejects some: shorter lengths, then other tokens in their places.  What stays is as it was."""
    gen = torch.Generator().manual_seed(13)
    P, heads, D = 16, 2, 64
    c = paged.PagedCache.empty(4, 4, heads, D, P, device=DEV)
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
    lens = lambda n: torch.tensor([n], dtype=torch.int32, device=DEV)  # noqa: E731
    x = torch.randn((40, heads, D), generator=gen).to(torch.bfloat16)
    kept, at = [], 0
    for new, stay, size in ((14, 14, 1.0), (5, 2, 8.0), (4, 1, 1.0), (5, 5, 0.25), (6, 3, 2.0)):
        t = dev((x[at:at + new].float() * size).to(torch.bfloat16))
        at += new
        n = len(kept) + new
        c.append(t, t, dev(table), lens(n), new_offsets=torch.tensor([0, new], dtype=torch.int32, device=DEV))
        kept += list(t[:stay].cpu())
    want = torch.stack(kept).double()
    n = len(kept)
    for pool, scale in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
        got = ref.dequantised(pool.cpu(), scale.cpu())[table[0].long()].transpose(1, 2).reshape(-1, heads, D)[:n]
        s = scale.cpu()[table[0].long()].double().repeat_interleave(P, 0)[:n, :, None]
        assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -9 * s).all())
    q = torch.randn((1, 4, D), generator=gen).to(torch.bfloat16)
    pages = tuple(t.cpu() for t in (c.k_pages, c.v_pages, c.k_scale, c.v_scale))
    close(c.attn(dev(q), dev(table), lens(n)), *ref.attention(q, pages, table, torch.tensor([n]), None, D ** -0.5, "f32"))


def test_rotated_keys_without_a_place(paged):
    # more new tokens than the length says, or than the table has room for: their queries are rotated, their keys' rows are left
    x = torch.randn((9, 1, 64), generator=torch.Generator().manual_seed(14)).to(torch.bfloat16)
    rotation = paged.rotation_table(40, 64, device="cpu")
    c = paged.PagedCache.empty(2, 1, 1, 64, 16, "bf16", device=DEV, rotation=dev(rotation))
    off = torch.tensor([0, 4, 9], dtype=torch.int32, device=DEV)
    ko = torch.full((9, 1, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    table, lens = torch.tensor([[0], [1]], dtype=torch.int32, device=DEV), torch.tensor([2, 18], dtype=torch.int32, device=DEV)
    qo = c.append(dev(x), dev(x), table, lens, new_offsets=off, q=dev(x), k_out=ko)
    pos = torch.tensor([-2, -1, 0, 1, 13, 14, 15, 16, 17]).clamp(min=0)
    want = ref.rotated(x.double(), pos, rotation, "halves")
    tol = 2.0 ** -8 * want.abs() + 3 * ref.U * want.abs().amax(-1, keepdim=True)
    close(qo, want, tol)
    close(ko[2:7], want[2:7], tol[2:7])
    assert bool((ko[:2] == 7.0).all()) and bool((ko[7:] == 7.0).all())


@pytest.mark.parametrize("heads", [200, 300, 600])
def test_hundreds_of_heads(paged, heads):
    # fewer workgroups per head than parts could be folded by, down to one
    base.test_attention_of_one_token(paged, [300, 5, 17], 16, heads, 1, 64, "fp8", "bf16", "f32")
    base.test_attention_of_several_tokens(paged, [200, 31], [3, 4], 16, heads, 2, 64, "bf16", "bf16", "f32")
    base.test_attention_of_several_tokens(paged, [600, 70], [70, 66], 32, heads, 1, 64, "fp8", "bf16", "bf16")
    base.test_attention_to_listed_tokens(paged, [300, 90], 150, 16, heads, 1, 64, "fp8", "bf16", "f32")
    base.test_append(paged, [40, 3], [25, 3], 16, heads, 1, 64, "fp8", "bf16", 64, "halves")


def test_thousands_of_sequences_under_a_table_for_16_million_tokens(paged):
    # units of work are of 512 tokens here, so that their sum stays within 32 bits whatever the lengths; 4.3 GB of page table
    gen = torch.Generator().manual_seed(15)
    B, P, heads, G, D = 16384, 256, 1, 2, 64
    lengths = torch.randint(0, 30, (B,), generator=gen).int()
    long = [(0, 1300), (63, 513), (64, 1024), (9000, 1600), (B - 1, 2000)]
    for b, t in long:
        lengths[b] = t
    n_pages = 64
    k, ks = ref.fill_pool(n_pages, heads, P, D, "fp8", gen)
    v, vs = ref.fill_pool(n_pages, heads, P, D, "fp8", gen)
    own = torch.randint(0, n_pages, (B, 8), generator=gen).int()  # pages are only read: sequences share them
    table = torch.full((B, 65536), -1, dtype=torch.int32, device=DEV)
    table[:, :8] = dev(own)
    c = paged.PagedCache(dev(k), dev(v), dev(ks / 64.0), dev(vs), n_q_heads=heads * G)
    q = torch.randn((B, heads * G, D), generator=gen).to(torch.bfloat16)
    some = [b for b, _ in long] + [1, 62, 65, 127, 128, 5000, B - 2]
    got = c.attn(dev(q), table, dev(lengths))
    few = 3 * torch.arange(B + 1, dtype=torch.int32)
    q3 = torch.randn((3 * B, heads * G, D), generator=gen).to(torch.bfloat16)
    got3 = c.attn(dev(q3), table, dev(lengths), q_offsets=dev(few))
    torch.cuda.synchronize()
    pages = (k, v, ks / 64.0, vs)
    for b in some:
        one = (own[b:b + 1], lengths[b:b + 1])
        close(got[b:b + 1], *ref.attention(q[b:b + 1], pages, *one, None, D ** -0.5, "f32"), f"sequence {b}")
        close(got3[3 * b:3 * b + 3], *ref.attention(q3[3 * b:3 * b + 3], pages, *one, torch.tensor([0, 3]), D ** -0.5, "f32"), f"queries of {b}")
    assert bool((got[dev(lengths) == 0] == 0).all())
