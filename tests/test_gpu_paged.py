"""GPU tests of the paged cache against a plain evaluation in 64 bits (tests/paged_reference.py, which derives the tolerances)."""
import dataclasses
import random

import numpy as np
import pytest
import torch

from paper_2407_12820_amd import workloads as wl

import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def paged():
    from paper_2407_12820_amd import paged as m
    m._load()
    return m


def dev(t):
    return None if t is None else t.to(DEV)


def place(lengths, P, gen, spare=3, extra_entries=1):
    """A shuffled page table for the lengths; entries behind a sequence name no page."""
    need = [-(-max(n, 0) // P) for n in lengths]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=gen).int()
    table = torch.full((len(lengths), max(need) + extra_entries), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def poison(pages, scale, table, lengths):
    """NaN wherever no sequence has a token: rows behind the last of each sequence, pages that nobody owns, and their scales."""
    P = pages.shape[2]
    raw = pages.view(torch.uint8 if pages.element_size() == 1 else torch.int16)
    live = torch.zeros(pages.shape[0], P, dtype=torch.bool)
    for b, n in enumerate(lengths):
        for e in range(-(-max(n, 0) // P)):
            if 0 <= int(table[b, e]) < pages.shape[0]:
                live[int(table[b, e]), : min(P, n - e * P)] = True
    raw.transpose(1, 2)[~live] = 0x7F if pages.element_size() == 1 else 0x7FFF
    if scale is not None:
        scale[~live.any(1)] = float("nan")


def make(paged, gen, lengths, P, heads, G, D, cache, dtype, out, **kw):
    table, n_pages = place(lengths, P, gen)
    k, ks = ref.fill_pool(n_pages, heads, P, D, cache, gen)
    v, vs = ref.fill_pool(n_pages, heads, P, D, cache, gen)
    if cache == "fp8":
        ks = ks / 64.0  # logits of a moderate size
    poison(k, ks, table, lengths)
    poison(v, vs, table, lengths)
    c = paged.PagedCache(dev(k), dev(v), dev(ks), dev(vs), n_q_heads=heads * G, dtype=dtype, out_dtype=out, **kw)
    return c, (k, v, ks, vs), table


def close(got, want, tol, what=""):
    got = got.double().cpu()
    skip = torch.isnan(want)
    assert torch.isfinite(got[~skip]).all(), what
    err, tol = (got - want).abs()[~skip], tol[~skip]
    over = err > tol
    assert not bool(over.any()), f"{what}: {int(over.sum())} values beyond the tolerance, up to {(err / tol)[over].max().item()} times, error {err.max().item()}"


# ------------------------------------------------------------------ attention, one token per sequence
ONE = [  # lengths, page_tokens, KV heads, G, D, cache, dtype, out
    ([1], 64, 1, 1, 128, "fp8", "bf16", "f32"),
    ([0, 1, 15, 16, 17, 31, 32, 33, 128, 129], 16, 2, 4, 128, "fp8", "bf16", "f32"),
    ([300, 0, 1025, 5, 2049], 64, 2, 8, 128, "fp8", "bf16", "bf16"),
    ([700, 63, 64, 65], 256, 3, 3, 64, "fp8", "bf16", "f32"),
    ([700, 257], 32, 1, 16, 128, "fp8", "f32", "f32"),
    ([515, 9], 128, 2, 5, 64, "fp8", "f32", "bf16"),
    ([300, 0, 1025, 5], 64, 2, 7, 128, "bf16", "bf16", "f32"),
    ([700, 63], 16, 1, 12, 64, "bf16", "bf16", "bf16"),
    ([1023, 1], 128, 1, 1, 128, "bf16", "f32", "f32"),
    ([511, 2], 256, 2, 2, 64, "bf16", "f32", "f32"),
    ([20011], 16, 1, 4, 128, "fp8", "bf16", "f32"),       # many splits, more pages per split than are staged at a time
    ([9000] + [3] * 70, 64, 2, 1, 64, "fp8", "bf16", "f32"),  # more sequences than lanes, one of them long
]


@pytest.mark.parametrize("lengths,P,heads,G,D,cache,dtype,out", ONE)
def test_attention_of_one_token(paged, lengths, P, heads, G, D, cache, dtype, out):
    gen = torch.Generator().manual_seed(len(lengths) * 1000 + P + G)
    c, pages, table = make(paged, gen, lengths, P, heads, G, D, cache, dtype, out)
    q = torch.randn((len(lengths), heads * G, D), generator=gen).to(IO[dtype])
    print(f"[case] {lengths[:6]} P={P} heads={heads} G={G} D={D} {cache} {dtype} {out}", flush=True)
    got = c.attn(dev(q), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)))
    torch.cuda.synchronize()
    want, tol = ref.attention(q, pages, table, torch.tensor(lengths), None, D ** -0.5, out)
    close(got, want, tol)


# ------------------------------------------------------------------ attention, several tokens per sequence
MANY = [  # lengths, queries, P, heads, G, D, cache, dtype, out
    ([40, 0, 7, 300], [5, 0, 7, 33], 16, 2, 4, 128, "fp8", "bf16", "f32"),
    ([3, 2, 200], [9, 2, 17], 64, 1, 3, 64, "fp8", "bf16", "f32"),        # more queries than tokens: rows that see nothing
    ([257, 100, 1], [257, 1, 1], 64, 2, 1, 128, "fp8", "bf16", "bf16"),
    ([500, 130], [129, 130], 256, 1, 16, 128, "fp8", "bf16", "bf16"),
    ([260], [260], 32, 1, 7, 64, "fp8", "f32", "f32"),
    ([150, 333], [64, 200], 128, 2, 2, 128, "bf16", "bf16", "bf16"),
    ([150, 90], [70, 90], 16, 1, 5, 64, "bf16", "f32", "f32"),
    ([3000, 10], [3, 10], 64, 1, 4, 128, "fp8", "bf16", "f32"),             # a few queries on a long cache: splits
    ([1500, 700], [300, 650], 64, 2, 4, 128, "fp8", "bf16", "bf16"),
    ([900], [900], 16, 1, 8, 128, "bf16", "bf16", "f32"),
    # tiles of 128 rows: groups that do not divide them, more queries than tokens, rows that see nothing, one long sequence of splits
    ([130, 77], [130, 70], 16, 2, 3, 64, "fp8", "bf16", "f32"),
    ([300, 20, 64, 0], [200, 90, 64, 3], 32, 1, 7, 128, "fp8", "bf16", "bf16"),
    ([129, 1, 257], [129, 1, 200], 256, 1, 5, 128, "bf16", "bf16", "f32"),
    ([200, 65], [150, 65], 64, 1, 6, 64, "bf16", "bf16", "bf16"),
    ([5000, 63], [40, 63], 64, 1, 4, 128, "fp8", "bf16", "f32"),
    ([6000], [33], 16, 1, 1, 128, "fp8", "bf16", "bf16"),
    ([40], [40], 128, 1, 13, 64, "fp8", "bf16", "f32"),
    ([300, 140, 9], [300, 33, 20], 64, 1, 4, 128, "fp8", "f32", "f32"),
    ([170, 2500], [170, 31], 128, 2, 3, 128, "bf16", "f32", "bf16"),
]


@pytest.mark.parametrize("lengths,queries,P,heads,G,D,cache,dtype,out", MANY)
def test_attention_of_several_tokens(paged, lengths, queries, P, heads, G, D, cache, dtype, out):
    gen = torch.Generator().manual_seed(sum(lengths) + P + G)
    c, pages, table = make(paged, gen, lengths, P, heads, G, D, cache, dtype, out)
    off = [0]
    for n in queries:
        off.append(off[-1] + n)
    n = off[-1] + 5  # a padded batch: rows behind the last sequence
    q = torch.randn((n, heads * G, D), generator=gen).to(IO[dtype])
    q[off[-1]:] = float("nan")
    res = torch.full((n, heads * G, D), 7.0, dtype=IO[out], device=DEV)
    print(f"[case] {lengths} {queries} P={P} heads={heads} G={G} D={D} {cache} {dtype} {out}", flush=True)
    offsets = torch.tensor(off, dtype=torch.int32)
    c.attn(dev(q), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)), q_offsets=dev(offsets), out=res)
    torch.cuda.synchronize()
    want, tol = ref.attention(q, pages, table, torch.tensor(lengths), offsets, D ** -0.5, out)
    close(res, want, tol)
    assert bool((res[off[-1]:] == 7.0).all()), "rows behind the last sequence"


@pytest.mark.parametrize("several", [0, 3, 40])  # query tokens of each sequence (0: one, without offsets)
def test_pages_that_are_not_there_and_lengths_out_of_range(paged, several):
    # entries outside the pool name no page: their tokens are left out; lengths are taken into the table's room
    gen = torch.Generator().manual_seed(5)
    lengths = [300, 200, 500, 160]
    c, pages, table = make(paged, gen, lengths, 64, 2, 4, 128, "fp8", "bf16", "f32")
    table[0, 1], table[1, 0], table[1, 3] = -1, pages[0].shape[0], 2 ** 31 - 1
    table[2, :], table[3, 0] = -7, -2 ** 31
    told = torch.tensor([300, 200, 500, 2 ** 31 - 1], dtype=torch.int32)  # the last: all of its row, whose rear entries are -1
    told_cut = torch.tensor([300, 200, 500, table.shape[1] * 64])
    n = 4 * several if several else 4
    off = several * torch.arange(5, dtype=torch.int32) if several else None
    q = torch.randn((n, 8, 128), generator=gen).to(torch.bfloat16)
    # (the fourth sequence ends inside its third page; what lies behind would be read if its length were believed)
    for name in (0, 1):
        raw = pages[name].view(torch.uint8)
        raw[int(table[3, 2]), :, 160 - 128:] = 0x30
    c.k_pages.view(torch.uint8).copy_(pages[0].view(torch.uint8))
    c.v_pages.view(torch.uint8).copy_(pages[1].view(torch.uint8))
    got = c.attn(dev(q), dev(table), dev(told), q_offsets=dev(off))
    neg = c.attn(dev(q), dev(table), dev(torch.tensor([-1, -2 ** 31, -5, 0], dtype=torch.int32)), q_offsets=dev(off))
    torch.cuda.synchronize()
    want, tol = ref.attention(q, pages, table, told_cut, off, 128 ** -0.5, "f32")
    close(got, want, tol)
    assert bool((neg == 0).all())


# ------------------------------------------------------------------ attention to listed tokens
LISTED = [  # lengths, listed, P, heads, G, D, cache, dtype, out
    ([50], 1, 64, 1, 1, 128, "fp8", "bf16", "f32"),
    ([400, 0, 33, 1], 70, 16, 2, 4, 128, "fp8", "bf16", "f32"),
    ([1000, 700], 515, 64, 2, 8, 128, "fp8", "bf16", "bf16"),
    ([9000], 3001, 256, 1, 3, 64, "fp8", "f32", "f32"),
    ([600, 90], 129, 128, 1, 16, 128, "bf16", "bf16", "f32"),
    ([300], 300, 32, 2, 5, 64, "bf16", "f32", "bf16"),
]


@pytest.mark.parametrize("lengths,count,P,heads,G,D,cache,dtype,out", LISTED)
def test_attention_to_listed_tokens(paged, lengths, count, P, heads, G, D, cache, dtype, out):
    gen = torch.Generator().manual_seed(count + P)
    c, pages, table = make(paged, gen, lengths, P, heads, G, D, cache, dtype, out)
    B = len(lengths)
    idx = torch.full((B, heads, count), -1, dtype=torch.int32)
    for b, t in enumerate(lengths):
        for h in range(heads):
            n = min(count, t)
            idx[b, h, :n] = torch.randperm(t, generator=gen)[:n].int()  # in no order
    if count > 60:
        idx[0, 0, 3], idx[0, 0, 17], idx[0, 0, 40] = lengths[0], 2 ** 31 - 1, -2 ** 31  # outside the sequence
        idx[0, 0, 5] = idx[0, 0, 6]  # twice
    q = torch.randn((B, heads * G, D), generator=gen).to(IO[dtype])
    print(f"[case] {lengths} {count} P={P} heads={heads} G={G} D={D} {cache} {dtype} {out}", flush=True)
    got = c.gather_attn(dev(q), dev(idx), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)))
    torch.cuda.synchronize()
    want, tol = ref.attention(q, pages, table, torch.tensor(lengths), None, D ** -0.5, out, listed=idx)
    close(got, want, tol)
    if heads > 1:  # a list of nothing
        idx[0, 1] = -1
        got = c.gather_attn(dev(q), dev(idx), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)))
        assert bool((got[0, G:2 * G] == 0).all())


# ------------------------------------------------------------------ append
APPEND = [  # lengths with the new tokens, new, P, heads, G, D, cache, dtype, rot, style
    ([1], [1], 64, 1, 1, 128, "fp8", "bf16", 128, "halves"),
    ([70, 1, 64, 65, 0], [1, 1, 1, 1, 0], 64, 2, 4, 128, "fp8", "bf16", 128, "halves"),
    ([300, 47, 16, 500], [130, 47, 3, 1], 16, 2, 2, 128, "fp8", "bf16", 64, "pairs"),
    ([300, 200], [37, 200], 256, 1, 5, 64, "fp8", "f32", 64, "halves"),
    ([300, 200], [37, 200], 256, 2, 3, 128, "fp8", "f32", 0, "halves"),
    ([129, 90, 33], [100, 1, 33], 32, 2, 7, 64, "bf16", "bf16", 32, "halves"),
    ([129, 90], [100, 90], 128, 3, 1, 128, "bf16", "f32", 128, "pairs"),
]


def projection(n, heads, G, D, dtype, gen):
    """q, k, v as parts of one row per token."""
    rows = torch.randn((n, (G + 2) * heads * D), generator=gen) * torch.exp2(torch.randint(-3, 5, (n, 1), generator=gen).float())
    rows = rows.to(IO[dtype])
    return rows, [x.unflatten(1, (-1, D)) for x in rows.split([G * heads * D, heads * D, heads * D], 1)]


@pytest.mark.parametrize("lengths,new,P,heads,G,D,cache,dtype,rot,style", APPEND)
def test_append(paged, lengths, new, P, heads, G, D, cache, dtype, rot, style):
    gen = torch.Generator().manual_seed(sum(lengths) + P)
    table, n_pages = place(lengths, P, gen)
    k, ks = ref.fill_pool(n_pages, heads, P, D, cache, gen, (-4, 1))
    v, vs = ref.fill_pool(n_pages, heads, P, D, cache, gen, (-4, 1))
    rotation = paged.rotation_table(max(lengths), rot, base=500000.0, device="cpu") if rot else None
    c = paged.PagedCache(dev(k), dev(v), dev(ks), dev(vs), n_q_heads=heads * G, dtype=dtype, rotation=dev(rotation), rot_style=style)
    off = [0]
    for m in new:
        off.append(off[-1] + m)
    n = off[-1] + 3  # rows behind the last sequence
    rows, (q0, k0, v0) = projection(n, heads, G, D, dtype, gen)
    q1, k1, v1 = (x.unflatten(1, (-1, D)) for x in dev(rows).split([G * heads * D, heads * D, heads * D], 1))
    offsets, lens = torch.tensor(off, dtype=torch.int32), torch.tensor(lengths, dtype=torch.int32)
    qo = torch.full((n, heads * G, D), 7.0, dtype=IO[dtype], device=DEV)
    ko = torch.full((n, heads, D), 7.0, dtype=IO[dtype], device=DEV)
    print(f"[case] {lengths} {new} P={P} heads={heads} G={G} D={D} {cache} {dtype} {rot} {style}", flush=True)
    assert c.append(k1, v1, dev(table), dev(lens), new_offsets=dev(offsets), q=q1, q_out=qo, k_out=ko) is qo
    torch.cuda.synchronize()

    m = off[-1]
    pos = torch.cat([torch.arange(t - w, t) for t, w in zip(lengths, new)]).long()
    kr, qr = (x[:m].double() if not rot else ref.rotated(x[:m].double(), pos, rotation, style) for x in (k0, q0))
    half = ref.U if dtype == "f32" else 2.0 ** -8
    for got, want in ((qo, qr), (ko, kr)):
        close(got[:m], want, half * want.abs() + 3 * ref.U * want.abs().amax(-1, keepdim=True) + 1e-30)
        assert bool((got[m:] == 7.0).all()), "rows behind the last sequence"
    for name, x, before, scale, pool, new_scale in (("k", kr, k, ks, c.k_pages, c.k_scale), ("v", v0[:m].double(), v, vs, c.v_pages, c.v_scale)):
        want, want_scale, tol = ref.append(x, before, scale, table, lens, offsets)
        if scale is not None:
            assert torch.equal(new_scale.cpu().double(), want_scale), name
        got = ref.dequantised(pool.cpu(), None if scale is None else new_scale.cpu())
        # what shares a page with new tokens but is neither kept nor new has no meaning: its codes, not its values, stay
        live = torch.zeros((n_pages, P), dtype=torch.bool)
        dead = torch.zeros((n_pages, P), dtype=torch.bool)
        for b, t in enumerate(lengths):
            for e in range(-(-t // P)):
                live[int(table[b, e]), : min(P, t - e * P)] = True
                dead[int(table[b, e]), min(P, t - e * P):] = True
        sel = live[:, None, :, None].expand_as(want)
        err = ((got - want).abs() - tol)[sel]
        assert bool((err <= 0).all()), (name, err.max().item())
        raw = torch.uint8 if cache == "fp8" else torch.int16
        rest = ~live[:, None, :, None].expand_as(want)
        assert torch.equal(pool.cpu().view(raw)[rest], before.view(raw)[rest]), "rows that hold no token"


def test_append_token_by_token_keeps_what_was_there(paged):
    # a page filled one token at a time, each larger than the last: the scale grows by powers of two, which moves older values
    # by half a step of the final subnormals at most
    gen = torch.Generator().manual_seed(9)
    P, heads, D = 64, 2, 128
    c = paged.PagedCache.empty(3, 4, heads, D, P, device=DEV)
    c.k_pages.view(torch.uint8).fill_(0x7F)
    c.v_pages.view(torch.uint8).fill_(0x7F)
    c.k_scale.fill_(float("nan"))  # a page that starts anew ignores what it held
    c.v_scale.fill_(1e30)
    table = torch.tensor([[1, 2]], dtype=torch.int32, device=DEV)
    xs = []
    for t in range(70):
        x = (torch.randn((1, 2 * heads, D), generator=gen) * 2.0 ** (t / 8.0 - 4.0)).to(torch.bfloat16)
        xs.append(x)
        c.append(dev(x[:, :heads].contiguous()), dev(x[:, heads:].contiguous()), table, torch.tensor([t + 1], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    x = torch.cat(xs).double()
    for at, pool, scale in ((0, c.k_pages, c.k_scale), (heads, c.v_pages, c.v_scale)):
        got = ref.dequantised(pool.cpu(), scale.cpu())
        for page, lo, hi in ((1, 0, 64), (2, 64, 70)):
            for h in range(heads):
                want = x[lo:hi, at + h]
                s = ref.power_scale(float(want.abs().max()))
                assert float(scale[page, h]) == s
                # each re-encoding leaves normal codes as they are and moves a subnormal one by half its step, which doubles every
                # time: together less than one step of the last
                tol = 2.0 ** -4 * want.abs() + 2.0 ** -9 * s
                assert bool(((got[page, h, : hi - lo] - want).abs() <= tol).all())


def test_positions_of_the_caller_and_places_beyond_the_table(paged):
    gen = torch.Generator().manual_seed(3)
    P, heads, D, n = 16, 1, 64, 40
    k, v = (ref.fill_pool(6, heads, P, D, "bf16", gen)[0] for _ in range(2))
    rotation = paged.rotation_table(50, D, device="cpu")
    c = paged.PagedCache(dev(k), dev(v), None, None, n_q_heads=1, rotation=dev(rotation))
    x = torch.randn((n, heads, D), generator=gen).to(torch.bfloat16)
    pos = torch.randint(-5, 70, (n,), generator=gen).int()  # taken into the table's rows
    table = torch.tensor([[3, -1], [5, 0]], dtype=torch.int32)
    offsets = torch.tensor([0, 28, 40], dtype=torch.int32)
    lengths = torch.tensor([20, 37], dtype=torch.int32)  # places -8 .. 19 (the second page is not there), 25 .. 36 (the table ends at 31)
    ko = torch.empty((n, heads, D), dtype=torch.bfloat16, device=DEV)
    qo = c.append(dev(x), dev(x), dev(table), dev(lengths), new_offsets=dev(offsets), q=dev(x), positions=dev(pos), k_out=ko)
    torch.cuda.synchronize()
    want = ref.rotated(x.double(), pos.long().clamp(0, 49), rotation, "halves")
    tol = 2.0 ** -8 * want.abs() + 3 * ref.U * want.abs().amax(-1, keepdim=True)
    close(qo, want, tol)
    stored = [t for t in range(8, 28)] + [t for t in range(28, 35)]  # of places in the sequences
    close(ko[stored], want[stored], tol[stored])
    for pool, before, y, t in ((c.k_pages, k, want, tol), (c.v_pages, v, x.double(), torch.zeros_like(tol))):
        after = before.double().clone()
        room = torch.zeros_like(after)
        after[3, 0, :16], room[3, 0, :16] = y[8:24, 0], t[8:24, 0]
        after[0, 0, 9:16], room[0, 0, 9:16] = y[28:35, 0], t[28:35, 0]
        assert bool(((pool.cpu().double() - after).abs() <= room).all())


# ------------------------------------------------------------------ what a program does around the calls
def test_offsets_beyond_32_bits(paged):
    # two pools of 5.4 GB each, the sequence in their last pages
    gen = torch.Generator().manual_seed(11)
    P, heads, D, n_pages = 256, 8, 128, 10300
    shape = (n_pages, heads, P, D)
    k, v = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert k.numel() * 2 > 2 ** 32
    c = paged.PagedCache(k, v, None, None, n_q_heads=8)
    lengths, new = torch.tensor([700], dtype=torch.int32), 700
    table = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2]], dtype=torch.int32)
    x = torch.randn((new, heads, D), generator=gen).to(torch.bfloat16)
    y = torch.randn((new, heads, D), generator=gen).to(torch.bfloat16)
    c.append(dev(x), dev(y), dev(table), dev(lengths), new_offsets=torch.tensor([0, new], dtype=torch.int32, device=DEV))
    q = torch.randn((1, heads, D), generator=gen).to(torch.bfloat16)
    got = c.attn(dev(q), dev(table), dev(lengths))
    idx = torch.randperm(700, generator=gen)[:300].int().expand(1, heads, 300).contiguous()
    some = c.gather_attn(dev(q), dev(idx), dev(table), dev(lengths))
    torch.cuda.synchronize()
    small = [t[-3:].cpu() for t in (k, v)]
    assert torch.equal(small[0][2, :, :256].transpose(0, 1), x[:256])
    local = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    close(got, *ref.attention(q, (*small, None, None), local, lengths, None, D ** -0.5, "f32"))
    close(some, *ref.attention(q, (*small, None, None), local, lengths, None, D ** -0.5, "f32", listed=idx))


def test_another_stream_and_equal_results_of_equal_calls(paged):
    gen = torch.Generator().manual_seed(21)
    lengths = [5000, 31, 900]
    c, pages, table = make(paged, gen, lengths, 64, 2, 4, 128, "fp8", "bf16", "f32")
    q = dev(torch.randn((3, 8, 128), generator=gen).to(torch.bfloat16))
    idx = dev(torch.randint(0, 31, (3, 2, 900), generator=gen).int())
    table, lens = dev(table), dev(torch.tensor(lengths, dtype=torch.int32))
    a, b = c.attn(q, table, lens), c.gather_attn(q, idx, table, lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream(device=DEV)
    outs = [c.attn(q, table, lens, stream=side) for _ in range(3)] + [c.gather_attn(q, idx, table, lens, stream=side) for _ in range(3)]
    with torch.cuda.stream(side):
        outs += [c.attn(q, table, lens), c.gather_attn(q, idx, table, lens)]
    torch.cuda.synchronize()
    for o, want in zip(outs, [a] * 3 + [b] * 3 + [a, b]):
        assert torch.equal(o, want)


def test_a_recorded_step_follows_its_tables_and_lengths(paged):
    # append + attention + listed attention of one token, recorded once and replayed while the cache grows; a second graph that
    # was recorded meanwhile shares nothing with it
    gen = torch.Generator().manual_seed(31)
    P, heads, G, D, B = 16, 2, 4, 128, 3
    start = [14, 200, 31]
    room = [t + 40 for t in start]
    table, n_pages = place(room, P, gen)
    c, e = (paged.PagedCache.empty(n_pages, heads * G, heads, D, P, device=DEV, rotation=paged.rotation_table(300, D, device=DEV)) for _ in range(2))
    table = dev(table)
    for x in (c, e):
        g2 = torch.Generator().manual_seed(32)
        off = dev(torch.tensor([0, 14, 214, 245], dtype=torch.int32))
        kv = dev(torch.randn((245, 2 * heads, D), generator=g2).to(torch.bfloat16))
        x.append(kv[:, :heads], kv[:, heads:], table, dev(torch.tensor(start, dtype=torch.int32)), new_offsets=off)
    lens = dev(torch.tensor(start, dtype=torch.int32))
    qkv = torch.zeros((B, (G + 2) * heads, D), dtype=torch.bfloat16, device=DEV)
    idx = dev(torch.randint(0, 14, (B, heads, 40), generator=gen).int())

    def step(cache):
        q = cache.append(qkv[:, G * heads:(G + 1) * heads], qkv[:, (G + 1) * heads:], table, lens, q=qkv[:, :G * heads])
        return q, cache.attn(q, table, lens), cache.gather_attn(q, idx, table, lens)

    lens += 1
    step(c)
    step(e)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = step(c)
        graphs.append((graph, res))
    for i in range(36):
        qkv.copy_(torch.randn(qkv.shape, generator=gen).to(torch.bfloat16))
        if i:
            lens += 1
        graph, res = graphs[i % 2]
        graph.replay()
        want = step(e)
        torch.cuda.synchronize()
        for a, b in zip(res, want):
            assert torch.equal(a, b), i
    for a, b in ((c.k_pages, e.k_pages), (c.v_pages, e.v_pages)):
        for row, t in zip(table.tolist(), lens.tolist()):
            for p in range(-(-t // P)):
                n = min(P, t - p * P)
                assert torch.equal(a[row[p], :, :n].view(torch.uint8), b[row[p], :, :n].view(torch.uint8))


@pytest.mark.parametrize("lengths,P,heads,G,D,cache,dtype", [
    ([20011] * 5, 16, 8, 4, 128, "fp8", "bf16"), ([9000] + [3] * 70, 64, 2, 1, 64, "fp8", "bf16"), ([2048], 64, 8, 4, 128, "fp8", "bf16"),
    ([1500, 0, 1300, 1], 32, 2, 16, 128, "bf16", "f32"), ([1900, 700], 128, 3, 3, 64, "bf16", "bf16"), ([2000, 1300, 700, 1], 64, 8, 8, 128, "fp8", "f32")])
def test_parts_folded_by_the_last_workgroup_or_by_a_kernel(paged, lengths, P, heads, G, D, cache, dtype):
    # either way within the tolerance, the same from call to call, and a call leaves its counters zero
    gen = torch.Generator().manual_seed(P + G)
    c, pages, table = make(paged, gen, lengths, P, heads, G, D, cache, dtype, "f32")
    B = len(lengths)
    q = torch.randn((B, heads * G, D), generator=gen).to(IO[dtype])
    idx = torch.randint(0, max(lengths), (B, heads, 2000), generator=gen).int()
    dq, di, dt, lens = dev(q), dev(idx), dev(table), dev(torch.tensor(lengths, dtype=torch.int32))
    last = [c.attn(dq, dt, lens) for _ in range(3)] + [c.gather_attn(dq, di, dt, lens) for _ in range(3)]
    torch.cuda.synchronize()
    scratch = c._scratch.streams[torch.cuda.current_stream().cuda_stream]
    assert c._counted and not bool(scratch.counters.any())
    c._counted = False
    own = [c.attn(dq, dt, lens) for _ in range(3)] + [c.gather_attn(dq, di, dt, lens) for _ in range(3)]
    torch.cuda.synchronize()
    few = [b for b in range(B) if lengths[b] < 5000][:3] + [0]
    for res in (last, own):
        for i, listed in ((0, None), (3, idx)):
            assert torch.equal(res[i], res[i + 1]) and torch.equal(res[i], res[i + 2])
            for b in few:
                want, tol = ref.attention(q[b:b + 1], pages, table[b:b + 1], torch.tensor(lengths[b:b + 1]), None, D ** -0.5, "f32",
                                          listed=None if listed is None else listed[b:b + 1])
                close(res[i][b:b + 1], want, tol, f"{i} {b}")


def test_launches_of_a_step(paged):
    from parity_utils import count_launches

    c, _, table = make(paged, torch.Generator().manual_seed(1), [3000] * 5, 64, 8, 4, 128, "fp8", "bf16", "f32")
    q, table, lens = torch.zeros((5, 32, 128), dtype=torch.bfloat16, device=DEV), dev(table), torch.tensor([3000] * 5, dtype=torch.int32, device=DEV)
    left = len(c._scratch.spare)
    assert count_launches(lambda: c.attn(q, table, lens)) == (1 if left else 2)
    c._counted = False
    assert count_launches(lambda: c.attn(q, table, lens)) == 2


def test_retrieval_over_a_paged_cache(paged):
    """A prompt, PQ structures of its rotated keys, then steps of generation: append, code of the new token, table, scan, top-k and
    attention to the selected tokens of the 8-bit cache; against 64 bits on the values that the cache stands for."""
    from paper_2407_12820_amd import binding

    gen = torch.Generator().manual_seed(41)
    w = wl.get("llama8b_32k", n_tokens=2000, batch=2)
    w = dataclasses.replace(w, topk=200, n_init=4, n_local=64, kmeans_iters=4)
    B, heads, G, D, P, cap = w.batch, w.n_kv_heads, w.group, w.head_dim, 64, 2048
    table, n_pages = place([cap] * B, P, gen)
    table = dev(table)
    cache = paged.PagedCache.empty(n_pages, w.n_q_heads, heads, D, P, device=DEV, rotation=paged.rotation_table(cap, D, device=DEV))
    prompt = 1990
    off = dev(torch.tensor([0, prompt, 2 * prompt], dtype=torch.int32))
    lens = dev(torch.tensor([prompt] * B, dtype=torch.int32))
    q, k, v = (dev(torch.randn((2 * prompt, h, D), generator=gen).to(torch.bfloat16)) for h in (w.n_q_heads, heads, heads))
    rotated_keys = torch.empty_like(k)
    qr = cache.append(k, v, table, lens, new_offsets=off, q=q, k_out=rotated_keys)
    out = cache.attn(qr[:, :].contiguous(), table, lens, q_offsets=off)
    torch.cuda.synchronize()
    pages = lambda: tuple(t.cpu() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale))  # noqa: E731
    # the last queries of the prompt, of two heads
    res = out.cpu().double()
    pg = pages()
    for b, i in ((0, prompt - 1), (1, prompt - 1), (1, 700)):
        for h in (0, 5):
            kk, _ = ref.rows_of(pg[0], pg[2], table.cpu()[b], h, i + 1)
            vv, _ = ref.rows_of(pg[1], pg[3], table.cpu()[b], h, i + 1)
            at = b * prompt + i
            want, tol = ref.attend(qr[at, h * G:(h + 1) * G].cpu().double(), kk, vv, torch.ones((G, i + 1), dtype=torch.bool), D ** -0.5, "f32", True)
            close(res[at, h * G:(h + 1) * G], want, tol)
    # PQ structures of the rotated keys, in buffers with room to grow
    keys = torch.zeros((B, heads, cap, D), dtype=torch.bfloat16, device=DEV)
    keys[:, :, :prompt] = rotated_keys.view(B, prompt, heads, D).transpose(1, 2)
    wp = dataclasses.replace(w, n_tokens=prompt)
    cent, codes = binding.pq_build(wp, keys, dev(torch.from_numpy(wl.kmeans_init_indices(wp, 0))), capacity=cap)
    ctx = binding.PQCache(wp, DEV, capacity=cap)
    new_key = torch.empty((B, heads, D), dtype=torch.bfloat16, device=DEV)
    for step in range(6):
        n = prompt + step + 1
        lens += 1
        q, k, v = (dev(torch.randn((B, h, D), generator=gen).to(torch.bfloat16)) for h in (w.n_q_heads, heads, heads))
        qr = cache.append(k, v, table, lens, q=q, k_out=new_key)
        binding.pq_encode_token(dataclasses.replace(w, n_tokens=n), new_key, cent, codes, n - 1, capacity=cap)
        ctx.set_length(n, w.topk)
        idx = ctx.topk(ctx.scan(ctx.lut(qr, cent), codes))
        got = cache.gather_attn(qr, idx, table, lens)
        torch.cuda.synchronize()
        assert idx.shape == (B, heads, 4 + 200 + 64) and int(idx.max()) == n - 1 and int(idx.min()) == 0
        want, tol = ref.attention(qr.cpu(), pages(), table.cpu(), lens.cpu(), None, D ** -0.5, "f32", listed=idx.cpu())
        close(got, want, tol, f"step {step}")


def test_random_shapes(paged):
    rng = random.Random(77)
    for i in range(24):
        gen = torch.Generator().manual_seed(i)
        D, P, heads = rng.choice([64, 128]), rng.choice([16, 32, 64, 128, 256]), rng.choice([1, 2, 3])
        G = rng.randint(1, 16)
        B = rng.choice([1, 2, 5])
        lengths = [rng.choice([0, 1, rng.randint(2, 60), rng.randint(60, 900)]) for _ in range(B)]
        lengths[0] = max(lengths[0], 1)
        queries = [rng.choice([0, 1, rng.randint(1, 40), t]) for t in lengths]
        cache, dtype, out = rng.choice(["fp8", "bf16"]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["f32", "bf16"])
        print(f"[case] {i}: {lengths} {queries} P={P} heads={heads} G={G} D={D} {cache} {dtype} {out}", flush=True)
        c, pages, table = make(paged, gen, lengths, P, heads, G, D, cache, dtype, out)
        off = torch.tensor([0] + list(np.cumsum(queries)), dtype=torch.int32)
        if int(off[-1]) == 0:
            continue
        q = torch.randn((int(off[-1]), heads * G, D), generator=gen).to(IO[dtype])
        got = c.attn(dev(q), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)), q_offsets=dev(off))
        torch.cuda.synchronize()
        close(got, *ref.attention(q, pages, table, torch.tensor(lengths), off, D ** -0.5, out), f"case {i}")


def test_a_refused_call_leaves_later_ones_alone(paged):
    # a table wider than 2^24 tokens is refused on the host; the next call of the same batch has its workspace all the same
    c, _, table = make(paged, torch.Generator().manual_seed(3), [300], 16, 2, 4, 64, "fp8", "bf16", "f32")
    q, lens = torch.randn((1, 8, 64), device=DEV).to(torch.bfloat16), torch.tensor([300], dtype=torch.int32, device=DEV)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    c._scratch.streams.pop(stream.cuda_stream, None)
    with pytest.raises(paged.PQCacheError):
        c.attn(q, torch.full((1, (1 << 20) + 1), -1, dtype=torch.int32, device=DEV), lens, stream=stream)
    got = c.attn(q, dev(table), lens, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(got, c.attn(q, dev(table), lens))


def test_threads_on_one_stream_keep_their_scratch_until_the_launch(paged):
    import threading

    c, _, table = make(paged, torch.Generator().manual_seed(4), [300], 16, 2, 4, 64, "fp8", "bf16", "f32")
    d, _, _ = make(paged, torch.Generator().manual_seed(4), [300], 16, 2, 4, 64, "fp8", "bf16", "f32")
    q, lens = torch.zeros((1, 8, 64), dtype=torch.bfloat16, device=DEV), torch.tensor([300], dtype=torch.int32, device=DEV)
    dt, stream = dev(table), torch.cuda.Stream()
    torch.cuda.synchronize()
    c._scratch.streams.pop(stream.cuda_stream, None)
    kept, failed = [], []

    def other():
        try:
            d.attn(q, dt, lens, stream=stream)  # needs more than the call below
        except Exception as e:
            failed.append(e)

    def launch(at, size, raw):  # in place of a launch: nothing runs
        thread.start()
        thread.join(0.5)
        kept.append(c._scratch.streams[raw].ptr == at)
        return 0

    thread = threading.Thread(target=other)
    with torch.cuda.stream(stream):
        c._place(dt, lens, None, 1)
        c._attend("a call", launch, 1, 300, ())
    thread.join()
    torch.cuda.synchronize()
    assert kept == [True] and not failed
