"""Tests of how exactly softmax weights enter the product with the values in attention over a paged cache."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged import DEV, IO, dev, paged, place  # noqa: F401  (paged: fixture)

gpu = pytest.mark.gpu
U = ref.U


def half_step(x):
    """Half the spacing of bf16 (8 significant bits) around x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=1e-30))) - 8.0)


def two_tokens(form, gen, D, cache, dtype):
    """Queries that see a token of weight 1 and value 0 and one of weight w in (1/2, 1), all else with a weight of 0: the result is
    w / (1 + w) of the second one's value.  -> (pages, table, lengths, offsets, q, the queries' logits)."""
    P, G = 64, 4
    m = {"one": 1, "listed": 1, "rows": 5, "block": 40}[form]
    B = {"one": 160, "listed": 160, "rows": 40, "block": 16}[form]
    k = torch.zeros((1, 1, P, D))
    v = torch.randn((1, 1, P, D), generator=gen)
    k[..., 1, 0] = 1.0
    k[..., 2:, 1] = -256.0  # logits of -65536
    v[..., 0, :] = 0.0
    v[..., 1, :] = torch.exp2(torch.randint(-3, 4, (D,), generator=gen).float())
    t = IO["bf16"] if cache == "bf16" else torch.float8_e4m3fn
    one = None if cache == "bf16" else torch.ones((1, 1))
    pages = (k.to(t), v.to(t), one, one)
    a = -0.69 * torch.rand((B * m, G), generator=gen)
    q = torch.zeros((B * m, G, D))
    q[..., 0], q[..., 1] = a, 256.0
    q = q.to(IO[dtype])
    table = torch.zeros((B, 1), dtype=torch.int32)
    lengths = torch.full((B,), m + 1, dtype=torch.int32)  # the first query of a sequence sees two tokens, later ones more
    offsets = None if m == 1 else m * torch.arange(B + 1, dtype=torch.int32)
    return pages, table, lengths, offsets, q


def run(paged, form, pages, table, lengths, offsets, q, dtype, out):
    c = paged.PagedCache(*(dev(x) for x in pages), n_q_heads=q.shape[1], dtype=dtype, out_dtype=out, softmax_scale=1.0)
    if form == "listed":
        idx = torch.tensor([1, 0], dtype=torch.int32).expand(q.shape[0], 1, 2).contiguous()
        return c.gather_attn(dev(q), dev(idx), dev(table), dev(lengths))
    return c.attn(dev(q), dev(table), dev(lengths), q_offsets=dev(offsets))


def tolerance(want, out):
    """Base-2 logits of at most 1 in size carry 5 roundings (the scale's factors, the product, for fp32 queries two sums of terms),
    the difference to the maximum one and exp2 two: 10 U of the weight at most, 20 U of the result in numerator and denominator.
    Three products with a weight's terms, two sums, folding and the division: 12 U.  A weight as three bf16 terms is exact (8 bits
    each); as two it is off by up to 2^-17, which only a bf16 output (8 bits) may have."""
    if out == "f32":
        return 32 * U * want.abs() + 1e-30
    return half_step(want) + (32 * U + 2.0 ** -17) * want.abs() + 1e-30


FORMS = ["one", "listed", "rows", "block"]


@gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,cache", [(128, "fp8"), (64, "bf16")])
@pytest.mark.parametrize("form", FORMS)
def test_weights_keep_their_bits(paged, form, D, cache, dtype, out):
    gen = torch.Generator().manual_seed(D + len(form))
    pages, table, lengths, offsets, q = two_tokens(form, gen, D, cache, dtype)
    print(f"[case] {form} D={D} {cache} {dtype} {out}", flush=True)
    got = run(paged, form, pages, table, lengths, offsets, q, dtype, out).double().cpu()
    w = torch.exp(q[..., 0].double())
    want = (w / (1.0 + w))[..., None] * pages[1][0, 0, 1].float().double()
    over = (got - want).abs() / tolerance(want, out)
    assert over.max().item() <= 1.0, f"{over.max().item()} times the tolerance"


def test_the_tolerance_tells_terms_apart():
    # on the CPU: with one bf16 term fewer than the kernels take, the results above leave the tolerance
    gen = torch.Generator().manual_seed(5)
    w = torch.exp(-0.69 * torch.rand(640, generator=gen).bfloat16().double()).float()
    want = (w.double() / (1.0 + w.double()))

    def kept(n):
        rest, held = w.clone(), torch.zeros_like(w, dtype=torch.float64)
        for _ in range(n):
            x = rest.bfloat16().float()
            held += x.double()
            rest -= x
        return held / (1.0 + w.double())

    assert bool(((kept(3) - want).abs() <= tolerance(want, "f32")).all())
    assert bool(((kept(2) - want).abs() > tolerance(want, "f32")).any())
    rounded = [kept(n).float().bfloat16().double() for n in (1, 2)]
    assert bool(((rounded[1] - want).abs() <= tolerance(want, "bf16")).all())
    assert bool(((rounded[0] - want).abs() > tolerance(want, "bf16")).any())


def attention64(q, pages, table, lengths, offsets, scale):
    """Causal attention in 64 bits on the GPU, head by head."""
    k_pages, v_pages, ks, vs = pages
    n, Hq, D = q.shape
    G = Hq // k_pages.shape[1]
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device=DEV)
    for b in range(lengths.shape[0]):
        lo, hi, t = int(offsets[b]), int(offsets[b + 1]), int(lengths[b])
        hidden = torch.ones((hi - lo, t), dtype=torch.bool, device=DEV).triu_(t - (hi - lo) + 1)
        for h in range(k_pages.shape[1]):
            k, v = (dev(ref.rows_of(x, s, table[b], h, t)[0]) for x, s in ((k_pages, ks), (v_pages, vs)))
            for g in range(h * G, h * G + G):
                w = (dev(q[lo:hi, g].double()) @ k.T.contiguous()).mul_(scale).masked_fill_(hidden, float("-inf"))
                out[lo:hi, g] = torch.softmax(w, -1) @ v
    return out


PROMPTS = [  # lengths, queries, P, heads, G, D, cache, dtype, out: prompts as long as the ones that are timed, pieces of prompts
    ([8192, 390], [8192, 3], 128, 1, 2, 128, "fp8", "bf16", "bf16"),
    ([2900, 4100], [1024, 1100], 64, 2, 4, 128, "fp8", "bf16", "bf16"),
    ([5000], [5000], 16, 1, 1, 64, "bf16", "bf16", "bf16"),
    ([2100, 1700], [2100, 900], 64, 1, 3, 128, "bf16", "f32", "bf16"),
    ([4500, 20], [4500, 20], 64, 1, 2, 128, "fp8", "bf16", "f32"),
    ([2500], [2500], 32, 1, 4, 128, "fp8", "f32", "f32"),
]


@gpu
@pytest.mark.parametrize("lengths,queries,P,heads,G,D,cache,dtype,out", PROMPTS)
def test_long_prompts(paged, lengths, queries, P, heads, G, D, cache, dtype, out):
    """A bf16 result is off by its own rounding and little else: the fp32 value in front of it is off by e, |e| far below half a step,
    so that the error's square sum is that of the exact result's rounding and of e, and of changed roundings next to a border (e in
    size there).  5 % leave e a third of the rounding; weights as one bf16 term add 25 % and more."""
    gen = torch.Generator().manual_seed(sum(lengths) + P)
    table, n_pages = place(lengths, P, gen)
    k, ks = ref.fill_pool(n_pages, heads, P, D, cache, gen)
    v, vs = ref.fill_pool(n_pages, heads, P, D, cache, gen)
    ks = None if ks is None else ks / 64.0
    off = torch.tensor([0] + torch.tensor(queries).cumsum(0).tolist(), dtype=torch.int32)
    q = torch.randn((int(off[-1]), heads * G, D), generator=gen).to(IO[dtype])
    c = paged.PagedCache(dev(k), dev(v), dev(ks), dev(vs), n_q_heads=heads * G, dtype=dtype, out_dtype=out)
    print(f"[case] {lengths} {queries} P={P} heads={heads} G={G} D={D} {cache} {dtype} {out}", flush=True)
    got = c.attn(dev(q), dev(table), dev(torch.tensor(lengths, dtype=torch.int32)), q_offsets=dev(off)).double()
    want = attention64(q, (k, v, ks, vs), table, torch.tensor(lengths), off, D ** -0.5)
    error = (got - want).norm()
    if out == "bf16":
        assert error <= 1.05 * (want.float().bfloat16().double() - want).norm(), (error / want.norm()).item()
    else:
        # a logit's D products of fp32 roundings add up like a random walk, about 11 U of it, which moves result and sum alike; as many
        # again for the weighted sums: 32 U
        assert error <= 2.0 ** -19 * want.norm(), (error / want.norm()).item()
