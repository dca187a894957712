"""GPU tests of NaN and infinities around the paged cache: they reach the results they belong to, and no others."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged import DEV, IO, close, dev, make, paged, place  # noqa: F401  (paged: fixture)

pytestmark = pytest.mark.gpu

# ------------------------------------------------------------------ attention
SHAPES = {  # lengths, query tokens per sequence (0: one, without offsets), listed tokens, heads, G: which way a tile goes
    "one, whole": ([50, 90], 0, 0, 2, 4),
    "one, folded": ([2048, 700], 0, 0, 8, 4),
    "one, folded by a kernel": ([20011, 700], 0, 0, 1, 4),
    "listed, whole": ([300, 90], 0, 60, 2, 4),
    "listed, folded": ([2500, 1800], 0, 1700, 8, 4),
    "rows, whole": ([100, 60], 6, 0, 2, 4),
    "rows, folded": ([6000, 3000], 6, 0, 2, 4),
    "block, whole": ([300, 150], 70, 0, 2, 4),
    "block, split": ([5000, 700], 50, 0, 1, 4),
}


class Call:
    """One call of a shape on finite inputs, whose keys, values and queries a test then spoils."""

    def __init__(self, paged, shape, cache, dtype="bf16", out="f32", seed=1):
        self.lengths, self.several, count, self.heads, self.G = SHAPES[shape]
        self.gen = torch.Generator().manual_seed(seed)
        self.c, self.pages, self.table = make(paged, self.gen, self.lengths, 64, self.heads, self.G, 128, cache, dtype, out)
        B = len(self.lengths)
        self.offsets = self.several * torch.arange(B + 1, dtype=torch.int32) if self.several else None
        self.m = self.several or 1
        self.q = torch.randn((B * self.m, self.heads * self.G, 128), generator=self.gen).to(IO[dtype])
        self.out = out
        self.idx = None
        if count:
            self.idx = torch.full((B, self.heads, count), -1, dtype=torch.int32)
            for b, t in enumerate(self.lengths):
                self.idx[b, :, :min(t, count)] = torch.randperm(t, generator=self.gen)[:count].int()

    def run(self):
        lens = dev(torch.tensor(self.lengths, dtype=torch.int32))
        if self.idx is not None:
            return self.c.gather_attn(dev(self.q), dev(self.idx), dev(self.table), lens)
        return self.c.attn(dev(self.q), dev(self.table), lens, q_offsets=dev(self.offsets))

    def expected(self):
        return ref.attention(self.q, self.pages, self.table, torch.tensor(self.lengths), self.offsets, 128 ** -0.5, self.out, listed=self.idx)

    def spoil(self, name, b, token, h, dim=None, value=float("nan")):
        """One value, or all, of a cached row on the device; what the reference reads stays finite."""
        pool = self.c.k_pages if name == "k" else self.c.v_pages
        page, slot = int(self.table[b, token // 64]), token % 64
        row = pool[page, h, slot].float()
        row[slice(None) if dim is None else dim] = value
        pool[page, h, slot] = row.to(pool.dtype)

    def seeing(self, b, token, h):
        """Rows [n][Hq] of sequence b and KV head h that see the token."""
        sees = torch.zeros(self.q.shape[:2], dtype=torch.bool)
        for i in range(self.m):
            if token <= self.lengths[b] - self.m + i:
                sees[b * self.m + i, h * self.G:(h + 1) * self.G] = True
        return sees


def check(call, spoiled, what):
    """Rows `spoiled` ([n][Hq], or with a last axis of dimensions) are NaN, the others as they were."""
    want, tol = call.expected()
    got = call.run()
    torch.cuda.synchronize()
    mask = (spoiled if spoiled.dim() == 3 else spoiled[..., None]).expand_as(want)
    nan = torch.isnan(got.cpu())
    assert bool(nan[mask].all()), f"{what}: {int((~nan[mask]).sum())} of {int(mask.sum())} values are not NaN"
    close(got, want.masked_fill(mask, float("nan")), tol, what)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_query_that_is_not_a_number(paged, shape, cache):
    call = Call(paged, shape, cache)
    row = call.q.shape[0] - 1 if call.m == 1 else 2
    print(f"[case] {shape} {cache}", flush=True)
    spoiled = torch.zeros(call.q.shape[:2], dtype=torch.bool)
    spoiled[row, 1] = True
    want = call.expected()
    call.expected = lambda: want
    call.q[row, 1, 77] = float("nan")
    check(call, spoiled, shape)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_key_that_is_not_a_number(paged, shape, cache):
    call = Call(paged, shape, cache)
    last = call.lengths[0] - 1
    tokens = [int(call.idx[0, 1, 3])] if call.idx is not None else [last] if call.m == 1 else [last - 2]  # the last two or three queries see it
    h = call.heads - 1
    print(f"[case] {shape} {cache}", flush=True)
    if call.idx is not None:
        tokens = [int(call.idx[0, h, 3])]
    call.spoil("k", 0, tokens[0], h, dim=5)
    check(call, call.seeing(0, tokens[0], h), shape)
    call.spoil("k", 0, 0 if call.idx is None else tokens[0], h, dim=9)  # and one that all of them see
    check(call, call.seeing(0, 0, h), shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_an_infinite_logit(paged, shape, dtype):
    # exp(inf - inf): the softmax of a row with a logit of +inf is not a number
    call = Call(paged, shape, "bf16", dtype)
    call.q[..., 5] = call.q[..., 5].abs() + 0.5
    h, token = call.heads - 1, call.lengths[0] // 2
    if call.idx is not None:
        token = int(call.idx[0, h, 7])
    print(f"[case] {shape} {dtype}", flush=True)
    call.spoil("k", 0, token, h, dim=5, value=float("inf"))
    check(call, call.seeing(0, token, h), shape)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_value_that_is_not_a_number(paged, shape, cache, out):
    call = Call(paged, shape, cache, out=out)
    h, token = call.heads - 1, 0
    if call.idx is not None:
        token = int(call.idx[0, h, 7])
    print(f"[case] {shape} {cache} {out}", flush=True)
    call.spoil("v", 0, token, h, dim=37)
    spoiled = call.seeing(0, token, h)[..., None] & (torch.arange(128) == 37)
    check(call, spoiled, shape)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("cache,value", [("fp8", float("nan")), ("bf16", float("nan")), ("bf16", float("inf"))])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s.startswith(("rows", "block"))])
def test_a_value_behind_a_query_is_not_its_own(paged, shape, cache, value, out):
    # tokens that only some queries of a tile see: the others give them a weight of nothing, which must not meet the value
    call = Call(paged, shape, cache, out=out)
    h, last = call.heads - 1, call.lengths[0] - 1
    print(f"[case] {shape} {cache} {out} {value}", flush=True)
    spoiled = torch.zeros((*call.q.shape[:2], 128), dtype=torch.bool)
    for token, dim in ((last, 3), (last - 1, 64), (last - call.m + 3, 127), (last - call.m // 2, 70)):
        call.spoil("v", 0, token, h, dim=dim, value=value)
        spoiled |= call.seeing(0, token, h)[..., None] & (torch.arange(128) == dim)
    want, tol = call.expected()
    got = call.run().cpu()
    assert not bool(torch.isfinite(got)[spoiled].any())
    close(got, want.masked_fill(spoiled, float("nan")), tol, shape)


# ------------------------------------------------------------------ append
def is_nan_code(pages):
    return (pages.view(torch.uint8) & 0x7F) == 0x7F


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinity_leaves_the_other_tokens_of_its_page(paged, dtype, D):
    """Scales are those of the finite values; what is not finite is a NaN of the type, in its own places alone."""
    gen = torch.Generator().manual_seed(8)
    P, heads, inf = 64, 2, float("inf")
    c = paged.PagedCache.empty(2, heads, heads, D, P, dtype=dtype, device=DEV)
    table = torch.tensor([[1]], dtype=torch.int32, device=DEV)
    x = torch.randn((60, heads, D), generator=gen)
    x[41] *= 8.0                                 # the scale grows in the same call as the infinities come
    bad = torch.zeros_like(x, dtype=torch.bool)
    for at, value in (((40, 0, 3), inf), ((41, 0, D - 1), -inf), ((41, 1, 17), inf), ((45, 1, 20), float("nan"))):
        x[at], bad[at] = value, True
    x[50, 0], bad[50, 0] = -inf, True            # a token without a finite value
    x = x.to(IO[dtype])
    done = 0
    for n in (20, 20, 2, 1, 5, 1, 1, 1, 9):      # the page's first call, then ones on top of what it holds
        part = dev(x[done:done + n].contiguous())
        done += n
        off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        c.append(part, part, table, torch.tensor([done], dtype=torch.int32, device=DEV), new_offsets=off)
    torch.cuda.synchronize()
    finite = x[:done].double().masked_fill(bad[:done], 0.0)
    for pool, scale in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
        got = ref.dequantised(pool.cpu(), scale.cpu())[1].transpose(0, 1)[:done]
        assert torch.equal(is_nan_code(pool.cpu())[1].transpose(0, 1)[:done], bad[:done])
        for h in range(heads):
            s = ref.power_scale(float(finite[:, h].abs().max()))
            assert float(scale[1, h]) == s
            want = finite[:, h]
            # as in a page that is filled token by token: half a step of e4m3, less than one step of the last subnormals
            err = (got[:, h] - want).abs().masked_fill(bad[:done, h], 0.0)
            assert bool((err <= 2.0 ** -4 * want.abs() + 2.0 ** -9 * s).all())


def test_a_page_that_begins_with_an_infinity(paged):
    gen = torch.Generator().manual_seed(9)
    c = paged.PagedCache.empty(1, 1, 1, 64, 16, device=DEV)
    c.k_scale.fill_(float("nan"))
    x = torch.randn((2, 1, 64), generator=gen).to(torch.bfloat16)
    first = torch.full((1, 1, 64), float("inf"), dtype=torch.bfloat16)
    table, at = torch.zeros((1, 1), dtype=torch.int32, device=DEV), lambda n: torch.tensor([n], dtype=torch.int32, device=DEV)
    c.append(dev(first), dev(first), table, at(1))
    assert bool(is_nan_code(c.k_pages)[0, 0, 0].all()) and float(c.k_scale) == 2.0 ** -100
    for i in range(2):
        c.append(dev(x[i:i + 1]), dev(x[i:i + 1]), table, at(2 + i))
    torch.cuda.synchronize()
    s = ref.power_scale(float(x.double().abs().max()))
    assert float(c.k_scale) == s and bool(is_nan_code(c.k_pages)[0, 0, 0].all())
    got = ref.dequantised(c.k_pages.cpu(), c.k_scale.cpu())[0, 0, 1:3]
    assert bool(((got - x[:, 0].double()).abs() <= 2.0 ** -4 * x[:, 0].double().abs() + 2.0 ** -9 * s).all())


# ------------------------------------------------------------------ logits of any size
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_logits_of_any_finite_size(paged, shape, dtype, sign):
    """Logits of 2^30 to 2^110, all of one sign: the softmax is that of equal or far apart numbers, never of masked ones."""
    call = Call(paged, shape, "bf16", dtype)
    call.q[:] = 0.0
    call.q[..., 3] = 1.3359375 * torch.exp2(torch.randint(-20, 61, call.q.shape[:2], generator=call.gen).float())
    h, best = call.heads - 1, call.lengths[0] // 3
    if call.idx is not None:
        best = int(call.idx[0, h, 11])
    print(f"[case] {shape} {dtype} {sign}", flush=True)
    k = call.pages[0]
    k[...] = 0.0
    k[..., 3] = sign * 1.6328125 * 2.0 ** 53
    # one head of the first sequence has a token far ahead of the others, the rest equal logits
    k[int(call.table[0, best // 64]), h, best % 64, 3] = sign * 2.0 ** 54 * (1.5 if sign > 0 else 0.5)
    call.c.k_pages.copy_(k)
    want, _ = call.expected()
    got = call.run().double().cpu()
    # every product and every logit is exact or equal to its like, weights are 1 or 0: what is left are the sums (values of up to 5 in size)
    assert (got - want).abs().max().item() <= 5 * (max(call.lengths) / 4 + 64) * ref.U
