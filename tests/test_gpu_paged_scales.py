"""GPU tests of pools whose scales another program chose: any positive scale, in every form of attention."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged import DEV, IO, close, dev, paged, place  # noqa: F401  (paged: fixture)

pytestmark = pytest.mark.gpu

FORMS = [  # lengths, query tokens per sequence (0: one), listed, heads, G, D, P, dtype, out
    ([300, 90], 0, 0, 2, 4, 128, 64, "bf16", "f32"),
    ([2500, 700], 0, 900, 2, 4, 128, 16, "bf16", "f32"),
    ([1000, 60], 5, 0, 2, 4, 128, 32, "bf16", "f32"),
    ([900, 150], 70, 0, 2, 4, 128, 16, "bf16", "f32"),
    ([700, 90], 70, 0, 1, 3, 64, 128, "bf16", "bf16"),
    ([3000, 70], 70, 0, 1, 5, 128, 32, "bf16", "bf16"),
    ([400, 100], 90, 0, 2, 2, 128, 64, "f32", "f32"),
    ([400, 100], 90, 0, 1, 7, 64, 16, "f32", "bf16"),
]


@pytest.mark.parametrize("some", [False, True])
@pytest.mark.parametrize("lengths,several,count,heads,G,D,P,dtype,out", FORMS)
def test_scales_that_are_no_powers_of_two(paged, lengths, several, count, heads, G, D, P, dtype, out, some):
    """Largest value / 448, as pools are quantised elsewhere; `some`: among pages whose scales are powers of two."""
    gen = torch.Generator().manual_seed(sum(lengths) + P)
    table, n_pages = place(lengths, P, gen)
    pools = []
    for size in (1.0, 3.0):
        x = size * torch.randn((n_pages, heads, P, D), generator=gen) * torch.exp2(torch.randint(-2, 3, (n_pages, heads, 1, 1), generator=gen).float())
        s = x.abs().amax((2, 3)) / 448.0
        if some:
            s = torch.where(torch.rand(s.shape, generator=gen) < 0.7, torch.exp2(torch.ceil(torch.log2(s))), s)
        pools.append(((x / s[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn), s))
    (k, ks), (v, vs) = pools
    B, m = len(lengths), several or 1
    off = several * torch.arange(B + 1, dtype=torch.int32) if several else None
    q = torch.randn((B * m, heads * G, D), generator=gen).to(IO[dtype])
    lens = torch.tensor(lengths, dtype=torch.int32)
    c = paged.PagedCache(dev(k), dev(v), dev(ks), dev(vs), n_q_heads=heads * G, dtype=dtype, out_dtype=out)
    print(f"[case] {lengths} {several} {count} {heads} {G} D={D} P={P} {dtype} {out} {some}", flush=True)
    idx = None
    if count:
        idx = torch.randint(0, max(lengths), (B, heads, count), generator=gen).int()
        got = c.gather_attn(dev(q), dev(idx), dev(table), dev(lens))
    else:
        got = c.attn(dev(q), dev(table), dev(lens), q_offsets=dev(off))
    torch.cuda.synchronize()
    # (the reference's factors of a logit and of a weight count the scale's rounding already)
    close(got, *ref.attention(q, (k, v, ks, vs), table, lens, off, D ** -0.5, out, listed=idx))
