"""GPU tests of where the operands of calls on the paged cache may lie, and of the forms of append that long calls take."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged import DEV, IO, close, dev, paged, place  # noqa: F401  (paged: fixture)

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
