"""Host-only checks of the paged cache: refusals of the C ABI (nothing is launched) and of the binding, workspace sizes."""
import ctypes as C

import pytest
import torch

from paper_2407_12820_amd import paged

P = 4096  # an aligned address that is never read: every call below is refused first


@pytest.fixture(scope="module")
def lib():
    return paged._load()


def config(**kw):
    c = paged.Config(2, 32, 8, 128, 64, 100, 16, 1, 2, 0, 0.0, 128, 0, 2048)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def pages(**kw):
    p = paged.Pages(P, P, P, P, P, P)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def attn(lib, cfg, pg, q=P, n=2, offsets=None, out=P, ws=P, size=1 << 40):
    return lib.pqc_paged_attn(C.byref(cfg) if cfg else None, C.byref(pg) if pg else None, q, n, offsets, out, ws, size, None)


def gather(lib, cfg, pg, q=P, idx=P, n_idx=100, out=P, ws=P, size=1 << 40):
    return lib.pqc_paged_gather_attn(C.byref(cfg) if cfg else None, C.byref(pg) if pg else None, q, idx, n_idx, out, ws, size, None)


def append(lib, cfg, pg, q=P, qs=4096, k=2 * P, ks=1024, v=3 * P, vs=1024, n=2, offsets=None, positions=None, rotation=P, q_out=4 * P, k_out=5 * P):
    return lib.pqc_paged_append(C.byref(cfg) if cfg else None, C.byref(pg) if pg else None, q, qs, k, ks, v, vs, n, offsets, positions, rotation, q_out,
                                k_out, None)


BAD_CONFIGS = [
    (dict(batch=0), -1), (dict(n_q_heads=30), -1), (dict(n_kv_heads=0), -1), (dict(page_tokens=0), -1), (dict(n_pages=0), -1), (dict(max_pages=0), -1),
    (dict(io_dtype=2), -1), (dict(io_dtype=7), -1), (dict(out_dtype=2), -1), (dict(cache_dtype=3), -1), (dict(softmax_scale=float("nan")), -1),
    (dict(softmax_scale=float("inf")), -1), (dict(rot_dims=-16), -1), (dict(rot_dims=144), -1), (dict(rot_positions=0), -1), (dict(rot_style=2), -1),
    (dict(head_dim=96, rot_dims=64), -2), (dict(head_dim=256), -2), (dict(n_q_heads=17 * 8), -2), (dict(cache_dtype=0), -2), (dict(rot_dims=24), -2),
    (dict(page_tokens=8), -2), (dict(page_tokens=48), -2), (dict(page_tokens=512), -2), (dict(batch=65536), -2), (dict(max_pages=(1 << 18) + 1), -2),
    (dict(n_pages=1 << 22), -2),
]


@pytest.mark.parametrize("change,status", BAD_CONFIGS)
def test_refused_configurations(lib, change, status):
    c, n = config(**change), config(**change).batch
    assert attn(lib, c, pages(), n=n) == status
    assert gather(lib, c, pages()) == status
    assert append(lib, c, pages(), n=n) == status
    assert lib.pqc_paged_workspace_bytes(C.byref(c), n, 0) == 0


@pytest.mark.parametrize("change", [dict(k_pages=None), dict(v_pages=None), dict(k_scale=None), dict(v_scale=None), dict(page_table=None), dict(lengths=None),
                                    dict(k_pages=P + 8), dict(v_pages=P + 4), dict(k_scale=P + 4), dict(page_table=P + 2), dict(lengths=P + 1)])
def test_refused_caches(lib, change):
    for call in (attn, gather, append):
        assert call(lib, config(), pages(**change)) == -1
        assert call(lib, config(), None) == -1
        assert call(lib, None, pages()) == -1


def test_refused_arguments_of_the_attention_calls(lib):
    c, p = config(), pages()
    for bad in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 4), dict(n=3), dict(n=-1), dict(offsets=P + 2)):
        assert attn(lib, c, p, **bad) == -1, bad
    assert attn(lib, c, p, n=1 << 27, offsets=P) == -2
    need = lib.pqc_paged_workspace_bytes(C.byref(c), 2, 0)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=P + 16), dict(size=need - 1)):
        assert attn(lib, c, p, **bad) == -3, bad
    for bad in (dict(q=None), dict(out=None), dict(idx=None), dict(n_idx=0), dict(n_idx=-5), dict(idx=P + 2)):
        assert gather(lib, c, p, **bad) == -1, bad
    assert gather(lib, c, p, n_idx=(1 << 24) + 1) == -2
    need = lib.pqc_paged_workspace_bytes(C.byref(c), 2, 5000)
    assert need > 0
    assert gather(lib, c, p, n_idx=5000, size=need - 1) == -3
    assert lib.pqc_paged_workspace_bytes(C.byref(c), 2, -1) == 0


def test_refused_arguments_of_append(lib):
    c, p = config(), pages()
    for bad in (dict(k=None), dict(v=None), dict(q_out=None), dict(rotation=None), dict(n=3), dict(ks=1016), dict(vs=1020), dict(ks=1028), dict(qs=4088),
                dict(k=P + 8), dict(q=P + 2), dict(q_out=P + 4), dict(k_out=P + 4), dict(positions=P + 1), dict(q_out=P), dict(k_out=2 * P), dict(k_out=3 * P),
                dict(k_out=4 * P)):
        assert append(lib, c, p, **bad) == -1, bad
    # without rotation no table is needed, without q no output for it: an empty call is accepted and does nothing
    assert append(lib, config(rot_dims=0, rot_positions=0), p, rotation=None, q=None, q_out=None, n=0, offsets=P) == 0
    assert append(lib, c, p, n=0, offsets=P) == 0
    assert attn(lib, c, p, n=0, offsets=P) == 0


def test_workspace_grows_with_neither_tokens_nor_pages(lib):
    sizes = {lib.pqc_paged_workspace_bytes(C.byref(config(batch=b, max_pages=m)), n, 0) for b, m, n in ((1, 1, 1), (64, 4096, 64), (3, 2000, 8192))}
    assert len(sizes) == 1 and 0 < sizes.pop() <= 64 << 20
    # a list that one workgroup takes needs none
    assert lib.pqc_paged_workspace_bytes(C.byref(config()), 2, 100) == 0


def test_counters_are_enough_for_calls_of_any_size(lib):
    # one word per border between workers and head; the most workers that any call has: 512 over all heads, one per head at least
    for heads, words in ((1, 512), (2, 512), (3, 510), (8, 512), (96, 480), (600, 600)):
        for most in (1, 16, 4096):
            c = config(n_q_heads=heads, n_kv_heads=heads, max_pages=most)
            assert lib.pqc_paged_counter_bytes(C.byref(c)) == 4 * words, (heads, most)
    assert lib.pqc_paged_counter_bytes(C.byref(config(head_dim=80, rot_dims=64))) == 0
    assert attn(lib, config(), pages(counters=P + 2)) == -1


def test_the_binding_says_what_is_wrong():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = paged.PagedCache(k, k.clone(), None, None, n_q_heads=4)
    table, lengths = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    idx = torch.zeros((2, 2, 5), dtype=torch.int32)
    bad = [
        lambda: cache.append(x.float(), x, table, lengths), lambda: cache.append(x, x[:1], table, lengths), lambda: cache.append(x, x, table.long(), lengths),
        lambda: cache.append(x, x, table, lengths[:1]), lambda: cache.append(x, x, table, lengths, new_offsets=torch.zeros(2, dtype=torch.int32)),
        lambda: cache.append(x, x, table, lengths, q=q[:, :3]), lambda: cache.append(x.transpose(0, 1), x, table, lengths),
        lambda: cache.append(x, x, table, lengths, k_out=x.float()), lambda: cache.append(x, x, table, lengths, positions=torch.zeros(2)),
        lambda: cache.append(torch.cat([x, x]), torch.cat([x, x]), table, lengths),
        lambda: cache.attn(q.float(), table, lengths), lambda: cache.attn(q[:, :2], table, lengths), lambda: cache.attn(q, table, lengths, out=q),
        lambda: cache.attn(torch.cat([q, q]), table, lengths), lambda: cache.gather_attn(q, idx[:, :1], table, lengths),
        lambda: cache.gather_attn(q, idx[:, :, :0], table, lengths), lambda: cache.gather_attn(q, idx.long(), table, lengths),
        lambda: cache.attn(q, table, lengths),  # everything in order but on the CPU
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")
    f8 = torch.zeros((4, 2, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.ones((4, 2))
    for make in (lambda: paged.PagedCache(f8, f8, None, None, n_q_heads=4), lambda: paged.PagedCache(f8, f8, s, s[:2], n_q_heads=4),
                 lambda: paged.PagedCache(k.float(), k.float(), None, None, n_q_heads=4), lambda: paged.PagedCache(k[0], k[0], None, None, n_q_heads=4),
                 lambda: paged.PagedCache(k, k[:2], None, None, n_q_heads=4), lambda: paged.PagedCache(k, k, None, None, n_q_heads=4, rotation=s.double())):
        with pytest.raises(ValueError):
            make()


def test_rotation_table():
    t = paged.rotation_table(1000, 64, base=500000.0, device="cpu")
    assert t.shape == (1000, 64) and t.dtype is torch.float32
    angle = 999.0 * 500000.0 ** (-2.0 * 5 / 64)
    assert abs(float(t[999, 5]) - torch.tensor(angle, dtype=torch.float64).cos().item()) < 1e-7
    assert abs(float(t[999, 32 + 5]) - torch.tensor(angle, dtype=torch.float64).sin().item()) < 1e-7


def test_streams_of_other_devices_and_outputs_over_inputs_are_refused():
    from types import SimpleNamespace

    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = paged.PagedCache(k, k.clone(), None, None, n_q_heads=4, out_dtype="bf16")
    table, lengths = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    x, q, idx = (torch.zeros((2, h, 64), dtype=torch.bfloat16) for h in (2, 4, 2))
    idx = idx[:, :, :5].int().contiguous()
    far = SimpleNamespace(device=torch.device("cuda", 1))
    for call in (lambda: cache.append(x, x, table, lengths, stream=far), lambda: cache.attn(q, table, lengths, stream=far),
                 lambda: cache.gather_attn(q, idx, table, lengths, stream=far)):
        with pytest.raises(ValueError, match="stream"):
            call()
    for call in (lambda: cache.attn(q, table, lengths, out=q), lambda: cache.gather_attn(q, idx, table, lengths, out=q)):
        with pytest.raises(ValueError, match="overlap"):
            call()


def test_calls_that_no_launch_takes_are_refused(lib):
    # 2^32 work items: 2^25 tokens are 8.4 million workgroups for keys and values and 16.8 million for queries
    assert append(lib, config(), pages(), n=1 << 25, offsets=P) == -2
    # tiles of 128 rows of 65535 sequences, 300 heads
    c = config(batch=65535, n_q_heads=300, n_kv_heads=300)
    assert attn(lib, c, pages(), n=64 * 65535, offsets=P) == -2
