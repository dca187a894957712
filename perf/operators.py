"""Operators around a paged key/value cache, as cases that can be timed and compared.

A serving program keeps the keys and values of sequences of different lengths in pages of a common pool, in bf16 or in
8 bits (e4m3) with one scale per page and head.  Three operators work on it: `append` rotates new keys (and queries) by
their positions and writes keys and values into the pages, `attn` attends to all tokens of each sequence (one query per
sequence in decoding, many with a causal mask for prompts), `listed` attends to a list of tokens per head, as a retrieval
step selects them.

Case fields: kind (append, attn, listed), heads and head_dim, `page` tokens per page, `tokens` (the longest sequence),
`new` (the most query or appended tokens of a sequence), `ragged` (whether sequences differ), `dtype` of q, k, v, `out` of
the attention, `cache` (fp8 or bf16), `rot` dimensions and `style` of the rotation, `count` listed tokens per head.
"""
import random

import torch

own = False

DEV = "cuda:0"
FP8_MAX = 448.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def _case(name, kind, batch, q_heads, kv_heads, tokens, new=1, page=64, head_dim=128, ragged=False, dtype="bf16", cache="fp8",
          out="f32", rot=128, style="halves", count=0, keys_out=True):
    c = dict(kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=page, tokens=tokens, new=new,
             ragged=ragged, dtype=dtype, cache=cache)
    if kind == "append":
        c.update(rot=rot, style=style, keys_out=keys_out)
    else:
        c.update(out=out)
    if kind == "listed":
        c.update(count=count)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token of one sequence joins its cache: the smallest call, launches and latency
        _case("append_one_token", "append", 1, 32, 8, 32768),
        # a decode step of 64 sequences of different lengths, each with one new token
        _case("append_batch_tokens", "append", 64, 64, 8, 16384, page=128, ragged=True),
        # the end of a prompt of 32K tokens: all its keys and values enter the cache
        _case("append_prompt_32k", "append", 1, 32, 8, 32768, new=32768),
        # prompts of odd lengths in single precision, interleaved partial rotation, a bf16 cache of small pages and heads
        _case("append_ragged_f32", "append", 5, 8, 2, 9001, new=3001, page=16, head_dim=64, ragged=True, dtype="f32", cache="bf16",
              rot=32, style="pairs", keys_out=False),
        # decoding with a short cache: latency
        _case("attn_one_4k", "attn", 1, 32, 8, 4096),
        # decoding with 128K tokens of context in 8 bits
        _case("attn_one_128k", "attn", 1, 32, 8, 131072),
        # continuous batching: 48 sequences from a few tokens to 16K, small pages, eight query heads per key head
        _case("attn_batch_ragged", "attn", 48, 64, 8, 16384, page=16, ragged=True),
        # a bf16 cache of eight sequences, as decoding had it before 8 bits
        _case("attn_bf16_cache", "attn", 8, 32, 8, 32768, page=128, cache="bf16"),
        # a piece of a long prompt: 1024 queries on top of what is cached
        _case("attn_piece_of_prompt", "attn", 1, 32, 8, 32768, new=1024, out="bf16"),
        # whole prompts of up to 8K tokens
        _case("attn_prompts_8k", "attn", 2, 32, 8, 8192, new=8192, page=128, ragged=True, out="bf16"),
        # attention to the tenth of 128K tokens that a retrieval step selected
        _case("listed_8b_128k", "listed", 1, 32, 8, 131072, count=13175),
        # the same for four sequences with eight query heads per key head
        _case("listed_70b_128k", "listed", 4, 64, 8, 131072, count=13175),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(["append"] * 3 + ["attn"] * 5 + ["listed"] * 2)
        kv_heads = rng.choice([1, 2, 4, 8, 8, 8])
        group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
        batch = rng.choice([1, 1, 2, 3, 4, 8, 17, 33, 64])
        tokens = _log_int(rng, 16, 131072)
        new = 1 if kind == "listed" or rng.random() < 0.5 else min(tokens, _log_int(rng, 2, 8192))
        head_dim = rng.choice([128, 128, 128, 64])
        c = _case("", kind, batch, group * kv_heads, kv_heads, tokens, new=new, page=rng.choice([16, 32, 64, 64, 128, 256]),
                  head_dim=head_dim, ragged=batch > 1 and rng.random() < 0.6, dtype="f32" if rng.random() < 0.15 else "bf16",
                  cache="bf16" if rng.random() < 0.25 else "fp8", out=rng.choice(["f32", "bf16"]),
                  rot=rng.choice([head_dim, head_dim, head_dim // 2]), style=rng.choice(["halves", "halves", "pairs"]),
                  count=max(1, min(tokens, tokens // rng.choice([2, 5, 10, 10, 20]) + 68)), keys_out=rng.random() < 0.7)
        e = 1 if c["cache"] == "fp8" else 2
        held = batch * kv_heads * tokens * head_dim * 2 * e
        if _cost(c) <= most[kind] and held <= 1.2e9 and batch * c["q_heads"] * new * tokens <= 2.2e9:
            return c


# ------------------------------------------------------------------------- geometry
def _lengths(c):
    """(tokens in the cache after the call, tokens that are new or that query) of every sequence."""
    if not c["ragged"]:
        return [c["tokens"]] * c["batch"], [c["new"]] * c["batch"]
    rng = random.Random(c["tokens"] * 1000003 + c["new"] * 1009 + c["batch"])
    total = [c["tokens"]] + [_log_int(rng, 1, c["tokens"]) for _ in range(c["batch"] - 1)]
    new = [c["new"]] + [_log_int(rng, 1, c["new"]) for _ in range(c["batch"] - 1)]
    return total, [min(n, t) for n, t in zip(new, total)]


def _pairs(total, new):
    """(query, token) pairs that the causal mask leaves."""
    return sum(n * t - n * (n - 1) // 2 for t, n in zip(total, new))


def work(case):
    c = case
    total, new = _lengths(c)
    e = 4 if c["dtype"] == "f32" else 2
    ce = 1 if c["cache"] == "fp8" else 2
    n, D, Hq, Hkv = sum(new), c["head_dim"], c["q_heads"], c["kv_heads"]
    if c["kind"] == "append":
        moved = n * D * ((Hq + 2 * Hkv) * e + Hq * e + (Hkv * e if c["keys_out"] else 0) + 2 * Hkv * ce) + n * c["rot"] * 4
        return {"bytes": moved, "flops": n * (Hq + Hkv) * c["rot"] * 3.0 + n * 2 * Hkv * D * 2.0}
    io = n * Hq * D * (e + (4 if c["out"] == "f32" else 2))
    scale = 8.0 / c["page"] if c["cache"] == "fp8" else 0.0  # two scales of four bytes per page
    if c["kind"] == "listed":
        rows = sum(min(c["count"], t) for t in total) * Hkv
        scales = min(rows * 8.0, sum(-(-t // c["page"]) for t in total) * Hkv * 8.0) if c["cache"] == "fp8" else 0.0
        return {"bytes": rows * 2 * D * ce + scales + len(total) * Hkv * c["count"] * 4 + io, "flops": rows * (Hq // Hkv) * D * 4.0}
    rows = sum(total) * Hkv
    return {"bytes": rows * (2 * D * ce + scale) + io, "flops": _pairs(total, new) * Hq * D * 4.0}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 3e14)


# ------------------------------------------------------------------------- inputs
def _power_scale(amax):
    """Smallest power of two s with amax <= 448 s (448 = 0.875 * 2^9), not below 2^-100."""
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875)).clamp(min=-100)
    return torch.ldexp(torch.ones_like(amax), e)


def _fill(c, x):
    """Pages [n][Hkv][P][D] of float values -> (pages as the cache holds them, scales [n][Hkv])."""
    if c["cache"] == "bf16":
        return x.to(torch.bfloat16), None
    s = _power_scale(x.abs().amax((2, 3)))
    return (x / s[..., None, None]).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    total, new = _lengths(c)
    B, Hq, Hkv, D, P = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    pages = [-(-t // P) for t in total]
    n_pages = sum(pages) + 2  # a pool has pages that no sequence owns
    order = torch.rand((n_pages,), generator=gen, device=DEV).argsort().to(torch.int32)
    table = torch.full((B, max(pages)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    T = off[-1]
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"case": c, "table": table, "lengths": dev(total), "offsets": dev(off), "total": total, "new": new}
    kt = TYPES[c["dtype"]]

    def pool(hot=None):
        x = torch.randn((n_pages, Hkv, P, D), generator=gen, device=DEV)
        if hot is not None:  # keys: some tokens that the queries look for, and a few channels of large magnitude
            x += (torch.rand((n_pages, Hkv, P, 1), generator=gen, device=DEV) < 0.01) * (2.0 * hot)[None, :, None, :]
            ch = torch.rand((Hkv, D), generator=gen, device=DEV).argsort(-1)[:, :2]
            x *= torch.ones((Hkv, D), device=DEV).scatter_(-1, ch, 4.0)[None, :, None, :]
        return _fill(c, x)

    if c["kind"] == "append":
        s["qkv"] = torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen, device=DEV).to(kt)  # as a projection leaves them
        # tokens' values differ in size from page to page, so that scales grow
        size = torch.exp2(torch.rand((T, 1), generator=gen, device=DEV).mul_(4).floor_())
        s["qkv"][:, Hq * D:] *= size.to(kt)
        r = c["rot"]
        pos = torch.arange(max(total), device=DEV, dtype=torch.float64)
        angle = pos[:, None] * 500000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
        s["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).contiguous()
        s["k_pages"], s["k_scale"] = pool()
        s["v_pages"], s["v_scale"] = pool()
        s["q_out"] = torch.empty((T, Hq, D), dtype=kt, device=DEV)
        s["k_out"] = torch.empty((T, Hkv, D), dtype=kt, device=DEV) if c["keys_out"] else None
        first = []  # of the call's tokens in each page that it touches
        for b in range(B):
            lo = total[b] - new[b]
            first += [off[b]] + [off[b] + p - lo for p in range((lo // P + 1) * P, total[b], P)]
        s["first"] = torch.tensor(first, device=DEV)
        return s
    q = torch.randn((T, Hq, D), generator=gen, device=DEV)
    s["q"] = q.to(kt)
    s["k_pages"], s["k_scale"] = pool(q.mean(0).view(Hkv, -1, D).mean(1) * min(T, 16) ** 0.5)
    s["v_pages"], s["v_scale"] = pool()
    s["out"] = torch.empty((T, Hq, D), dtype=TYPES[c["out"]], device=DEV)
    if c["kind"] == "listed":
        idx = torch.full((B, Hkv, c["count"]), -1, dtype=torch.int32, device=DEV)
        for b, t in enumerate(total):
            n = min(c["count"], t)
            # selected tokens cluster: some stretches of the text matter, most do not
            heat = torch.rand((Hkv, -(-t // 96)), generator=gen, device=DEV).pow(4).repeat_interleave(96, -1)[:, :t]
            score = torch.rand((Hkv, t), generator=gen, device=DEV) + heat
            idx[b, :, :n] = score.topk(n, dim=-1).indices.sort(-1).values.to(torch.int32)
        s["idx"] = idx
    return s


# ------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2407_12820_amd import paged

    c = s["case"]
    cache = s.get("handle")
    if cache is None:  # a program makes it once, around its pages
        cache = s["handle"] = paged.PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], n_q_heads=c["q_heads"], dtype=c["dtype"],
                                               out_dtype=c.get("out", "f32"), rotation=s.get("rotation"), rot_style=c.get("style", "halves"))
    one = None if c["new"] > 1 else s["lengths"]  # one token per sequence needs no offsets
    offsets = s["offsets"] if one is None else None
    if c["kind"] == "append":
        Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
        q, k, v = (x.unflatten(1, (-1, D)) for x in s["qkv"].split([Hq * D, Hkv * D, Hkv * D], 1))
        cache.append(k, v, s["table"], s["lengths"], new_offsets=offsets, q=q, q_out=s["q_out"], k_out=s["k_out"])
        return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale", "q_out", "k_out")}
    if c["kind"] == "listed":
        return cache.gather_attn(s["q"], s["idx"], s["table"], s["lengths"], out=s["out"])
    return cache.attn(s["q"], s["table"], s["lengths"], q_offsets=offsets, out=s["out"])


# ------------------------------------------------------------------------- plain forms
def _places(s):
    """Sequence, place in it and number of new tokens of its sequence, of every new token."""
    T = sum(s["new"])
    i = torch.arange(T, device=DEV)
    off = s["offsets"].long()
    b = torch.searchsorted(off[1:], i, right=True)
    return b, i - off[b], (off[1:] - off[:-1])[b]


def _rotate(x, cos, sin, style):
    r = 2 * cos.shape[-1]
    y = x.clone()
    lo, hi = (slice(0, r // 2), slice(r // 2, r)) if style == "halves" else (slice(0, r, 2), slice(1, r, 2))
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return y


def _plain_store(c, pages, scale, x, page, slot, first):
    if c["cache"] == "bf16":
        pages[page, :, slot] = x.to(torch.bfloat16)
        return
    group = torch.searchsorted(first, torch.arange(x.shape[0], device=DEV), right=True) - 1
    amax = torch.zeros((first.shape[0], x.shape[1]), device=DEV)
    amax.scatter_reduce_(0, group[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    p, held = page[first], slot[first]
    before = torch.where(held[:, None] > 0, scale[p], 0.0)
    after = torch.maximum(before, _power_scale(amax))
    raw = pages.view(torch.uint8)
    old = raw[p].view(torch.float8_e4m3fn).float() * (before / after)[..., None, None]
    keep = torch.arange(c["page"], device=DEV) < held[:, None]
    raw[p] = torch.where(keep[:, None, :, None], old.to(torch.float8_e4m3fn).view(torch.uint8), raw[p])
    scale[p] = after
    raw[page, :, slot] = (x / after[group][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    Hq, Hkv, D, P = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    b, i, n = _places(s)
    pos = s["lengths"][b] - n + i
    q, k, v = (x.float().unflatten(1, (-1, D)) for x in s["qkv"].split([Hq * D, Hkv * D, Hkv * D], 1))
    cos, sin = s["rotation"][pos].unsqueeze(1).chunk(2, -1)
    q, k = _rotate(q, cos, sin, c["style"]), _rotate(k, cos, sin, c["style"])
    page, slot = s["table"][b, pos // P].long(), pos % P
    _plain_store(c, s["k_pages"], s["k_scale"], k, page, slot, s["first"])
    _plain_store(c, s["v_pages"], s["v_scale"], v, page, slot, s["first"])
    s["q_out"].copy_(q)
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
    return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale", "q_out", "k_out")}


def _dense(s, name):
    """[B][Hkv][tokens][D] of a paged tensor, zero where a sequence has no page."""
    table = s["table"].clamp(min=0).long()
    x = s[name + "_pages"]
    x = x.view(torch.uint8)[table].view(x.dtype).float()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][table][..., None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_softmax(scores, seen):
    scores = scores.masked_fill_(~seen, float("-inf"))
    scores -= scores.amax(-1, keepdim=True).clamp(min=-1e30)
    return scores.exp_()


def _plain_attn(s):
    c = s["case"]
    B, Hkv, D, G, Tm = c["batch"], c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"], c["new"]
    off, n = s["offsets"].long(), (s["offsets"][1:] - s["offsets"][:-1]).long()
    i = torch.arange(Tm, device=DEV)
    q = s["q"][(off[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)].float()  # [B][Tm][Hq][D], padded
    q = q.view(B, Tm, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Tm, D)
    k, v = _dense(s, "k"), _dense(s, "v")
    last = s["lengths"][:, None] - n[:, None] + i  # [B][Tm]: the last token that a query sees
    seen = (torch.arange(k.shape[2], device=DEV) <= last[..., None])[:, None, None]
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, Hkv, G, Tm, -1)
    p = _plain_softmax(p, seen)
    den = p.sum(-1)
    o = torch.matmul(p.flatten(2, 3), v).view(B, Hkv, G, Tm, D) / den.clamp(min=1e-30)[..., None]
    at, j, _ = _places(s)
    return o.permute(0, 3, 1, 2, 4).reshape(B, Tm, -1, D)[at, j].to(TYPES[c["out"]])


def _plain_listed(s):
    c = s["case"]
    B, Hkv, D, G, P = c["batch"], c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"], c["page"]
    idx = s["idx"].long()
    seen = (idx >= 0) & (idx < s["lengths"][:, None, None])
    t = torch.where(seen, idx, 0)
    page = s["table"].long().gather(1, (t // P).flatten(1)).view_as(t)
    h = torch.arange(Hkv, device=DEV)[None, :, None]

    def rows(name):
        x = s[name + "_pages"]
        x = x.view(torch.uint8)[page, h, t % P].view(x.dtype).float()
        return x if s[name + "_scale"] is None else x * s[name + "_scale"][page, h][..., None]

    q = s["q"].float().view(B, Hkv, G, D)
    p = _plain_softmax(torch.matmul(q, rows("k").transpose(2, 3).contiguous()) * D ** -0.5, seen[:, :, None])
    o = torch.matmul(p, rows("v")) / p.sum(-1).clamp(min=1e-30)[..., None]
    return o.view(B, -1, D).to(TYPES[c["out"]])


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attn": _plain_attn, "listed": _plain_listed}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------- in 64 bits
def _e4m3(x):
    """Nearest e4m3 value (ties to even) of |x| <= 448."""
    e = torch.frexp(x).exponent.clamp(min=-5) - 4  # 2^e: the spacing, 2^-9 for subnormals
    step = torch.ldexp(torch.ones_like(x), e)
    return torch.round(x / step) * step


def _bf16(x):
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256.0), e - 8)


def _exact_append(c, s):
    D, P, Hq, Hkv, r = c["head_dim"], c["page"], c["q_heads"], c["kv_heads"], c["rot"]
    qkv = s["qkv"].double().view(-1, Hq + 2 * Hkv, D)
    pos = torch.cat([torch.arange(t - n, t, device=DEV) for t, n in zip(s["total"], s["new"])])
    cs = s["rotation"].double()[pos]
    z = torch.complex(cs[:, : r // 2], cs[:, r // 2:])[:, None]
    x = qkv[:, : Hq + Hkv, :r].reshape(-1, Hq + Hkv, *((2, r // 2) if c["style"] == "halves" else (r // 2, 2)))
    d = 2 if c["style"] == "halves" else 3
    y = torch.complex(x.select(d, 0), x.select(d, 1)) * z
    y = torch.stack([y.real, y.imag], d).flatten(2)
    qk = torch.cat([y, qkv[:, : Hq + Hkv, r:]], -1)
    held = {"q_out": qk[:, :Hq], "k_out": qk[:, Hq:] if c["keys_out"] else None}
    for name, new in (("k", qk[:, Hq:]), ("v", qkv[:, Hq + Hkv:])):
        pages = s[name + "_pages"].double()
        scale = None if s[name + "_scale"] is None else s[name + "_scale"].double()
        at = 0
        for b, (t, n) in enumerate(zip(s["total"], s["new"])):
            lo = t - n
            while lo < t:
                hi = min(t, (lo // P + 1) * P)
                x = new[at:at + hi - lo].transpose(0, 1)  # [Hkv][tokens][D]
                p, a, z = int(s["table"][b, lo // P]), lo % P, lo % P + hi - lo
                if scale is None:
                    pages[p, :, a:z] = _bf16(x)
                else:
                    most = x.abs().amax((1, 2))
                    want = torch.exp2(torch.ceil(torch.log2(most / FP8_MAX)).clamp(min=-100))
                    if a:
                        want = torch.maximum(want, scale[p])
                        pages[p, :, :a] = _e4m3(pages[p, :, :a] * (scale[p] / want)[:, None, None])
                    scale[p] = want
                    pages[p, :, a:z] = _e4m3(x / want[:, None, None])
                at += hi - lo
                lo = hi
        held[name + "_pages"], held[name + "_scale"] = pages, scale
    return held


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "append":
        if sum(-(-n // c["page"]) + 1 for n in s["new"]) > 20000:
            return None
        return _exact_append(c, s)
    Hkv, D, G, P = c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"], c["page"]
    out = torch.zeros((s["q"].shape[0], c["q_heads"], D), dtype=torch.float64, device=DEV)
    at = 0
    for b, (t, n) in enumerate(zip(s["total"], s["new"])):
        pages = s["table"][b, : -(-t // P)].long()
        for h in range(Hkv):
            k, v = (s[x + "_pages"].view(torch.uint8 if c["cache"] == "fp8" else torch.int16)[pages, h].view(s[x + "_pages"].dtype).double() for x in "kv")
            if c["cache"] == "fp8":
                k, v = k * s["k_scale"][pages, h].double()[:, None, None], v * s["v_scale"][pages, h].double()[:, None, None]
            k, v = k.reshape(-1, D)[:t], v.reshape(-1, D)[:t]
            if c["kind"] == "listed":
                i = s["idx"][b, h].long()
                i = i[(i >= 0) & (i < t)]
                k, v = k[i], v[i]
            for g in range(h * G, h * G + G):
                w = (s["q"][at:at + n, g].double() @ k.T) / D ** 0.5
                if n > 1:
                    w.masked_fill_(torch.ones_like(w, dtype=torch.bool).triu_(t - n + 1), float("-inf"))
                out[at:at + n, g] = torch.softmax(w, -1) @ v
        at += n
    return out
