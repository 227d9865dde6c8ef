"""The operators around a key/value cache held in 4 bits, as measurable cases.

Between the tile attention of a prompt and the tokens generated after it, one
GPU rotates Q and K by their positions, hands out the pages of its cache,
stores K and V there in 4 bits (E2M1 elements, one power-of-two scale for 32 of
them), attends new queries to what is stored, and reads stored rows back as a
KV buffer of the tile kernels:

  tables   mesh_attn_cache_tables   block table, slots, positions of a step
  append   mesh_attn_cache_append   new K, V into the cache; their values, read
                                    back, are the outputs
  read     mesh_attn_cache_read     stored rows as bfloat16 K, V
  attend   mesh_attn_cache_fwd      (O, LSE) of new queries over the cache
  rope     mesh_attn_rope           rotary positions with several axes, or the
                                    inverse rotation (the gradient's)

A cache is [pages][KV heads][page bytes].  With ps tokens a page and head dim d
a (page, head) block holds, in bytes,
  K codes   [ps][d/2]              byte j: dims 2j (low four bits), 2j + 1
  V codes   [ps/8][16][8][d/32]    token 8a + c, dims n d/16 .. at [a][n][c]
  K scales  [ps][d/32]             code c stands for 2^(c - 127), 255 for NaN
  V scales  [d/32][ps]
A GPU of a mesh of n holds the positions p, p + n, p + 2n, .. of every sequence
(striped) or [p P, p P + P) (contiguous).
"""

import math
import random

import torch

own = False  # True: the package's entry points; False: plain torch operations

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _cache(hkv, d, ps, layout="striped", n=1, p=0, P=0):
    return dict(hkv=hkv, d=d, ps=ps, layout=layout, n=n, p=p, P=P)


def listed():
    return [
        # One decode step of a small batch: 40 requests take a token each.
        dict(name="tables decode 40", kind="tables", B=40, longest=16384,
             new="one", **_cache(8, 128, 64)),
        # A prompt chunk's step: hundreds of requests, a few with long chunks.
        dict(name="tables chunks 700", kind="tables", B=700, longest=65536,
             new="mixed", **_cache(8, 128, 16, "striped", 4, 3)),
        # What a decode step of 64 requests stores: rows scattered over pages.
        dict(name="append decode 64", kind="append", rows=64, packed=False,
             **_cache(8, 128, 64)),
        # A 32K prompt's K and V, slices of the fused projection's output.
        dict(name="append prompt 32k", kind="append", rows=32768, packed=True,
             **_cache(8, 128, 64)),
        # A short, odd prefix of a small model, pages out of order.
        dict(name="read 777 d64", kind="read", rows=777, **_cache(4, 64, 16)),
        # A 64K prefix that goes back into the tile kernels.
        dict(name="read prefix 64k", kind="read", rows=65536,
             **_cache(8, 128, 64)),
        # One request, one token, a short context: the smallest decode step.
        dict(name="attend one 1k", kind="attend", B=1, new="one", longest=1021,
             spread=False, group=4, out="bf16", **_cache(8, 128, 16)),
        # A serving batch of very different lengths.
        dict(name="attend ragged 128", kind="attend", B=128, new="one",
             longest=16384, spread=True, group=4, out="bf16",
             **_cache(8, 128, 64)),
        # One of four GPUs that share four requests of 1M tokens: float32
        # partials, merged with the other GPUs' afterwards.
        dict(name="attend share of 1m", kind="attend", B=4, new="one",
             longest=1048573, spread=False, group=4, out="fp32",
             **_cache(8, 128, 64, "striped", 4, 1)),
        # Two prompt chunks of about 1000 tokens over a 32K context.
        dict(name="attend chunk 1000", kind="attend", B=2, new=1000,
             longest=33000, spread=False, group=4, out="bf16",
             **_cache(8, 128, 64)),
        # Q and K of 16K tokens of text and images, slices of the fused
        # projection's output.
        dict(name="rope 16k", kind="rope", rows=16384, hq=32, hkv=8, d=128,
             rot=128, axes=3, interleaved=False, dtype="bf16", inverse=False,
             fused=True),
        # The tile backward's float32 dQ, dK of 3001 tokens rotated back.
        dict(name="rope gradient 3001", kind="rope", rows=3001, hq=12, hkv=4,
             d=64, rot=32, axes=1, interleaved=True, dtype="fp32",
             inverse=True, fused=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_cache(rng):
    n = rng.choice((1, 1, 1, 2, 4, 7))
    if n > 1 and rng.random() < 0.4:
        return _cache(rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128)),
                      rng.choice((16, 32, 64, 128, 256)), "contiguous", n,
                      rng.randrange(n), _log(rng, 100, 8192))
    return _cache(rng.choice((1, 2, 4, 5, 8, 16)), rng.choice((64, 128, 128)),
                  rng.choice((16, 32, 64, 128, 256)), "striped", n,
                  rng.randrange(n))


def draw(rng):
    kind = rng.choice(("tables", "append", "read", "attend", "attend",
                       "attend", "attend", "rope", "rope"))
    if kind == "rope":
        d = rng.choice((64, 128, 128))
        hkv = rng.choice((1, 2, 4, 8))
        hq = hkv * rng.choice((1, 2, 3, 4, 8))
        rot = d if rng.random() < 0.7 else d // 2
        return dict(kind="rope", rows=min(_log(rng, 1, 32768),
                                          16384 * 40 * 128 // (hq + hkv) // d),
                    hq=hq, hkv=hkv, d=d, rot=rot,
                    axes=rng.choice((1, 2, 3)),
                    interleaved=rng.random() < 0.4,
                    dtype=rng.choice(("bf16", "bf16", "fp32")),
                    inverse=rng.random() < 0.4, fused=rng.random() < 0.5)
    c = _draw_cache(rng)
    if kind == "tables":
        return dict(kind=kind, B=_log(rng, 1, 700),
                    longest=_log(rng, 64, 65536),
                    new=rng.choice(("one", "mixed")), **c)
    if kind in ("append", "read"):
        most = 32768 * 8 * 128 // (c["hkv"] * c["d"])
        rows = min(_log(rng, 1, 65536), most)
        if kind == "read":
            return dict(kind=kind, rows=rows, **c)
        return dict(kind=kind, rows=rows, packed=rng.random() < 0.5, **c)
    group = rng.choice((1, 2, 4, 4, 7, 8, 16))
    new = rng.choice(("one", "one", "one", rng.randrange(2, 9),
                      _log(rng, 16, 1000)))
    # Within the listed ones' bytes (1M tokens of 8 heads) and products.
    tokens = 8 * (1 << 20) // c["hkv"] // 2
    if new != "one":
        tokens = min(tokens, 2 * 1000 * 33000 * 32
                     // (new * c["hkv"] * group))
    B = _log(rng, 1, 256)
    while B > 1 and B * 16 > tokens:
        B //= 2
    longest = _log(rng, 16, max(17, min(tokens // B, 200000)))
    return dict(kind=kind, B=B, new=new, longest=longest * c["n"],
                spread=rng.random() < 0.6, group=group,
                out=rng.choice(("bf16", "bf16", "fp32")), **c)


# ---------------------------------------------------------------------------
# Lengths, pages and data
# ---------------------------------------------------------------------------

def _share(c, length):
    """How many of the positions below `length` the cache's GPU holds."""
    if c["layout"] == "contiguous":
        return min(max(length - c["p"] * c["P"], 0), c["P"])
    return max(length - c["p"] + c["n"] - 1, 0) // c["n"]


def _lengths(c):
    """Per request (tokens stored before the step, new tokens): the case's
    own, the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items()
                                    if k != "name")))
    out = []
    for b in range(c["B"]):
        if c.get("spread", True):
            have = _log(rng, 1, c["longest"])
        else:
            have = c["longest"] - rng.randrange(0, 1 + c["longest"] // 100)
        new = c["new"]
        if new == "one":
            new = 1
        elif new == "mixed":
            new = rng.choice((0, 1, 1, 1, rng.randrange(2, 9),
                              _log(rng, 16, 512)))
        out.append((have, new))
    if c["kind"] == "attend":  # lengths with the new tokens in the cache
        out = [(max(have, new), new) for have, new in out]
    return out


def _page_bytes(c):
    return c["ps"] * (c["d"] + c["d"] // 16)


def _quantize(x):
    """Codes (0 .. 15) and scale codes of [.., d], and the values held."""
    g = x.float().unflatten(-1, (-1, 32))
    bits = g.abs().amax(-1, keepdim=True).view(torch.int32)
    e = (bits >> 23) - 129 + ((bits & 0x7fffff) > 0x600000).int()
    e = e.clamp(-126, 125)
    y = g * ((127 - e) << 23).view(torch.float32)
    a = y.abs()
    a = torch.where(a < 2, (a * 2).round() / 2,
                    torch.where(a < 4, a.round(), (a / 2).round() * 2))
    a = a.clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))
    code = code.to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    value = torch.copysign(a, y) * ((e + 127) << 23).view(torch.float32)
    return (code.flatten(-2), (e + 127).to(torch.uint8).squeeze(-1),
            value.flatten(-2))


def _pack(c, k, v):
    """Blocks [m, page bytes] of K, V [m, ps, d]."""
    m, ps, d = k.shape
    kc, ks, _ = _quantize(k)
    vc, vs, _ = _quantize(v)
    kc = kc[..., 0::2] | (kc[..., 1::2] << 4)
    vc = vc[..., 0::2] | (vc[..., 1::2] << 4)
    vc = vc.view(m, ps // 8, 8, 16, d // 32).transpose(2, 3)
    return torch.cat([kc.reshape(m, -1), vc.reshape(m, -1),
                      ks.reshape(m, -1), vs.transpose(1, 2).reshape(m, -1)], 1)


def _fill(c, pages, gen):
    """A cache of `pages` pages whose blocks come from a pool of quantized
    normal K, V; K has a few larger channels, as keys do."""
    pool = max(16, 8192 // c["ps"])
    k = torch.randn(pool, c["ps"], c["d"], generator=gen, device="cuda")
    k[..., 5::41] *= 4
    v = torch.randn(pool, c["ps"], c["d"], generator=gen, device="cuda")
    blocks = _pack(c, k, v)
    pick = torch.randint(pool, (pages * c["hkv"],), generator=gen,
                         device="cuda")
    return blocks[pick].view(pages, c["hkv"], -1)


def _plan(c, pages, max_pages):
    import paper_2512_20968_amd as ma
    return ma.Cache.make(dict(
        num_pages=pages, page_size=c["ps"], num_kv_heads=c["hkv"],
        head_dim=c["d"], max_pages=max_pages,
        layout=0 if c["layout"] == "contiguous" else 1,
        num_partitions=c["n"], partition=c["p"], partition_len=c["P"]))


def _inv_freq(c):
    half = c["rot"] // 2
    return [500000.0 ** (-i / half) for i in range(half)]


def _axis(c):
    """Axis of each frequency: contiguous sections, the first the longest."""
    half, axes = c["rot"] // 2, c["axes"]
    rest = half * 3 // (4 * axes)
    first = half - rest * (axes - 1)
    return [0 if i < first else 1 + (i - first) // rest for i in range(half)]


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype).cuda()


def _prepare_tables(c, gen, order):
    lens = _lengths(c)
    lens = [lens[i] for i in order]
    before = [-(-_share(c, h) // c["ps"]) for h, _ in lens]
    after = [-(-_share(c, h + n) // c["ps"]) for h, n in lens]
    max_pages = max(after + [1]) + 3
    used, want = sum(before), sum(a - b for a, b in zip(after, before))
    pages = used + want + 8
    ids = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((c["B"], max_pages), -1, dtype=torch.int32,
                       device="cuda")
    at = torch.arange(max_pages, device="cuda")
    mine = at[None, :] < _ints(before)[:, None]
    table[mine] = ids[:used]
    rows = sum(n for _, n in lens)
    rows += 7 * (rows % 2)  # some steps are padded to a captured size
    free = ids[used:].contiguous()
    s = dict(pages=pages, max_pages=max_pages, rows=rows, table=table,
             lens=_ints([h for h, _ in lens]), new=_ints([n for _, n in lens]),
             free=free, range=_ints([1, free.numel()]))
    if own:
        i32 = dict(dtype=torch.int32, device="cuda")
        s.update(plan=_plan(c, pages, max_pages), table=table.clone(),
                 lens_out=torch.empty(c["B"], **i32),
                 cu=torch.empty(c["B"] + 1, **i32),
                 slots=torch.empty(rows, dtype=torch.int64, device="cuda"),
                 pos=torch.empty(rows, **i32),
                 range_out=torch.empty(2, **i32),
                 refused=torch.empty(1, **i32))
    return s


def _prepare_attend(c, gen, order):
    lens = _lengths(c)
    lens = [lens[i] for i in order]
    need = [-(-_share(c, h) // c["ps"]) for h, _ in lens]
    max_pages, pages = max(need + [1]), max(sum(need), 1)
    ids = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((c["B"], max_pages), -1, dtype=torch.int32,
                       device="cuda")
    at = torch.arange(max_pages, device="cuda")
    table[at[None, :] < _ints(need)[:, None]] = ids[:sum(need)]
    cu = [0]
    pos = []
    for h, n in lens:
        cu.append(cu[-1] + n)
        pos += range(h - n, h)
    hq = c["hkv"] * c["group"]
    q = torch.randn(cu[-1], hq, c["d"], generator=gen, device="cuda") * 1.5
    s = dict(data=_fill(c, pages, gen), table=table, cu=_ints(cu),
             lens=_ints([h for h, _ in lens]), pos=_ints(pos),
             q=q.to(torch.bfloat16), host=(lens, need))
    if own:
        import paper_2512_20968_amd as ma
        s["plan"] = _plan(c, pages, max_pages)
        s["o"] = torch.empty(q.shape, device="cuda", dtype=torch.float32
                             if c["out"] == "fp32" else torch.bfloat16)
        s["lse"] = torch.empty(hq, cu[-1], device="cuda")
        s["ws"] = torch.empty(ma.mesh_attn_cache_fwd_workspace_size(
            s["plan"], hq, c["B"], cu[-1]), dtype=torch.uint8, device="cuda")
    return s


def _slots(c, rows, pages, packed, gen):
    """Slots of `rows` rows: whole pages in random order, or any slots."""
    if not packed:
        return torch.randperm(pages * c["ps"], generator=gen,
                              device="cuda")[:rows]
    ids = torch.randperm(pages, generator=gen, device="cuda")
    at = torch.arange(rows, device="cuda")
    return ids[at // c["ps"]] * c["ps"] + at % c["ps"]


def _prepare_append(c, gen):
    rows, hkv, d = c["rows"], c["hkv"], c["d"]
    pages = rows // c["ps"] + 3
    # K and V as slices of a fused projection of 4 query heads per KV head.
    qkv = torch.randn(rows, 6 * hkv, d, generator=gen, device="cuda")
    qkv[:, 4 * hkv:5 * hkv, 5::41] *= 4
    qkv = qkv.to(torch.bfloat16)
    s = dict(k=qkv[:, 4 * hkv:5 * hkv], v=qkv[:, 5 * hkv:],
             slots=_slots(c, rows, pages, c["packed"], gen))
    if own:
        s.update(plan=_plan(c, pages, 1), data=torch.zeros(
            pages, hkv, _page_bytes(c), dtype=torch.uint8, device="cuda"),
            ko=torch.empty(rows, hkv, d, dtype=torch.bfloat16, device="cuda"),
            vo=torch.empty(rows, hkv, d, dtype=torch.bfloat16, device="cuda"))
    return s


def _prepare_read(c, gen):
    rows, hkv, d = c["rows"], c["hkv"], c["d"]
    pages = rows // c["ps"] + 3
    s = dict(data=_fill(c, pages, gen),
             slots=_slots(c, rows, pages, True, gen))
    if own:
        s.update(plan=_plan(c, pages, 1),
                 ko=torch.empty(rows, hkv, d, dtype=torch.bfloat16,
                                device="cuda"),
                 vo=torch.empty(rows, hkv, d, dtype=torch.bfloat16,
                                device="cuda"))
    return s


def _prepare_rope(c, gen):
    rows, hq, hkv, d = c["rows"], c["hq"], c["hkv"], c["d"]
    dtype = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    x = torch.randn(rows, hq + hkv + (hkv if c["fused"] else 0), d,
                    generator=gen, device="cuda").to(dtype)
    if c["fused"]:
        q, k = x[:, :hq], x[:, hq:hq + hkv]
    else:
        q, k = x[:, :hq].contiguous(), x[:, hq:].contiguous()
    # The first axis counts on through a long sequence; the others run over
    # the rows and columns of images.
    start = torch.randint(900000, (1,), generator=gen, device="cuda")
    at = torch.arange(rows, device="cuda")
    pos = [start + at, start + at // 64 % 48, start + at % 64][:c["axes"]]
    s = dict(q=q, k=k, pos=torch.stack(pos).int())
    if own:
        import paper_2512_20968_amd as ma
        s["rope"] = ma.Rope.make(dict(
            head_dim=d, rotary_dim=c["rot"], num_axes=c["axes"],
            interleaved=c["interleaved"], inv_freq=_inv_freq(c),
            axis=_axis(c)))
        s["qo"] = torch.empty(rows, hq, d, dtype=dtype, device="cuda")
        s["ko"] = torch.empty(rows, hkv, d, dtype=dtype, device="cuda")
    return s


def prepare(case, seed):
    c = case
    gen = torch.Generator("cuda").manual_seed(seed)
    if c["kind"] in ("tables", "attend"):
        order = list(range(c["B"]))
        random.Random(seed).shuffle(order)
        make = _prepare_tables if c["kind"] == "tables" else _prepare_attend
        s = make(c, gen, order)
    else:
        s = {"append": _prepare_append, "read": _prepare_read,
             "rope": _prepare_rope}[c["kind"]](c, gen)
    s["c"] = c
    return s


# ---------------------------------------------------------------------------
# The package's entry points
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2512_20968_amd as ma
    c = s["c"]
    if c["kind"] == "tables":
        ma.mesh_attn_cache_tables(
            s["plan"], s["lens"], s["new"], s["free"], s["range"], s["table"],
            s["lens_out"], s["cu"], s["slots"], s["pos"], s["range_out"],
            s["refused"])
        return [s["table"], s["lens_out"], s["cu"], s["slots"], s["pos"],
                s["range_out"], s["refused"]]
    if c["kind"] == "append":
        ma.mesh_attn_cache_append(s["plan"], s["k"], s["v"], s["slots"],
                                  s["data"])
        ma.mesh_attn_cache_read(s["plan"], s["slots"], s["data"], s["ko"],
                                s["vo"])
        return [s["ko"], s["vo"]]
    if c["kind"] == "read":
        ma.mesh_attn_cache_read(s["plan"], s["slots"], s["data"], s["ko"],
                                s["vo"])
        return [s["ko"], s["vo"]]
    if c["kind"] == "attend":
        ma.mesh_attn_cache_fwd(s["plan"], c["d"] ** -0.5, s["q"], s["pos"],
                               s["cu"], s["lens"], s["table"], s["data"],
                               s["o"], s["lse"], s["ws"])
        return [s["o"], s["lse"]]
    ma.mesh_attn_rope(s["rope"], s["pos"], s["q"], s["qo"], s["k"], s["ko"],
                      inverse=int(c["inverse"]))
    return [s["qo"], s["ko"]]


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _share_t(c, length):
    if c["layout"] == "contiguous":
        return (length - c["p"] * c["P"]).clamp(0, c["P"])
    return (length - c["p"] + c["n"] - 1).clamp(min=0) // c["n"]


def _plain_tables(c, s):
    lens, new = s["lens"].long(), s["new"].long()
    ps, dev = c["ps"], lens.device
    total = lens + new
    before = (_share_t(c, lens) + ps - 1) // ps
    after = (_share_t(c, total) + ps - 1) // ps
    fits = after <= s["max_pages"]
    want = torch.where(fits, after - before, 0)
    ends = want.cumsum(0)
    first, last = s["range"].long().unbind()
    ok = fits & ((want == 0) | (ends <= last - first))
    # New pages of the accepted requests.
    table = s["table"].clone()
    at = torch.arange(s["max_pages"], device=dev)[None, :]
    take = ok[:, None] & (at >= before[:, None]) & (at < after[:, None])
    src = first + (ends - want - before)[:, None] + at
    ids = s["free"][src.clamp(0, s["free"].numel() - 1)]
    table = torch.where(take, ids, table)
    # Rows.
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev),
                    new.cumsum(0)])
    row = torch.arange(s["rows"], device=dev)
    b = torch.searchsorted(cu, row, right=True) - 1
    live = b < c["B"]
    b = b.clamp(max=c["B"] - 1)
    live &= ok[b]
    pos = torch.where(live, lens[b] + row - cu[b], -1)
    local = _share_t(c, pos)
    here = live & (_share_t(c, pos + 1) > local)
    page = table[b, (local // ps).clamp(0, s["max_pages"] - 1)].long()
    here &= (page >= 0) & (page < s["pages"])
    slots = torch.where(here, page * ps + local % ps, -1)
    taken = torch.where(ok, ends, 0).amax()
    return [table, torch.where(ok, total, lens).int(), cu.int(), slots,
            pos.int(), torch.stack([first + taken, last]).int(),
            (~ok).sum().int().view(1)]


_PAIRS = {}


def _pairs(dev):
    """The two values of every byte."""
    if dev not in _PAIRS:
        one = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=dev)
        i = torch.arange(256, device=dev)
        _PAIRS[dev] = torch.stack([one[i & 15], one[i >> 4]], -1)
    return _PAIRS[dev]


def _scales(code):
    bits = code.to(torch.int32) << 23
    return torch.where(code == 255, math.nan, bits.view(torch.float32))


def _unpack(c, blocks):
    """K, V [.., ps, d] float32 of blocks [.., page bytes]."""
    ps, d = c["ps"], c["d"]
    lead = blocks.shape[:-1]
    kc, vc, ks, vs = blocks.split(
        [ps * d // 2, ps * d // 2, ps * d // 32, ps * d // 32], -1)
    pairs = _pairs(blocks.device)
    k = pairs[kc.int()].view(*lead, ps, d // 32, 32)
    vc = vc.reshape(*lead, ps // 8, 16, 8, d // 32).transpose(-3, -2)
    v = pairs[vc.int()].reshape(*lead, ps, d // 32, 32)
    k = k * _scales(ks).view(*lead, ps, d // 32, 1)
    v = v * _scales(vs).view(*lead, d // 32, ps).transpose(-1, -2)[..., None]
    return k.flatten(-2), v.flatten(-2)


def _plain_read(c, s):
    page, at = s["slots"] // c["ps"], s["slots"] % c["ps"]
    k, v = _unpack(c, s["data"])
    return [k[page, :, at].to(torch.bfloat16),
            v[page, :, at].to(torch.bfloat16)]


def _plain_append(c, s):
    return [_quantize(s["k"])[2].to(torch.bfloat16),
            _quantize(s["v"])[2].to(torch.bfloat16)]


def _plain_attend(c, s):
    lens, need = s["host"]
    hkv, g, d, ps = c["hkv"], c["group"], c["d"], c["ps"]
    q = s["q"].float()
    o = torch.empty_like(q)
    lse = torch.empty(hkv * g, q.shape[0], device=q.device)
    row = 0
    for b, (have, new) in enumerate(lens):
        rows = slice(row, row + new)
        row += new
        local = _share(c, have)
        if new == 0:
            continue
        if local == 0:
            o[rows] = 0
            lse[:, rows] = -math.inf
            continue
        seen = _share_t(c, s["pos"][rows].long() + 1)
        key = torch.arange(local, device=q.device)
        hidden = (key[None, :] >= seen[:, None]).repeat_interleave(g, 0)
        blocks = s["data"][s["table"][b, :need[b]].long()]
        # All heads of a short request at once, one by one of a long one.
        step = hkv if local * (256 * d // 128 + new * g) < 1 << 24 else 1
        for h in range(0, hkv, step):
            k, v = _unpack(c, blocks[:, h:h + step])
            k = k.transpose(0, 1).reshape(step, -1, d)[:, :local]
            v = v.transpose(0, 1).reshape(step, -1, d)[:, :local]
            heads = slice(h * g, (h + step) * g)
            x = q[rows, heads].reshape(new, step, g, d).transpose(0, 1)
            x = x.reshape(step, new * g, d) * d ** -0.5
            p = torch.bmm(x, k.transpose(1, 2).contiguous())
            p.masked_fill_(hidden, -math.inf)
            top = p.amax(-1, keepdim=True)
            top.masked_fill_(top == -math.inf, 0.0)
            p.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            y = torch.bmm(p, v.contiguous())
            y = torch.where(total > 0, y / total, 0.0)
            o[rows, heads] = y.view(step, new, g, d).transpose(0, 1).reshape(
                new, step * g, d)
            lse[heads, rows] = (top + total.log()).view(
                step, new, g).transpose(1, 2).reshape(step * g, new)
    return [o.to(torch.float32 if c["out"] == "fp32" else torch.bfloat16),
            lse]


def _plain_rope(c, s):
    half, inter = c["rot"] // 2, c["interleaved"]
    freq = torch.tensor(_inv_freq(c), dtype=torch.float64).cuda()
    axis = torch.tensor(_axis(c)).cuda()
    angle = s["pos"].double()[axis].transpose(0, 1) * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    cos, sin = cos[:, None], sin[:, None] * (-1 if c["inverse"] else 1)
    out = []
    for x in (s["q"], s["k"]):
        f = x.float()
        a = f[..., 0:c["rot"]:2] if inter else f[..., :half]
        b = f[..., 1:c["rot"]:2] if inter else f[..., half:c["rot"]]
        y = [a * cos - b * sin, b * cos + a * sin]
        y = torch.stack(y, -1).flatten(-2) if inter else torch.cat(y, -1)
        out.append(torch.cat([y, f[..., c["rot"]:]], -1).to(x.dtype))
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _plain_tables, "append": _plain_append,
            "read": _plain_read, "attend": _plain_attend,
            "rope": _plain_rope}[state["c"]["kind"]](state["c"], state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "rope":
        elem = 4 if c["dtype"] == "fp32" else 2
        n = c["rows"] * (c["hq"] + c["hkv"])
        return {"bytes": 2 * n * c["d"] * elem + 4 * c["rows"] * c["axes"],
                "flops": 3 * n * c["rot"]}
    token = c["hkv"] * (c["d"] + c["d"] // 16)
    if c["kind"] == "tables":
        lens = _lengths(c)
        rows = sum(n for _, n in lens)
        rows += 7 * (rows % 2)
        pages = sum(-(-_share(c, h + n) // c["ps"])
                    - -(-_share(c, h) // c["ps"]) for h, n in lens)
        return {"bytes": 16 * c["B"] + 8 * pages + 12 * rows,
                "flops": 8 * c["B"] + 4 * rows}
    if c["kind"] in ("append", "read"):
        values = c["rows"] * c["hkv"] * c["d"] * 4  # K and V in bfloat16
        moved = c["rows"] * (token + 8) + values
        if c["kind"] == "append":  # stored, then read back
            return {"bytes": 2 * moved, "flops": 3 * values // 2}
        return {"bytes": moved, "flops": values // 2}
    lens = _lengths(c)
    stored = pairs = rows = 0
    for have, new in lens:
        rows += new
        stored += _share(c, have) if new else 0
        pairs += sum(_share(c, have - new + i + 1) for i in range(new))
    hq = c["hkv"] * c["group"]
    out = 4 if c["out"] == "fp32" else 2
    return {"bytes": stored * token + rows * hq * (c["d"] * (2 + out) + 4)
            + 4 * (rows + 2 * c["B"] + stored // c["ps"]),
            "flops": 4 * c["d"] * hq * max(pairs, 1)}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_value(code):
    """E2M1: sign, two exponent bits (bias 1), one fraction bit."""
    s, e, m = code >> 3, (code >> 1) & 3, (code & 1).double()
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e.double() - 1))
    return torch.where(s == 1, -mag, mag)


def _exact_rows(c, data, page, at, head):
    """K, V [rows, d] in float64 of one head at (page, token in page)."""
    ps, d = c["ps"], c["d"]
    flat = data.view(-1)
    base = (page * c["hkv"] + head) * _page_bytes(c)
    dim = torch.arange(d, device=data.device)
    ka = base[:, None] + at[:, None] * (d // 2) + dim // 2
    va = (base + ps * d // 2 + at // 8 * (4 * d) + at % 8 * (d // 32))[:, None]
    va = va + dim // (d // 16) * (d // 4) + dim % (d // 16) // 2
    ksa = (base + ps * d + at * (d // 32))[:, None] + dim // 32
    vsa = (base + ps * d + ps * d // 32 + at)[:, None] + dim // 32 * ps
    out = []
    for a, sa in ((ka, ksa), (va, vsa)):
        byte, scale = flat[a].int(), flat[sa].double()
        x = _exact_value((byte >> (4 * (dim % 2))) & 15)
        out.append(x * 2.0 ** (scale - 127))
    return out


def _exact_quantized(x):
    """Nearest of the fifteen values times the group's scale, ties to the even
    code, in float64."""
    d = x.shape[-1]
    g = x.double().reshape(-1, 32)
    top = g.abs().max(1).values
    mant, exp = torch.frexp(top)  # top = mant 2^exp, mant in [1/2, 1)
    e = (exp - 1 - 2 + (mant > 0.875).int()).clamp(-126, 125)
    e = torch.where(top == 0, -126, e)
    y = g / (2.0 ** e.double())[:, None]
    values = torch.tensor(E2M1, dtype=torch.float64).to(x.device)
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.long)
    for i in range(7):
        mid = (values[i] + values[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)  # ties to the even code
    z = torch.copysign(values[code], y) * (2.0 ** e.double())[:, None]
    return z.reshape(x.shape[:-1] + (d,))


def exact(case, seed):
    c = case
    if c["kind"] == "tables":
        return None
    s = prepare(case, seed)
    if c["kind"] == "append":
        return [torch.cat([_exact_quantized(y) for y in x.split(4096)])
                for x in (s["k"], s["v"])]
    if c["kind"] == "read":
        page, at = s["slots"] // c["ps"], s["slots"] % c["ps"]
        heads = [_exact_rows(c, s["data"], page, at, h)
                 for h in range(c["hkv"])]
        return [torch.stack([x[i] for x in heads], 1) for i in (0, 1)]
    if c["kind"] == "rope":
        out = []
        turn = -1.0 if c["inverse"] else 1.0
        for x in (s["q"], s["k"]):
            y = x.double().clone()
            for i, (f, axis) in enumerate(zip(_inv_freq(c), _axis(c))):
                j, l = ((2 * i, 2 * i + 1) if c["interleaved"]
                        else (i, i + c["rot"] // 2))
                phi = (s["pos"][axis].double() * f * turn)[:, None]
                a, b = x[..., j].double(), x[..., l].double()
                y[..., j] = a * torch.cos(phi) - b * torch.sin(phi)
                y[..., l] = a * torch.sin(phi) + b * torch.cos(phi)
            out.append(y)
        return out
    lens, _ = s["host"]
    hkv, g, d = c["hkv"], c["group"], c["d"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((hkv * g, s["q"].shape[0]), -math.inf,
                     dtype=torch.float64, device="cuda")
    row = 0
    for b, (have, new) in enumerate(lens):
        first, row = row, row + new
        local = _share(c, have)
        if new == 0 or local == 0:
            continue
        key = torch.arange(local, device="cuda")
        page = s["table"][b].long()[key // c["ps"]]
        # Global position of every stored key.
        where = (c["p"] * c["P"] + key if c["layout"] == "contiguous"
                 else key * c["n"] + c["p"])
        for h in range(hkv):
            k, v = _exact_rows(c, s["data"], page, key % c["ps"], h)
            for r in range(first, row, 128):
                e = min(r + 128, row)
                q = s["q"][r:e, h * g:(h + 1) * g].double().reshape(-1, d)
                x = (q @ k.T) / math.sqrt(d)
                pos = s["pos"][r:e].long().repeat_interleave(g)
                x = torch.where(where[None] <= pos[:, None], x, -math.inf)
                z = torch.logsumexp(x, 1)
                w = torch.where(x == -math.inf, 0.0, torch.exp(
                    x - torch.where(z == -math.inf, 0.0, z)[:, None]))
                o[r:e, h * g:(h + 1) * g] = (w @ v).view(e - r, g, d)
                lse[h * g:(h + 1) * g, r:e] = z.view(e - r, g).T
    return [o, lse]
