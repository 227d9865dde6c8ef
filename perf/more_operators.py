"""Attention under a score rule, and the step that feeds its cache, as
measurable cases.

Scores that are capped by a tanh, get a bias that falls with the distance, or
are seen through documents, prefixes and windows, for one GPU's tile of a long
sequence and for the tokens generated after it:

  fwd     mesh_attn_score_fwd          (O, LSE) of a tile's rows
  bwd     mesh_attn_score_bwd          dQ, dK, dV of a tile, from O and LSE
  cache   mesh_attn_cache_score_fwd    (O, LSE) of new tokens over the paged
                                       4-bit cache
  append  mesh_attn_cache_rope_append  Q and K rotated by their positions, K
                                       and V stored in 4 bits; Q and the stored
                                       values, read back, are the outputs

Row i at position p_i scores key j at position p_j as
  x_ij = cap tanh(s <q_i, k_j> / cap) - slope_h |p_i - p_j|
and sees it where key_begin_i <= p_j < key_end_i (without a key_end: up to its
own position if causal, else everything); O = sum_j exp(x_ij - LSE_i) v_j.

A tile stacks partitions of P tokens: token r of partition p of n has position
p P + r (contiguous) or r n + p (striped).  A cache is [pages][KV heads][page
bytes]; with ps tokens a page and head dim d a (page, head) block holds
  K codes   [ps][d/2]              byte j: dims 2j (low four bits), 2j + 1
  V codes   [ps/8][16][8][d/32]    token 8a + c, dims n d/16 .. at [a][n][c]
  K scales  [ps][d/32]             code c stands for 2^(c - 127), 255 for NaN
  V scales  [d/32][ps]
"""

import math
import random

import torch

own = False  # True: the package's entry points; False: plain torch operations

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LOG = math.log


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _tile(kind, P, hq, hkv, d, mask, cap=0.0, slopes=False, n=1, q="0", kv="0",
          layout="contiguous", out="bf16", fused=False):
    """q, kv: the tile's partitions.  mask: causal, full, docs (packed
    documents, causal inside each, the sequence's end padding), prefix (docs
    whose first third is seen by all of the document), window (causal, the last
    quarter of the sequence at most)."""
    return dict(kind=kind, P=P, hq=hq, hkv=hkv, d=d, mask=mask, cap=cap,
                slopes=slopes, n=n, q=q, kv=kv, layout=layout, out=out,
                fused=fused)


def _cache(kind, hkv, d, ps, n=1, p=0, **more):
    return dict(kind=kind, hkv=hkv, d=d, ps=ps, n=n, p=p, **more)


def listed():
    return [
        # A short odd sequence of a small model: what a call costs at least.
        dict(name="fwd 77 tokens d64",
             **_tile("fwd", 77, 4, 2, 64, "causal", slopes=True)),
        # A training step's packed documents, Q, K, V slices of the fused
        # projection's output.
        dict(name="fwd documents 8k",
             **_tile("fwd", 8192, 32, 8, 128, "docs", cap=50.0, fused=True)),
        # One GPU of a striped mesh of four: prefixes and a distance bias,
        # float32 partials to be merged with the other GPUs'.
        dict(name="fwd prefixes d64",
             **_tile("fwd", 1501, 12, 12, 64, "prefix", slopes=True, n=4,
                     q="1,2", kv="0,1,2,3", layout="striped", out="fp32")),
        # One long causal sequence with capped scores.
        dict(name="fwd causal 16k",
             **_tile("fwd", 16384, 32, 8, 128, "causal", cap=30.0)),
        # The gradients of a small model's odd prefixes with a distance bias.
        dict(name="bwd prefixes d64",
             **_tile("bwd", 3001, 12, 4, 64, "prefix", slopes=True)),
        # A training step's packed documents.
        dict(name="bwd documents 4k",
             **_tile("bwd", 4096, 32, 8, 128, "docs", cap=50.0)),
        # One long causal sequence with capped scores.
        dict(name="bwd causal 8k",
             **_tile("bwd", 8192, 32, 8, 128, "causal", cap=30.0)),
        # One request, one token, a short context: the smallest decode step.
        dict(name="cache one 1k",
             **_cache("cache", 8, 128, 16, B=1, new=1, longest=1021,
                      spread=False, group=4, out="bf16", cap=30.0,
                      slopes=False, window=0)),
        # A serving batch of long contexts seen through windows of 4096.
        dict(name="cache window 64",
             **_cache("cache", 8, 128, 64, B=64, new=1, longest=65536,
                      spread=True, group=4, out="bf16", cap=50.0,
                      slopes=False, window=4096)),
        # Two prompt chunks of about 1000 tokens over a 16K context.
        dict(name="cache chunk 1000",
             **_cache("cache", 8, 128, 64, B=2, new=1000, longest=16500,
                      spread=False, group=4, out="bf16", cap=30.0,
                      slopes=True, window=0)),
        # What a decode step of 64 requests rotates and stores.
        dict(name="append decode 64",
             **_cache("append", 8, 128, 64, rows=64, group=4, rot=128, axes=1,
                      interleaved=False, fused=True)),
        # A prompt of 16K tokens.
        dict(name="append prompt 16k",
             **_cache("append", 8, 128, 64, rows=16384, group=4, rot=128,
                      axes=1, interleaved=False, fused=True)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(LOG(lo), LOG(hi)))))


def draw(rng):
    kind = rng.choice(("fwd", "fwd", "bwd", "bwd", "cache", "cache", "append"))
    d = rng.choice((64, 128, 128))
    if kind == "append":
        hkv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 8))
        most = 16384 * 48 * 128 // (hkv * (group + 2) * d)
        return _cache(kind, hkv, d, rng.choice((16, 32, 64, 128, 256)),
                      rows=min(_log(rng, 1, 32768), most), group=group,
                      rot=rng.choice((d, d, d // 2)), axes=rng.choice((1, 3)),
                      interleaved=rng.random() < 0.4,
                      fused=rng.random() < 0.5)
    cap = rng.choice((0.0, 20.0, 30.0, 50.0))
    slopes = rng.random() < 0.4
    if kind == "cache":
        hkv, group = rng.choice((1, 2, 4, 5, 8)), rng.choice((1, 2, 4, 7, 8))
        new = rng.choice((1, 1, rng.randrange(2, 9), _log(rng, 16, 1000)))
        n = rng.choice((1, 1, 2, 4))
        tokens = min(8 * 1000000 // hkv // 2,
                     2 * 1000 * 16500 * 32 // (new * hkv * group))
        B = _log(rng, 1, 128)
        while B > 1 and B * 16 > tokens:
            B //= 2
        return _cache(kind, hkv, d, rng.choice((16, 32, 64, 128, 256)), n,
                      rng.randrange(n), B=B, new=new,
                      longest=n * _log(rng, 16, max(17, min(tokens // B,
                                                            100000))),
                      spread=rng.random() < 0.6, group=group,
                      out=rng.choice(("bf16", "bf16", "fp32")), cap=cap,
                      slopes=slopes, window=rng.choice((0, 0, 100, 1024)))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 3, 4))
    longest = 16384 if kind == "fwd" else 8192
    n = rng.choice((1, 1, 2, 4, 7))
    lists = ["0", "0"]
    if n > 1:
        for i in (0, 1):
            some = rng.sample(range(n), rng.randrange(1, n + 1))
            lists[i] = ",".join(str(x) for x in some)
    tokens = min(_log(rng, n, longest),
                 int(longest * math.sqrt(32 * 128 / (hq * d))))
    tokens = min(tokens, longest)
    return _tile(kind, max(tokens // n, 1), hq, hkv, d,
                 rng.choice(("causal", "full", "docs", "docs", "prefix",
                             "window")), cap=cap, slopes=slopes, n=n,
                 q=lists[0], kv=lists[1],
                 layout=rng.choice(("contiguous", "striped")),
                 out="bf16" if kind == "bwd" else rng.choice(
                     ("bf16", "bf16", "fp32")),
                 fused=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# Positions, ranges, lengths and data
# ---------------------------------------------------------------------------

def _positions(c, lst):
    """Positions of the rows of a buffer of the partitions `lst`."""
    part = torch.tensor([int(x) for x in lst.split(",")])[:, None]
    r = torch.arange(c["P"])[None, :]
    pos = r * c["n"] + part if c["layout"] == "striped" else part * c["P"] + r
    return pos.reshape(-1)


def _ranges(c):
    """(key_begin, key_end) of every position, None where the causal flag
    says it: the case's own, the same for every seed."""
    total = c["n"] * c["P"]
    at = torch.arange(total)
    if c["mask"] in ("causal", "full"):
        return None, None
    if c["mask"] == "window":
        return (at - max(total // 4, 1) + 1).clamp(min=0), None
    rng = random.Random("%d %s" % (total, c["mask"]))
    begin, end = torch.zeros(total).long(), torch.zeros(total).long()
    x, stop = 0, total - total // 32  # behind it: padding that sees nothing
    while x < stop:
        y = min(x + _log(rng, max(total // 64, 1), max(total // 3, 2)), stop)
        begin[x:y], end[x:y] = x, at[x:y] + 1
        if c["mask"] == "prefix":
            end[x:y] = end[x:y].clamp(min=x + (y - x) // 3)
        x = y
    return begin, end


def _slopes(hq):
    return [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]


def _share(c, length):
    """How many of the positions below `length` the cache's GPU holds."""
    return max(length - c["p"] + c["n"] - 1, 0) // c["n"]


def _lengths(c):
    """Per request (tokens, the new ones among them, new tokens): the case's
    own, the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items()
                                    if k != "name")))
    out = []
    for b in range(c["B"]):
        have = (_log(rng, 1, c["longest"]) if c["spread"] else
                c["longest"] - rng.randrange(0, 1 + c["longest"] // 100))
        out.append((max(have, c["new"]), c["new"]))
    return out


def _page_bytes(c):
    return c["ps"] * (c["d"] + c["d"] // 16)


def _quantize(x):
    """Codes (0 .. 15), scale codes and values of [.., d] in float64: a group
    of 32 has the least power of two that keeps its largest in 7 units."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.frexp(top).exponent - 3
    e = (e + (top > 7 * torch.ldexp(torch.ones_like(top), e)).int())
    e = torch.where(top > 0, e, -126).clamp(-126, 125)
    unit = torch.ldexp(torch.ones_like(top), e)
    y = g / unit
    a = y.abs()
    a = torch.where(a < 2, (a * 2).round() / 2,
                    torch.where(a < 4, a.round(), (a / 2).round() * 2))
    a = a.clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))
    code = code.to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    return (code.flatten(-2), (e + 127).to(torch.uint8).squeeze(-1),
            (torch.copysign(a, y) * unit).flatten(-2))


def _fill(c, pages, gen):
    """A cache of `pages` pages whose blocks come from a pool of quantized
    normal K, V; K has a few larger channels, as keys do."""
    ps, d = c["ps"], c["d"]
    m = max(16, 8192 // ps)
    k = torch.randn(m, ps, d, generator=gen, device="cuda")
    k[..., 5::41] *= 4
    v = torch.randn(m, ps, d, generator=gen, device="cuda")
    (kc, ks, _), (vc, vs, _) = _quantize(k), _quantize(v)
    kc = kc[..., 0::2] | (kc[..., 1::2] << 4)
    vc = vc[..., 0::2] | (vc[..., 1::2] << 4)
    vc = vc.view(m, ps // 8, 8, 16, d // 32).transpose(2, 3)
    pool = torch.cat([kc.reshape(m, -1), vc.reshape(m, -1), ks.reshape(m, -1),
                      vs.transpose(1, 2).reshape(m, -1)], 1)
    pick = torch.randint(m, (pages * c["hkv"],), generator=gen, device="cuda")
    return pool[pick].view(pages, c["hkv"], -1)


def _plan(c, pages, max_pages):
    import paper_2512_20968_amd as ma
    return ma.Cache.make(dict(
        num_pages=pages, page_size=c["ps"], num_kv_heads=c["hkv"],
        head_dim=c["d"], max_pages=max_pages, num_partitions=c["n"],
        partition=c["p"]))


def _ints(x, dtype=torch.int32):
    return torch.as_tensor(x).to(dtype).cuda()


def _prepare_tile(c, gen):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    qpos, kpos = _positions(c, c["q"]), _positions(c, c["kv"])
    begin, end = _ranges(c)
    rows, keys = len(qpos), len(kpos)

    def part(n, heads):  # a slice of a wider row, or rows of its own
        wide = heads + hkv if c["fused"] else heads
        x = torch.randn(n, wide, d, generator=gen, device="cuda")
        return x.to(torch.bfloat16)[:, wide - heads:]

    q, k, v = part(rows, hq), part(keys, hkv), part(keys, hkv)
    q.mul_(2)  # scores far enough out for the cap to bend them
    k[..., 5::41] *= 4
    s = dict(q=q, k=k, v=v, qpos=qpos.cuda(), kpos=kpos.cuda(),
             begin=None if begin is None else _ints(begin[qpos]),
             end=None if end is None else _ints(end[qpos]),
             slopes=torch.tensor(_slopes(hq)).cuda() if c["slopes"] else None)
    if c["kind"] == "bwd":
        s["do"] = torch.randn(rows, hq, d, generator=gen,
                              device="cuda").to(torch.bfloat16)
        s["o"], s["lse"] = _plain_fwd(c, s)
    if own:
        import paper_2512_20968_amd as ma
        s["prob"] = ma.Problem.make(dict(
            num_partitions=c["n"], partition_len=c["P"], num_q_heads=hq,
            num_kv_heads=hkv, head_dim=d, causal=int(c["mask"] != "full"),
            layout=int(c["layout"] == "striped"), softmax_scale=d ** -0.5))
        s["lists"] = [[int(x) for x in c[k].split(",")] for k in ("q", "kv")]
        s["score"] = ma.Score.make(dict(
            cap=c["cap"], slopes=s["slopes"], key_begin=s["begin"],
            key_end=s["end"]))
        nq, nkv = (len(x) for x in s["lists"])
        if c["kind"] == "fwd":
            n = ma.mesh_attn_score_fwd_workspace_size(s["prob"], nq, nkv)
            s["out"] = [torch.empty(rows, hq, d, device="cuda", dtype=_out(c)),
                        torch.empty(hq, rows, device="cuda")]
        else:
            n = ma.mesh_attn_score_bwd_workspace_size(s["prob"], nq, nkv)
            s["out"] = [torch.empty(x.shape, device="cuda",
                                    dtype=torch.bfloat16) for x in (q, k, v)]
        s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    return s


def _out(c):
    return torch.float32 if c["out"] == "fp32" else torch.bfloat16


def _prepare_cache(c, gen, order):
    lens = _lengths(c)
    lens = [lens[i] for i in order]
    need = [-(-_share(c, h) // c["ps"]) for h, _ in lens]
    max_pages, pages = max(need + [1]), max(sum(need), 1)
    ids = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((c["B"], max_pages), -1, dtype=torch.int32,
                       device="cuda")
    at = torch.arange(max_pages, device="cuda")
    table[at[None, :] < _ints(need)[:, None]] = ids[:sum(need)]
    new = c["new"]
    pos = torch.tensor([h - n for h, n in lens])[:, None] + torch.arange(new)
    pos = _ints(pos.reshape(-1))
    hq = c["hkv"] * c["group"]
    q = torch.randn(len(pos), hq, c["d"], generator=gen, device="cuda") * 3
    s = dict(data=_fill(c, pages, gen), table=table, pos=pos,
             cu=_ints(torch.arange(c["B"] + 1) * new),
             lens=_ints([h for h, _ in lens]), q=q.to(torch.bfloat16),
             begin=(pos - c["window"] + 1).clamp(min=0) if c["window"]
             else None, host=(lens, need),
             slopes=torch.tensor(_slopes(hq)).cuda() if c["slopes"] else None)
    if own:
        import paper_2512_20968_amd as ma
        s["plan"] = _plan(c, pages, max_pages)
        s["score"] = ma.Score.make(dict(cap=c["cap"], slopes=s["slopes"],
                                        key_begin=s["begin"]))
        s["o"] = torch.empty(q.shape, device="cuda", dtype=_out(c))
        s["lse"] = torch.empty(hq, len(pos), device="cuda")
        n = ma.mesh_attn_cache_score_fwd_workspace_size(s["plan"], hq, c["B"],
                                                        len(pos))
        s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    return s


def _inv_freq(c):
    half = c["rot"] // 2
    return [500000.0 ** (-i / half) for i in range(half)]


def _axis(c):
    """Axis of each frequency: sections of about the same length."""
    half = c["rot"] // 2
    return [i * c["axes"] // half for i in range(half)]


def _prepare_append(c, gen):
    rows, hkv, d, hq = c["rows"], c["hkv"], c["d"], c["hkv"] * c["group"]
    pages = rows // c["ps"] + 3
    x = torch.randn(rows, hq + 2 * hkv, d, generator=gen, device="cuda")
    x[:, hq:hq + hkv, 5::41] *= 4
    x = x.to(torch.bfloat16)
    qkv = [x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]]
    if not c["fused"]:
        qkv = [y.contiguous() for y in qkv]
    start = torch.randint(900000, (1,), generator=gen, device="cuda")
    at = torch.arange(rows, device="cuda")
    pos = [start + at, start + at // 64 % 48, start + at % 64][:c["axes"]]
    ids = torch.randperm(pages, generator=gen, device="cuda")
    s = dict(q=qkv[0], k=qkv[1], v=qkv[2], pos=torch.stack(pos).int(),
             slots=ids[at // c["ps"]] * c["ps"] + at % c["ps"])
    if own:
        import paper_2512_20968_amd as ma
        bf = dict(dtype=torch.bfloat16, device="cuda")
        s.update(plan=_plan(c, pages, 1), rope=ma.Rope.make(dict(
            head_dim=d, rotary_dim=c["rot"], num_axes=c["axes"],
            interleaved=c["interleaved"], inv_freq=_inv_freq(c),
            axis=_axis(c))), data=torch.zeros(
                pages, hkv, _page_bytes(c), dtype=torch.uint8, device="cuda"),
            out=[torch.empty(rows, h, d, **bf) for h in (hq, hkv, hkv)])
    return s


def prepare(case, seed):
    c = case
    gen = torch.Generator("cuda").manual_seed(seed)
    if c["kind"] == "cache":
        order = list(range(c["B"]))
        random.Random(seed).shuffle(order)
        s = _prepare_cache(c, gen, order)
    else:
        s = (_prepare_append if c["kind"] == "append" else _prepare_tile)(
            c, gen)
    s["c"] = c
    return s


# ---------------------------------------------------------------------------
# The package's entry points
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2512_20968_amd as ma
    c = s["c"]
    if c["kind"] == "fwd":
        ma.mesh_attn_score_fwd(s["prob"], *s["lists"], s["score"], s["q"],
                               s["k"], s["v"], *s["out"], ws=s["ws"])
        return s["out"]
    if c["kind"] == "bwd":
        ma.mesh_attn_score_bwd(s["prob"], *s["lists"], s["score"], s["q"],
                               s["k"], s["v"], s["o"], s["do"], s["lse"],
                               *s["out"], ws=s["ws"])
        return s["out"]
    if c["kind"] == "cache":
        ma.mesh_attn_cache_score_fwd(
            s["plan"], c["d"] ** -0.5, s["score"], s["q"], s["pos"], s["cu"],
            s["lens"], s["table"], s["data"], s["o"], s["lse"], ws=s["ws"])
        return [s["o"], s["lse"]]
    ma.mesh_attn_cache_rope_append(s["plan"], s["rope"], s["pos"], s["q"],
                                   s["out"][0], s["k"], s["v"], s["slots"],
                                   s["data"])
    ma.mesh_attn_cache_read(s["plan"], s["slots"], s["data"], s["out"][1],
                            s["out"][2])
    return s["out"]


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

PIECE = 1 << 30  # scores held at once: what a piece of the query rows makes


def _by_heads(x, hkv):
    """[rows, heads, d] as float32 [hkv, group * rows, d]."""
    rows, heads, d = x.shape
    x = x.float().view(rows, hkv, heads // hkv, d)
    return x.permute(1, 2, 0, 3).reshape(hkv, -1, d)


def _to_rows(x, heads):
    """The other way round."""
    hkv, _, d = x.shape
    x = x.view(hkv, heads // hkv, -1, d).permute(2, 0, 1, 3)
    return x.reshape(-1, heads, d)


def _hidden(c, s, rows):
    """[rows, keys] of the rows' hidden keys; None: there are none."""
    kpos, qpos = s["kpos"][None, :], s["qpos"][rows, None]
    begin, end = s["begin"], s["end"]
    if end is None and c["mask"] == "full":
        return None
    out = kpos > qpos if end is None else kpos >= end[rows, None]
    return out if begin is None else out | (kpos < begin[rows, None])


def _scored(c, x, slopes, qpos, kpos):
    """Scaled products [hkv, group, rows, keys], capped and biased in place;
    the cap's tanh, None without one."""
    t = None
    if c["cap"] > 0:
        t = x.div_(c["cap"]).tanh_()
        x = t * c["cap"]
    if slopes is not None:
        far = (qpos[:, None] - kpos[None, :]).abs().float()
        x = x.sub_(slopes.view(x.shape[0], -1, 1, 1) * far)
    return x, t


def _pieces(c, s):
    step = max(PIECE // (c["hq"] * len(s["kpos"])), 1)
    return [slice(a, a + step) for a in range(0, len(s["qpos"]), step)]


def _tile_scores(c, s, rows, k):
    hkv = c["hkv"]
    q = _by_heads(s["q"][rows], hkv)
    x = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(c["d"] ** -0.5)
    x = x.view(hkv, c["hq"] // hkv, -1, k.shape[1])
    x, t = _scored(c, x, s["slopes"], s["qpos"][rows], s["kpos"])
    hidden = _hidden(c, s, rows)
    return q, x if hidden is None else x.masked_fill_(hidden, -math.inf), t


def _softmax(x):
    top = x.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    total = x.sub_(top).exp_().sum(-1, keepdim=True)
    return x, total, top + total.log()


def _plain_fwd(c, s):
    hkv = c["hkv"]
    k, v = _by_heads(s["k"], hkv), _by_heads(s["v"], hkv)
    o, lse = [], []
    for rows in _pieces(c, s):
        _, x, _ = _tile_scores(c, s, rows, k)
        p, total, z = _softmax(x)
        y = torch.bmm(p.view(hkv, -1, k.shape[1]), v)
        y = torch.where(total.view(hkv, -1, 1) > 0,
                        y / total.view(hkv, -1, 1), 0.0)
        o.append(_to_rows(y, c["hq"]))
        lse.append(z.reshape(c["hq"], -1))
    return [torch.cat(o).to(_out(c)), torch.cat(lse, 1)]


def _plain_bwd(c, s):
    hkv, hq, scale = c["hkv"], c["hq"], c["d"] ** -0.5
    k, v = _by_heads(s["k"], hkv), _by_heads(s["v"], hkv)
    vt = v.transpose(1, 2).contiguous()
    dq, dk, dv = [], torch.zeros_like(k), torch.zeros_like(v)
    for rows in _pieces(c, s):
        q, x, t = _tile_scores(c, s, rows, k)
        do = _by_heads(s["do"][rows], hkv)
        delta = (do * _by_heads(s["o"][rows], hkv)).sum(-1, keepdim=True)
        z = s["lse"][:, rows].reshape(x.shape[:3] + (1,))
        p = x.sub_(torch.where(z == -math.inf, 0.0, z)).exp_()
        p = p.view(hkv, -1, k.shape[1])
        dv += torch.bmm(p.transpose(1, 2).contiguous(), do)
        ds = torch.bmm(do, vt).sub_(delta).mul_(p)
        if t is not None:
            ds = ds.view(t.shape).mul_(t.square_().neg_().add_(1)).view_as(p)
        dq.append(_to_rows(torch.bmm(ds, k).mul_(scale), hq))
        dk += torch.bmm(ds.transpose(1, 2).contiguous(), q).mul_(scale)
    return [torch.cat(dq).to(torch.bfloat16),
            _to_rows(dk, hkv).to(torch.bfloat16),
            _to_rows(dv, hkv).to(torch.bfloat16)]


_PAIRS = {}


def _pairs(dev):
    """The two values of every byte."""
    if dev not in _PAIRS:
        one = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=dev)
        i = torch.arange(256, device=dev)
        _PAIRS[dev] = torch.stack([one[i & 15], one[i >> 4]], -1)
    return _PAIRS[dev]


def _unpack(c, blocks):
    """K, V [.., ps, d] float32 of blocks [.., page bytes]."""
    ps, d = c["ps"], c["d"]
    lead = blocks.shape[:-1]
    kc, vc, ks, vs = blocks.split(
        [ps * d // 2, ps * d // 2, ps * d // 32, ps * d // 32], -1)
    pairs = _pairs(blocks.device)
    ks, vs = ((x.int() << 23).view(torch.float32) for x in (ks, vs))
    k = pairs[kc.int()].view(*lead, ps, d // 32, 32)
    vc = vc.reshape(*lead, ps // 8, 16, 8, d // 32).transpose(-3, -2)
    v = pairs[vc.int()].reshape(*lead, ps, d // 32, 32)
    k = k * ks.reshape(*lead, ps, d // 32, 1)
    v = v * vs.reshape(*lead, d // 32, ps).transpose(-1, -2)[..., None]
    return k.flatten(-2), v.flatten(-2)


def _plain_cache(c, s):
    lens, need = s["host"]
    hkv, g, d, ps, n = c["hkv"], c["group"], c["d"], c["ps"], c["n"]
    q, new = s["q"].float(), c["new"]
    o = torch.zeros_like(q)
    lse = torch.full((hkv * g, q.shape[0]), -math.inf, device=q.device)
    for b, (have, _) in enumerate(lens):
        rows = slice(b * new, (b + 1) * new)
        # Whole pages from the first one that a row sees.
        first = 0
        if c["window"]:
            first = _share(c, max(have - new - c["window"] + 1, 0)) // ps
        local = _share(c, have)
        if local == 0:
            continue
        blocks = s["data"][s["table"][b, first:need[b]].long()]
        kpos = torch.arange(first * ps, local, device=q.device) * n + c["p"]
        qpos = s["pos"][rows].long()
        hidden = kpos[None, :] > qpos[:, None]
        if c["window"]:
            hidden |= kpos[None, :] < s["begin"][rows, None]
        k, v = (x.transpose(0, 1).reshape(hkv, -1, d)[:, :len(kpos)]
                .contiguous() for x in _unpack(c, blocks))
        x = q[rows].view(new, hkv, g, d).permute(1, 2, 0, 3)
        x = torch.bmm(x.reshape(hkv, g * new, d),
                      k.transpose(1, 2).contiguous()).mul_(d ** -0.5)
        x, _ = _scored(c, x.view(hkv, g, new, -1), s["slopes"], qpos, kpos)
        p, total, z = _softmax(x.masked_fill_(hidden, -math.inf))
        y = torch.bmm(p.view(hkv, g * new, -1), v)
        y = torch.where(total.view(hkv, -1, 1) > 0,
                        y / total.view(hkv, -1, 1), 0.0)
        o[rows] = _to_rows(y, hkv * g)
        lse[:, rows] = z.reshape(hkv * g, -1)
    return [o.to(_out(c)), lse]


def _rotated(c, x, pos):
    """x turned by its positions, in float64: far angles need it, and values
    next to a border of the 4-bit ones."""
    half, inter = c["rot"] // 2, c["interleaved"]
    freq = torch.tensor(_inv_freq(c), dtype=torch.float64).cuda()
    angle = pos.double()[torch.tensor(_axis(c)).cuda()].transpose(0, 1) * freq
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    f = x.double()
    a = f[..., 0:c["rot"]:2] if inter else f[..., :half]
    b = f[..., 1:c["rot"]:2] if inter else f[..., half:c["rot"]]
    y = [a * cos - b * sin, b * cos + a * sin]
    y = torch.stack(y, -1).flatten(-2) if inter else torch.cat(y, -1)
    return torch.cat([y, f[..., c["rot"]:]], -1)


def _plain_append(c, s):
    return [_rotated(c, s["q"], s["pos"]).to(torch.bfloat16),
            _quantize(_rotated(c, s["k"], s["pos"]))[2].to(torch.bfloat16),
            _quantize(s["v"])[2].to(torch.bfloat16)]


def run(state):
    if own:
        return _run_own(state)
    return {"fwd": _plain_fwd, "bwd": _plain_bwd, "cache": _plain_cache,
            "append": _plain_append}[state["c"]["kind"]](state["c"], state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _pairs_seen(c):
    """(row, key) pairs that are seen, and the keys that some row sees."""
    total = c["n"] * c["P"]
    begin, end = _ranges(c)
    at = torch.arange(total)
    begin = torch.zeros(total).long() if begin is None else begin
    if end is None:
        end = at + 1 if c["mask"] != "full" else torch.full((total,), total)
    kpos, qpos = _positions(c, c["kv"]), _positions(c, c["q"])
    have = torch.zeros(total + 1).long()
    have[kpos + 1] = 1
    below = have.cumsum(0)  # keys of the tile below a position
    lo, hi = begin[qpos], end[qpos].maximum(begin[qpos])
    edge = torch.zeros(total + 1).long()
    edge.index_add_(0, lo, torch.ones_like(lo))
    edge.index_add_(0, hi, -torch.ones_like(hi))
    return (int((below[hi] - below[lo]).sum()),
            int((edge.cumsum(0)[kpos] > 0).sum()))


def work(case):
    c = case
    if c["kind"] == "append":
        rows, width = c["rows"], c["hkv"] * c["d"]
        stored = rows * (c["hkv"] * (c["d"] + c["d"] // 16) + 8)
        # Q in and out; K and V in, stored, and read back.
        return {"bytes": 4 * rows * c["group"] * width + 4 * rows * width
                + 4 * rows * c["axes"] + 2 * stored + 4 * rows * width,
                "flops": 3 * rows * (c["group"] + 1) * c["hkv"] * c["rot"]
                + 6 * rows * width}
    out = 4 if c["out"] == "fp32" else 2
    d = c["d"]
    if c["kind"] == "cache":
        lens, hq = _lengths(c), c["hkv"] * c["group"]
        stored = pairs = 0
        for have, new in lens:
            first = max(have - new - c["window"] + 1, 0) if c["window"] else 0
            stored += _share(c, have) - _share(c, first)
            for p in range(have - new, have):
                low = max(p - c["window"] + 1, 0) if c["window"] else 0
                pairs += _share(c, p + 1) - _share(c, low)
        rows = sum(n for _, n in lens)
        return {"bytes": stored * c["hkv"] * (d + d // 16)
                + rows * hq * (d * (2 + out) + 4) + 8 * rows + 8 * c["B"]
                + 4 * (stored // c["ps"]),
                "flops": 4 * d * hq * max(pairs, 1)}
    pairs, keys = _pairs_seen(c)
    rows = len(c["q"].split(",")) * c["P"]
    ranges = 4 * rows * {"docs": 2, "prefix": 2, "window": 1}.get(c["mask"], 0)
    every = len(c["kv"].split(",")) * c["P"]
    if c["kind"] == "fwd":
        return {"bytes": rows * c["hq"] * (d * (2 + out) + 4) + ranges
                + 4 * keys * c["hkv"] * d,
                "flops": 4 * d * c["hq"] * max(pairs, 1)}
    return {"bytes": rows * c["hq"] * (8 * d + 4) + ranges
            + 4 * (keys + every) * c["hkv"] * d,
            "flops": 10 * d * c["hq"] * max(pairs, 1)}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_scores(c, q, k, qpos, kpos, lo, hi, slope):
    """x [rows, keys] of one head, and its derivative by the product."""
    x = (q.double() @ k.double().T) / math.sqrt(c["d"])
    grad = torch.ones_like(x)
    if c["cap"] > 0:
        grad = 1 / torch.cosh(x / c["cap"]) ** 2
        x = c["cap"] * torch.tanh(x / c["cap"])
    if slope:
        x = x - slope * (qpos[:, None] - kpos[None, :]).abs().double()
    seen = (lo[:, None] <= kpos[None, :]) & (kpos[None, :] < hi[:, None])
    return torch.where(seen, x, -math.inf), grad


def _exact_weights(x, z):
    return torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])


def _exact_tile(c, s):
    hq, g = c["hq"], c["hq"] // c["hkv"]
    qpos, kpos = s["qpos"], s["kpos"]
    lo = torch.zeros_like(qpos) if s["begin"] is None else s["begin"].long()
    hi = s["end"].long() if s["end"] is not None else (
        qpos + 1 if c["mask"] != "full" else qpos * 0 + c["n"] * c["P"])
    slope = s["slopes"].double().tolist() if c["slopes"] else [0.0] * hq
    q, k, v = s["q"], s["k"], s["v"]
    new = dict(dtype=torch.float64, device="cuda")
    out = [torch.zeros(x.shape, **new) for x in (q, k, v)]
    lse = torch.zeros(hq, len(qpos), **new)
    for h in range(hq):
        x, grad = _exact_scores(c, q[:, h], k[:, h // g], qpos, kpos, lo, hi,
                                slope[h])
        if c["kind"] == "fwd":
            lse[h] = torch.logsumexp(x, 1)
            out[0][:, h] = _exact_weights(x, lse[h]) @ v[:, h // g].double()
            continue
        p = _exact_weights(x, s["lse"][h].double())
        do = s["do"][:, h].double()
        ds = p * grad * (do @ v[:, h // g].double().T
                         - (do * s["o"][:, h].double()).sum(1)[:, None])
        ds /= math.sqrt(c["d"])
        out[0][:, h] = ds @ k[:, h // g].double()
        out[1][:, h // g] += ds.T @ q[:, h].double()
        out[2][:, h // g] += p.T @ do
    return [out[0], lse] if c["kind"] == "fwd" else out


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
        code = (flat[a].int() >> (4 * (dim % 2))) & 15
        e, m = (code >> 1) & 3, (code & 1).double()
        x = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e.double() - 1))
        x = torch.where(code > 7, -x, x)
        out.append(x * 2.0 ** (flat[sa].double() - 127))
    return out


def _exact_cache(c, s):
    lens, _ = s["host"]
    hkv, g, d, new = c["hkv"], c["group"], c["d"], c["new"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((hkv * g, len(o)), -math.inf, dtype=torch.float64,
                     device="cuda")
    slope = s["slopes"].double().tolist() if c["slopes"] else [0.0] * hkv * g
    for b, (have, _) in enumerate(lens):
        local, r = _share(c, have), slice(b * new, (b + 1) * new)
        if local == 0:
            continue
        key = torch.arange(local, device="cuda")
        page = s["table"][b].long()[key // c["ps"]]
        qpos = s["pos"][r].long()
        lo = s["begin"][r].long() if c["window"] else qpos * 0
        for h in range(hkv * g):
            if h % g == 0:
                k, v = _exact_rows(c, s["data"], page, key % c["ps"], h // g)
            x, _ = _exact_scores(c, s["q"][r, h], k, qpos,
                                 key * c["n"] + c["p"], lo, qpos + 1, slope[h])
            lse[h, r] = torch.logsumexp(x, 1)
            o[r, h] = _exact_weights(x, lse[h, r]) @ v
    return [o, lse]


def _exact_append(c, s):
    turned = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        for i, (f, axis) in enumerate(zip(_inv_freq(c), _axis(c))):
            j, l = ((2 * i, 2 * i + 1) if c["interleaved"]
                    else (i, i + c["rot"] // 2))
            phi = (s["pos"][axis].double() * f)[:, None]
            a, b = x[..., j].double(), x[..., l].double()
            y[..., j] = a * torch.cos(phi) - b * torch.sin(phi)
            y[..., l] = a * torch.sin(phi) + b * torch.cos(phi)
        turned.append(y)
    out = [turned[0]]
    values = torch.tensor(E2M1, dtype=torch.float64).cuda()
    for x in (turned[1], s["v"].double()):
        parts = []
        for y in x.split(2048):
            w = y.reshape(-1, 32)
            mant, exp = torch.frexp(w.abs().max(1).values)
            e = torch.where(mant == 0, -126, exp - 3 + (mant > 0.875).int())
            unit = (2.0 ** e.clamp(-126, 125).double())[:, None]
            a = w.abs() / unit
            code = torch.zeros_like(a, dtype=torch.long)
            for i in range(7):
                mid = (values[i] + values[i + 1]) / 2
                code += (a >= mid) if i % 2 else (a > mid)  # ties: even code
            parts.append((torch.copysign(values[code], w) * unit)
                         .view(y.shape))
        out.append(torch.cat(parts))
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"cache": _exact_cache, "append": _exact_append}.get(
        c["kind"], _exact_tile)(c, s)
