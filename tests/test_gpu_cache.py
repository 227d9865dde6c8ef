"""The 4-bit key/value cache on the GPU: page tables, append, read and the
attention over it, against the float64 oracle and definitions."""

import numpy as np
import pytest
import torch

import paper_2512_20968_amd as ma
from oracle import cache as oc

from helpers import ExactScores

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def cache_of(**kw):
    c = dict(num_pages=40, page_size=16, num_kv_heads=2, head_dim=64,
             max_pages=12, layout=1, num_partitions=1, partition=0,
             partition_len=0)
    c.update(kw)
    return c


def random_bytes(c, seed=0):
    """A cache that was never written: any bytes, NaN scales among them."""
    gen = torch.Generator("cuda").manual_seed(seed)
    data = torch.randint(0, 256, (c["num_pages"], c["num_kv_heads"],
                                  oc.page_bytes(c)), dtype=torch.uint8,
                         device="cuda", generator=gen)
    data[torch.rand(data.shape, device="cuda", generator=gen) < 0.05] = 255
    return data


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def i64(x):
    return torch.tensor(np.asarray(x), dtype=torch.int64).cuda()


# -- the conversions ----------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
def test_read_every_code_and_scale(d):
    """Every byte of codes under every scale code that append writes, and the
    NaN code: the values are exact."""
    c = cache_of(num_pages=256, num_kv_heads=1, head_dim=d)
    data = np.zeros((256, 1, oc.page_bytes(c)), dtype=np.uint8)
    n = 16 * d // 2
    data[:, 0, :n] = (np.arange(n) * 37 + np.arange(256)[:, None]) % 256
    data[:, 0, n:2 * n] = (np.arange(n) + np.arange(256)[:, None]) % 256
    data[:, 0, 2 * n:] = np.arange(256)[:, None]  # page i: scale code i
    slots = np.arange(256 * 16)
    k = torch.empty(len(slots), 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    ma.mesh_attn_cache_read(c, i64(slots), torch.tensor(data).cuda(), k, v)
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    for s in slots:
        if s // 16 in (0, 253, 254):
            continue  # never written
        wk, wv = oc.read_row(c, data, s)
        np.testing.assert_array_equal(k[s], wk)
        np.testing.assert_array_equal(v[s], wv)


def append_inputs(d, hkv, rows, seed):
    """bf16 rows with every kind of group: all magnitudes, zeros, infinities,
    NaN, ties, subnormals."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, hkv, d))
    x *= 2.0 ** rng.integers(-140, 128, (rows, hkv, d // 32)).repeat(32, -1)
    x[::5] = rng.choice(np.arange(-28, 29) / 4.0, (len(x[::5]), hkv, d))
    x[1::11, :, :32] = 0
    x[2::13, 0, 3] = np.inf
    x[3::17, 0, 40] = np.nan
    x[4::19, 0, 5] = -np.inf
    t = torch.tensor(x).to(torch.float32).to(torch.bfloat16)
    if seed % 2:  # any bit pattern
        bits = torch.tensor(rng.integers(0, 65536, (rows, hkv, d)))
        t[6::7] = bits.to(torch.uint16).view(torch.bfloat16)[6::7]
    return t


@pytest.mark.parametrize("d,hkv,ps,rows", [
    (128, 1, 16, 1), (64, 3, 16, 7), (128, 2, 64, 33), (64, 2, 256, 300),
    (128, 5, 32, 161), (128, 1, 128, 257)])
def test_append_is_the_oracle_byte_for_byte(d, hkv, ps, rows):
    c = cache_of(head_dim=d, num_kv_heads=hkv, page_size=ps, num_pages=21)
    rng = np.random.default_rng(rows)
    total = 21 * ps
    slots = rng.permutation(total)[:rows]
    if rows > 5:
        slots[2], slots[3], slots[4] = -1, total, 2**40
    k, v = append_inputs(d, hkv, rows, 2 * d), append_inputs(d, hkv, rows, 77)
    data = random_bytes(c)
    want = data.cpu().numpy().copy()
    # Slices of a fused projection: row strides of their own.
    fused = torch.zeros(rows, 3 * hkv, d, dtype=torch.bfloat16, device="cuda")
    fused[:, hkv:2 * hkv], fused[:, 2 * hkv:] = k.cuda(), v.cuda()
    ma.mesh_attn_cache_append(c, fused[:, hkv:2 * hkv], fused[:, 2 * hkv:],
                              i64(slots), data)
    oc.write_rows(c, want, k.double().numpy(), v.double().numpy(), slots)
    np.testing.assert_array_equal(data.cpu().numpy(), want)
    ko = torch.full((rows, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    vo = ko.clone()
    ma.mesh_attn_cache_read(c, i64(slots), data, ko, vo)
    for r, s in enumerate(slots):
        wk, wv = oc.read_row(c, want, s)
        np.testing.assert_array_equal(ko[r].double().cpu().numpy(), wk)
        np.testing.assert_array_equal(vo[r].double().cpu().numpy(), wv)


@pytest.mark.parametrize("start", [0, 16, 5])
@pytest.mark.parametrize("d,ps", [(128, 64), (64, 16), (128, 16), (64, 128)])
def test_append_runs_of_slots(d, ps, start):
    """A prompt's rows: runs of slots, aligned or not, with a gap and a page
    change inside a workgroup's rows."""
    c = cache_of(head_dim=d, page_size=ps, num_pages=30)
    pages = np.random.default_rng(start).permutation(30)
    rows = 150
    at = start + np.arange(rows)
    slots = pages[at // ps] * ps + at % ps
    slots[70] = -1
    slots[100:] += 0
    k, v = append_inputs(d, 2, rows, 4), append_inputs(d, 2, rows, 9)
    data = random_bytes(c, 3)
    want = data.cpu().numpy().copy()
    ma.mesh_attn_cache_append(c, k.cuda(), v.cuda(), i64(slots), data)
    oc.write_rows(c, want, k.double().numpy(), v.double().numpy(), slots)
    np.testing.assert_array_equal(data.cpu().numpy(), want)


# -- tables -------------------------------------------------------------------

def run_tables(c, lens, new, free, rng, table, rows, stream=None):
    b = len(lens)
    out = dict(table=i32(table).view(b, c["max_pages"]),
               lens=torch.full((b,), -7, **I32),
               cu=torch.full((b + 1,), -7, **I32),
               slots=torch.full((rows,), -7, dtype=torch.int64, device="cuda"),
               pos=torch.full((rows,), -7, **I32),
               rng=torch.full((2,), -7, **I32),
               refused=torch.full((1,), -7, **I32))
    ma.mesh_attn_cache_tables(c, i32(lens), i32(new), i32(free), i32(rng),
                              out["table"], out["lens"], out["cu"],
                              out["slots"], out["pos"], out["rng"],
                              out["refused"], stream=stream)
    return [x.cpu().numpy() for x in out.values()]


SHARES = [dict(), dict(num_partitions=3, partition=1),
          dict(num_partitions=5, partition=4),
          dict(layout=0, num_partitions=3, partition=1, partition_len=70)]


@pytest.mark.parametrize("share", SHARES)
@pytest.mark.parametrize("b", [1, 2, 63, 64, 65, 300])
def test_tables(share, b):
    rng = np.random.default_rng(b)
    c = cache_of(num_pages=4000, max_pages=14, **share)
    for round_ in range(3):
        lens = rng.integers(0, 230, b)
        new = rng.choice([0, 1, 1, 2, 17, 90], b)
        lens[rng.random(b) < 0.1] = -3
        new[rng.random(b) < 0.05] = -1
        lens[rng.random(b) < 0.02] = 2**31 - 1
        ids = rng.permutation(4000)
        table = np.full((b, 14), -1)
        for i in range(b):
            n = min(-(-oc.stored(c, max(int(lens[i]), 0)) // 16), 14)
            table[i, :n] = ids[:n]
            ids = ids[n:] if len(ids) > n + 300 else ids
        if b > 1 and round_ == 1:
            table[1] = 4000  # not a page
        free = ids[:max(1, (b * 2, b, 3 * b)[round_])]
        first = (0, 3, 1)[round_]
        last = (len(free), len(free) + 9, len(free) - 1)[round_]
        total = int(np.maximum(new, 0).sum())
        rows = max((total, total + 13, total // 2)[round_], 0)
        got = run_tables(c, lens, new, free, [first, last], table, rows)
        want = oc.tables(c, lens, new, free, [first, last], table, rows)
        for g, w in zip(got, want):
            np.testing.assert_array_equal(g, w)


def test_tables_edges():
    c = cache_of()
    got = run_tables(c, np.zeros(0), np.zeros(0), [3], [0, 1],
                     np.zeros((0, 12)), 5)
    assert got[2].tolist() == [0] and got[3].tolist() == [-1] * 5
    assert got[5].tolist() == [0, 1] and got[6].tolist() == [0]
    # No free page at all, ranges that make no sense, sums past 31 bits.
    for rng in ([0, 0], [5, 2], [-4, 100], [2**31 - 1, -2**31]):
        lens, new = [4, 16, 0], [2**31 - 1, 1, 2**31 - 1]
        got = run_tables(c, lens, new, [], rng, np.zeros((3, 12)), 40)
        want = oc.tables(c, lens, new, [], rng, np.zeros((3, 12)), 40)
        for g, w in zip(got, want):
            np.testing.assert_array_equal(g, w)


def test_tables_most_requests_and_long_rows():
    rng = np.random.default_rng(2)
    b = 4096
    c = cache_of(num_pages=70000, page_size=16, max_pages=200)
    lens, new = rng.integers(0, 60, b), rng.integers(0, 3, b)
    new[17], new[4095] = 2500, 900
    table = np.full((b, 200), -1)
    ids = rng.permutation(70000)
    at = 0
    for i in range(b):
        n = -(-int(lens[i]) // 16)
        table[i, :n] = ids[at:at + n]
        at += n
    free = ids[at:]
    rows = int(new.sum()) + 100
    got = run_tables(c, lens, new, free, [0, len(free)], table, rows)
    want = oc.tables(c, lens, new, free, [0, len(free)], table, rows)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g, w)


# -- attention ----------------------------------------------------------------

class Batch:
    """Requests over a cache that holds append's K, V (the rest: any bytes)."""

    def __init__(self, c, lens, new, group=2, seed=0, positions=None, pad=0,
                 k_scale=1.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.c, self.new = c, list(new)
        ps, hkv, d = c["page_size"], c["num_kv_heads"], c["head_dim"]
        self.hq = hkv * group
        local = [min(oc.stored(c, n), ps * c["max_pages"]) for n in lens]
        need = [-(-n // ps) for n in local]
        assert sum(need) <= c["num_pages"]
        ids = rng.permutation(c["num_pages"])
        self.table = np.full((len(lens), c["max_pages"]), -1)
        at = 0
        slots = []
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
            r = np.arange(local[b])
            slots.append(self.table[b, r // ps] * ps + r % ps)
        slots = np.concatenate(slots).astype(np.int64)
        self.k = torch.randn(len(slots), hkv, d, generator=gen) * k_scale
        self.v = torch.randn(len(slots), hkv, d, generator=gen)
        self.k = self.k.to(torch.bfloat16)
        self.v = self.v.to(torch.bfloat16)
        self.slots = slots
        self.data = random_bytes(c, seed)
        ma.mesh_attn_cache_append(c, self.k.cuda(), self.v.cuda(), i64(slots),
                                  self.data)
        self.lens = np.array(lens)
        self.cu = np.concatenate([[0], np.cumsum(new)])
        rows = int(self.cu[-1]) + pad
        if positions is None:
            positions = np.concatenate(
                [np.arange(n - m, n) for n, m in zip(lens, new)]
                + [np.full(pad, 3)])
        self.positions = np.asarray(positions)
        self.q = torch.randn(rows, self.hq, d, generator=gen).to(
            torch.bfloat16)
        self.scale = d ** -0.5

    def run(self, dtype=torch.float32, q=None, ws=None, stream=None):
        rows = self.q.shape[0]
        o = torch.full((rows, self.hq, self.c["head_dim"]), 123.0,
                       dtype=dtype, device="cuda")
        lse = torch.full((self.hq, rows), 123.0, device="cuda")
        ma.mesh_attn_cache_fwd(
            self.c, self.scale, self.q.cuda() if q is None else q,
            i32(self.positions), i32(self.cu), i32(self.lens), i32(self.table),
            self.data, o, lse, ws=ws, stream=stream)
        return o, lse

    def want(self, heads=None):
        """As oracle.cache.attention, of all keys of a request at once; of some
        heads."""
        c = self.c
        rows, hq, d = self.q.shape
        hkv, ps = c["num_kv_heads"], c["page_size"]
        group = hq // hkv
        q = self.q.double().numpy()
        o, mass = np.full((2, rows, hq, d), np.nan)
        lse, reach = np.full((2, hq, rows), np.nan)
        for b in range(len(self.lens)):
            lo = max(int(self.cu[b]), 0)
            hi = min(int(self.cu[b + 1]), rows)
            if hi <= lo:
                continue
            n = min(oc.stored(c, max(int(self.lens[b]), 0)),
                    c["max_pages"] * ps)
            r = np.arange(n)
            page = self.table[b, r // ps]
            ok = (page >= 0) & (page < c["num_pages"])
            slots = np.where(ok, page * ps + r % ps, -1)
            k = torch.empty(n, hkv, d, dtype=torch.bfloat16, device="cuda")
            v = torch.empty_like(k)
            ma.mesh_attn_cache_read(c, i64(slots), self.data, k, v)
            k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
            sees = ok[None] & (oc.key_positions(c, n)[None]
                               <= self.positions[lo:hi, None])
            for h in range(hq) if heads is None else heads:
                kh, vh = k[:, h // group], v[:, h // group]
                x = self.scale * (q[lo:hi, h] @ kh.T)
                x[~sees] = -np.inf
                top = x.max(1, initial=-np.inf)
                top = np.where(np.isinf(top), 0.0, top)
                p = np.exp(x - top[:, None])
                p[~sees] = 0.0
                s = p.sum(1)
                full = np.where(s == 0, 1.0, s)[:, None]
                with np.errstate(divide="ignore"):
                    lse[h, lo:hi] = top + np.log(s)
                # A hidden key's V does not count, whatever it is.
                o[lo:hi, h] = [pp[m] @ vh[m] for pp, m in zip(p / full, sees)]
                mass[lo:hi, h] = [pp[m] @ np.abs(vh[m])
                                  for pp, m in zip(p / full, sees)]
                reach[h, lo:hi] = [
                    self.scale * (np.abs(kh[m]) @ np.abs(qq)).max(initial=0.0)
                    for qq, m in zip(q[lo:hi, h], sees)]
        if heads is not None:
            o, lse, mass, reach = o[:, heads], lse[heads], mass[:, heads], \
                reach[heads]
        return o, lse, mass, reach


def check(got, want, d, keys=4096):
    """Errors against a bound by arithmetic.  With u = 2^-24 and reach = scale
    * max_j sum_i |q_i k_ji|: a score is a float32 sum of d exact products
    (truncation allowed for: 2u each) times a rounded scale, so it is off by at
    most (d + 16) 2u reach; a probability by twice that and its exponential's
    and the sums' roundings, together (the 2^-23 of a probability's three bf16
    parts for a float32 O too) below 2^-14 for up to 4096 keys; bf16 O adds 2^-8
    for the probabilities and 2^-8 for itself."""
    o, lse = (x.double().cpu().numpy() for x in got)
    wo, wl, mass, reach = want
    live = ~np.isnan(reach)
    rows = live.T[..., None].repeat(d, -1)
    bad = np.isnan(wo) & rows
    np.testing.assert_array_equal(np.isnan(o) & rows, bad)
    rel = 2 * (d + 16) * 2.0**-23 * reach.T[..., None] + 2.0**-14
    tol = mass * rel
    if got[0].dtype == torch.bfloat16:
        tol = tol + (mass + np.abs(wo)) * 2.0**-8
    ok = ~(np.abs(o - wo) > tol)
    assert np.all(ok[rows & ~bad]), np.nanmax(np.where(rows, np.abs(o - wo)
                                                       - tol, -1))
    nl = np.isnan(wl) & live
    np.testing.assert_array_equal(np.isnan(lse) & live, nl)
    empty = live & (wl == -np.inf)
    assert np.all(lse[empty] == -np.inf)
    assert np.all(o[empty.T] == 0)
    fine = live & ~nl & ~empty
    ltol = (d + 16) * 2.0**-23 * reach + 2.0**-14 + np.abs(wl) * 2.0**-22
    assert np.all(np.abs(lse[fine] - wl[fine]) <= ltol[fine])
    # Rows of no request are left alone.
    assert np.all(o[~live.T] == 123.0) and np.all(lse[~live] == 123.0)


@pytest.mark.parametrize("d,hkv,group,new,requests,pages", [
    (128, 2, 4, 1, 40, 1), (64, 2, 2, 1, 40, 200), (128, 2, 4, 8, 11, 200),
    (64, 1, 3, 40, 5, 1), (128, 1, 4, 30, 5, 200), (64, 16, 2, 1, 520, 1),
    (128, 16, 4, 12, 90, 1)])
def test_float32_probabilities_keep_24_bits(d, hkv, group, new, requests,
                                            pages):
    """Exact scores and values of one sign, two keys a request: what is left of
    a float32 O's error (the bound is derived beside the inputs), too little for
    probabilities of two bf16."""
    c = cache_of(head_dim=d, num_kv_heads=hkv, num_pages=requests,
                 max_pages=pages)
    x = ExactScores(requests, new, hkv, group, d)
    slots = (np.arange(requests)[:, None] * 16 + np.arange(2)).ravel()
    data = random_bytes(c)
    bf = [torch.tensor(a).to(torch.bfloat16).cuda() for a in (x.q, x.k, x.v)]
    ma.mesh_attn_cache_append(c, bf[1], bf[2], i64(slots), data)
    rows = requests * new
    table = np.full((requests, pages), -1)
    table[:, 0] = np.arange(requests)
    o = torch.full((rows, hkv * group, d), 123.0, device="cuda")
    lse = torch.full((hkv * group, rows), 123.0, device="cuda")
    ma.mesh_attn_cache_fwd(c, x.scale, bf[0], i32([1] * rows),
                           i32(np.arange(requests + 1) * new),
                           i32([2] * requests), i32(table), data, o, lse)
    want_o, want_lse = x.want()
    got = o.double().cpu().numpy()
    assert np.all(np.abs(got - want_o) <= x.O_BOUND * want_o)
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse)
                  <= x.LSE_BOUND)


LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 160, 190]


def test_small_batch_against_the_oracle():
    for share in SHARES:
        c = cache_of(num_pages=60, **share)
        b = Batch(c, [1, 40, 0, 130], [1, 3, 0, 5], seed=1)
        want = oc.attention(c, b.scale, b.q.double().numpy(), b.positions,
                            b.cu, b.lens, b.table, b.data.cpu().numpy())
        mine = b.want()
        for x, y in zip(want, mine):
            np.testing.assert_allclose(x, y, atol=1e-12)
        check(b.run(), want, 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lengths_around_every_border(d, ps, dtype):
    c = cache_of(head_dim=d, page_size=ps, max_pages=max(12, 256 // ps),
                 num_pages=130)
    b = Batch(c, LENGTHS, [1] * len(LENGTHS), group=3, seed=ps + d)
    check(b.run(dtype), b.want(), d)


@pytest.mark.parametrize("d,hkv,group", [
    (128, 1, 1), (64, 5, 1), (128, 2, 4), (128, 1, 7), (64, 2, 8),
    (128, 1, 16), (64, 1, 17), (128, 2, 40), (64, 1, 71)])
@pytest.mark.parametrize("new", [1, 2, 6, 33])
def test_rows_and_groups(d, hkv, group, new):
    c = cache_of(head_dim=d, num_kv_heads=hkv, page_size=32)
    lens = [new, 40 + new, 301]
    b = Batch(c, lens, [new, new, 1], group=group, seed=new)
    check(b.run(torch.float32 if new % 2 else torch.bfloat16), b.want(), d)


@pytest.mark.parametrize("share", SHARES)
@pytest.mark.parametrize("d", [64, 128])
def test_shares_and_rows_without_keys(share, d):
    """Rows before the first stored position, positions of -1 and far past the
    end, a length past the table."""
    c = cache_of(head_dim=d, num_pages=60, **share)
    lens = [1, 2, 100, 190, 5000]  # the last one past the table
    new = [1, 2, 7, 20, 3]
    b = Batch(c, lens, new, group=4, seed=4)
    b.positions[5] = -1
    b.positions[6] = 2**31 - 1
    b.positions[7] = -2**31
    check(b.run(), b.want(), d)
    check(b.run(torch.bfloat16), b.want(), d)


@pytest.mark.parametrize("d", [64, 128])
def test_bad_pages_hide_their_keys(d):
    c = cache_of(head_dim=d)
    b = Batch(c, [100, 150, 16, 190], [2, 1, 1, 4], group=4, seed=5)
    b.table[0, 2] = -1
    b.table[0, 6] = 40
    b.table[1, 0] = 2**31 - 1
    b.table[2, 0] = -2**31  # all of its keys
    b.table[3, 11] = 41
    check(b.run(), b.want(), d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nan_reaches_the_rows_that_see_it(d, dtype):
    c = cache_of(head_dim=d, num_kv_heads=1)
    for at, what in ((5, "k"), (150, "k"), (181, "k"), (0, "v"), (185, "v"),
                     (170, "v"), (189, "v")):
        b = Batch(c, [190, 30], [12, 2], group=3, seed=6)
        slot = i64([b.slots[at]])
        k, v = b.k[at:at + 1].cuda(), b.v[at:at + 1].cuda()
        (k if what == "k" else v)[0, 0, 40] = float("nan")
        (k if what == "k" else v)[0, 0, 2] = -float("inf") if at % 2 else 1.0
        ma.mesh_attn_cache_append(c, k, v, slot, b.data)
        o, lse, mass, reach = b.want()
        seen = (np.arange(14) < 12) & (b.positions >= at)
        # A NaN score makes the row NaN; a NaN value its group of dims.
        if what == "k":
            lse[:, seen] = np.nan
            o[seen] = np.nan
        else:
            o[seen, :, 32:64] = np.nan
            if at % 2:
                o[seen, :, :32] = np.nan
        check(b.run(dtype), (o, lse, np.nan_to_num(mass),
                             np.nan_to_num(reach) + 0 * b.positions), d)


def test_no_key_survives_a_nan_length_of_garbage():
    """Rows behind the last request stay; a decreasing or absurd cu_new touches
    nothing outside the buffers."""
    c = cache_of()
    b = Batch(c, [50, 60], [3, 2], pad=4, seed=7)
    check(b.run(), b.want(), 64)
    for cu in ([0, 3, 1], [-5, 3, 2**31 - 1], [9, 9, 9], [4, 0, 2]):
        b.cu = np.array(cu)
        o, lse = b.run()
        assert o.shape[0] == 9 and not torch.isnan(lse).any()


@pytest.mark.parametrize("d,group,rows,dtype", [
    (64, 2, 9, torch.float32), (128, 4, 70, torch.bfloat16),
    (128, 8, 300, torch.float32)])
def test_absurd_row_ranges_stay_inside_the_buffers(d, group, rows, dtype):
    """cu_new that decreases, or lies outside the rows: the rows it still gives
    to a request are right, all others and what lies around O and LSE as they
    were."""
    c = cache_of(head_dim=d, page_size=64, num_pages=100, max_pages=40)
    b = Batch(c, [700, 60], [rows - 4, 2], group=group, seed=7, pad=2)
    b.positions = np.random.default_rng(rows).integers(-2, 800, rows)
    top, guard, heads = 2**31 - 1, 4096, [0, b.hq - 1]
    for cu in ([0, 3, 1], [-5, 3, top], [rows, rows, rows], [4, 0, 2],
               [-top - 1, -7, -3], [top, top, top], [0, top, 0],
               [rows - 1, rows + 1, top], [2, 2, rows], [rows + 9, 1, rows]):
        b.cu = np.array(cu)
        flat = [torch.full((guard + n + guard,), 123.0, dtype=t, device="cuda")
                for n, t in ((rows * b.hq * d, dtype),
                             (b.hq * rows, torch.float32))]
        o = flat[0][guard:-guard].view(rows, b.hq, d)
        lse = flat[1][guard:-guard].view(b.hq, rows)
        ma.mesh_attn_cache_fwd(c, b.scale, b.q.cuda(), i32(b.positions),
                               i32(b.cu), i32(b.lens), i32(b.table), b.data, o,
                               lse)
        for x in flat:
            assert torch.all(x[:guard] == 123.0), cu
            assert torch.all(x[-guard:] == 123.0), cu
        want = b.want(heads)
        check((o[:, heads], lse[heads]), want, d)
        of_none = torch.tensor(np.isnan(want[3][0])).cuda()
        assert torch.all(o[of_none] == 123.0), cu
        assert torch.all(lse[:, of_none] == 123.0), cu


@pytest.mark.parametrize("d,ps,share", [(128, 64, SHARES[0]),
                                        (128, 16, SHARES[1]),
                                        (64, 256, SHARES[3])])
def test_ragged_batch_against_the_oracles_own_reader(d, ps, share):
    """Keys and values by the oracle from the cache's bytes, none of them by the
    read kernel; several pages a request, and one of them not a page."""
    c = cache_of(head_dim=d, page_size=ps, num_pages=60,
                 max_pages=max(2, 320 // ps), **share)
    b = Batch(c, [300, 0, 65, 17, 129], [3, 0, 1, 2, 1], group=3, seed=27,
              pad=1)
    b.table[4, 0] = 60
    want = oc.attention(c, b.scale, b.q.double().numpy(), b.positions, b.cu,
                        b.lens, b.table, b.data.cpu().numpy())
    check(b.run(), want, d)
    check(b.run(torch.bfloat16), want, d)


def test_requests_that_share_pages_and_positions_in_any_order():
    c = cache_of(head_dim=128, num_pages=60)
    b = Batch(c, [190, 170, 190, 40], [9, 5, 17, 1], group=4, seed=16)
    b.table[1, :8] = b.table[0, :8]
    b.table[2] = b.table[0]
    rng = np.random.default_rng(16)
    for _ in range(2):
        check(b.run(), b.want(), 128)
        check(b.run(torch.bfloat16), b.want(), 128)
        b.positions = rng.integers(-2, 200, len(b.positions))


def test_scores_of_every_size():
    """Large scores (one key dominates), and late maxima: keys grow along the
    sequence, so that the running maximum moves at every step."""
    c = cache_of(head_dim=128, num_pages=60, max_pages=40)
    b = Batch(c, [600], [3], group=4, seed=8, k_scale=30.0)
    check(b.run(), b.want(), 128)
    b = Batch(c, [600], [3], group=4, seed=9)
    grow = torch.linspace(0.01, 8, 600)[:, None, None]
    ma.mesh_attn_cache_append(c, (b.k * grow).to(torch.bfloat16).cuda(),
                              b.v.cuda(), i64(b.slots), b.data)
    check(b.run(), b.want(), 128)


def test_query_slices_streams_and_workspaces():
    c = cache_of(head_dim=128)
    b = Batch(c, [100, 150, 190], [1, 1, 3], group=4, seed=10)
    want_o, want_l = b.run()
    fused = torch.zeros(5, 8 + 4, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, :8] = b.q.cuda()
    o, lse = b.run(q=fused[:, :8])
    assert torch.equal(o, want_o) and torch.equal(lse, want_l)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = b.run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, want_o) and torch.equal(lse, want_l)


RAGGED = [3, 4000, 17, 0, 1, 900, 2500, 64, 65, 1300, 7, 5200]


@pytest.mark.parametrize("d,ps,hkv,group", [
    (128, 64, 8, 4), (64, 16, 2, 8), (128, 16, 1, 20), (128, 256, 4, 1)])
@pytest.mark.parametrize("new", [1, 3])
def test_ragged_lengths(d, ps, hkv, group, new):
    """Lengths that differ by orders of magnitude share the workgroups."""
    c = cache_of(head_dim=d, page_size=ps, num_kv_heads=hkv, num_pages=1000,
                 max_pages=5400 // ps)
    news = [min(new, n) for n in RAGGED]
    b = Batch(c, RAGGED, news, group=group, seed=11)
    want = b.want()
    got = b.run()
    check(got, want, d)
    again = b.run()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    check(b.run(torch.bfloat16), want, d)


@pytest.mark.parametrize("d,hkv,group,new,have", [
    (128, 2, 4, 200, 333), (64, 1, 1, 517, 0), (128, 1, 8, 97, 1200),
    (64, 2, 5, 130, 64)])
def test_prompt_chunks(d, hkv, group, new, have):
    c = cache_of(head_dim=d, num_kv_heads=hkv, page_size=64, num_pages=60,
                 max_pages=24)
    b = Batch(c, [have + new, 70, 0], [new, 1, 0], group=group, seed=12)
    want = b.want()
    check(b.run(), want, d)
    check(b.run(torch.bfloat16), want, d)


def test_far_pages():
    """Pages whose byte offsets pass 2^32, slots of any number."""
    c = cache_of(num_pages=70000, page_size=64, num_kv_heads=8, head_dim=128,
                 max_pages=4)
    data = torch.zeros(70000, 8, oc.page_bytes(c), dtype=torch.uint8,
                       device="cuda")
    assert data.numel() > 2**32
    gen = torch.Generator().manual_seed(3)
    k, v = torch.randn(2, 200, 8, 128, generator=gen).to(torch.bfloat16)
    table = np.array([[69999, 5, 69998, 62000]])
    r = np.arange(200)
    slots = table[0, r // 64] * 64 + r % 64
    ma.mesh_attn_cache_append(c, k.cuda(), v.cuda(), i64(slots), data)
    small = cache_of(num_pages=4, page_size=64, num_kv_heads=8, head_dim=128,
                     max_pages=4)
    near = torch.zeros(4, 8, oc.page_bytes(c), dtype=torch.uint8,
                       device="cuda")
    ma.mesh_attn_cache_append(small, k.cuda(), v.cuda(), i64(r), near)
    assert torch.equal(data[i64(table[0])], near)
    ko, vo = torch.empty(2, 200, 8, 128, dtype=torch.bfloat16, device="cuda")
    kn, vn = torch.empty_like(ko), torch.empty_like(vo)
    ma.mesh_attn_cache_read(c, i64(slots), data, ko, vo)
    ma.mesh_attn_cache_read(small, i64(r), near, kn, vn)
    assert torch.equal(ko, kn) and torch.equal(vo, vn)
    q = torch.randn(1, 32, 128, generator=gen).to(torch.bfloat16).cuda()
    out = []
    for cc, t, dd in ((c, table, data), (small, [[0, 1, 2, 3]], near)):
        o = torch.empty(1, 32, 128, device="cuda")
        lse = torch.empty(32, 1, device="cuda")
        ma.mesh_attn_cache_fwd(cc, 0.1, q, i32([199]), i32([0, 1]), i32([200]),
                               i32(t), dd, o, lse)
        out.append((o, lse))
    assert torch.equal(out[0][0], out[1][0])
    assert torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("b,new", [(257, 1), (1000, 1), (4096, 1), (300, 3)])
def test_many_requests(b, new, hkv=1):
    """More requests than a workgroup keeps the lengths of, up to the limit."""
    rng = np.random.default_rng(b)
    c = cache_of(num_pages=8000, page_size=16, num_kv_heads=hkv, max_pages=70)
    lens = np.minimum(np.exp(rng.uniform(0, 4.5, b)).astype(int), 60)
    lens[rng.integers(b)] = 1100
    lens = np.maximum(lens, new)
    lens[:3] = 0
    news = np.where(lens > 0, new, 0)
    x = Batch(c, lens.tolist(), news.tolist(), group=2, seed=b)
    check(x.run(), x.want(), 64)


def test_many_heads_of_many_requests():
    """More sequences than workgroups, several of one to a workgroup."""
    test_many_requests(1300, 1, hkv=6)


@pytest.mark.parametrize("d,group,new,dtype", [
    (64, 3, 1, torch.float32), (128, 2, 1, torch.bfloat16),
    (128, 5, 4, torch.float32), (128, 7, 6, torch.bfloat16),
    (64, 4, 20, torch.bfloat16)])
def test_a_sequence_of_hundreds_of_runs(d, group, new, dtype):
    """Every run keeps a few hundred keys: no sum is longer than before."""
    c = cache_of(head_dim=d, page_size=64, num_kv_heads=1, num_pages=700,
                 max_pages=600)
    b = Batch(c, [38000, 5, 3000], [new, 1, new], group=group, seed=18)
    check(b.run(dtype), b.want(), d)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,ps,b,group,new", [
    (64, 16, 500, 1, 1), (128, 32, 500, 2, 1), (128, 16, 80, 4, 30),
    (64, 64, 80, 4, 30), (128, 64, 70, 7, 33)])
@pytest.mark.parametrize("share", SHARES[:2])
def test_more_short_sequences_than_waves(d, ps, b, group, new, dtype, share):
    """16 KV heads: a wave each for whole sequences, some of them empty."""
    rng = np.random.default_rng(b + new)
    c = cache_of(head_dim=d, page_size=ps, num_kv_heads=16, num_pages=3000,
                 max_pages=512 // ps, **share)
    lens = rng.integers(0, 90, b)
    lens[rng.integers(b, size=3)] = 300
    news = np.minimum(lens, rng.integers(1, new + 1, b) if new > 1 else 1)
    news[::3] = np.minimum(lens[::3], new)
    # What the rows are counted by on the host: padding makes them more.
    x = Batch(c, lens.tolist(), news.tolist(), group=group, seed=17,
              pad=b * new - int(news.sum()))
    rows = len(x.positions)
    x.positions[rng.integers(rows, size=9)] = -1
    x.positions[rng.integers(rows, size=9)] = 7
    x.table[5, 0] = -3
    x.table[6, 0] = 3000
    check(x.run(dtype), x.want(), d)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,share", [
    ([1400], [1350], SHARES[0]), ([1200, 700, 90], [1100, 600, 1], SHARES[0]),
    ([3900], [1300], SHARES[1]), ([30000, 300], [300, 280], SHARES[2])])
def test_prompts_of_more_tiles_than_workgroups(d, dtype, lens, new, share):
    """Whether sequences are cut is the kernel's choice, by lengths and rows; rows
    that see more or less than that supposes are as right."""
    c = cache_of(head_dim=d, page_size=64, num_kv_heads=16, num_pages=200,
                 max_pages=100, **share)
    b = Batch(c, lens, new, group=2, seed=20)
    heads = [1, 12, 31]
    o, lse = b.run(dtype)
    check((o[:, heads], lse[heads]), b.want(heads), d)
    rng = np.random.default_rng(20)
    b.positions = np.where(np.arange(len(b.positions)) % 3 == 0,
                           rng.integers(-1, max(lens), len(b.positions)),
                           max(lens) - 1)
    o, lse = b.run(dtype)
    check((o[:, heads], lse[heads]), b.want(heads), d)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,ps,group,long", [
    (64, 64, 4, [2048, 2049, 3900]), (128, 16, 4, [3000] * 5),
    (128, 64, 7, []), (64, 16, 5, [4096, 0, 4095])])
def test_short_and_long_sequences_of_many_tiles(d, ps, group, long, dtype):
    """Enough for all waves; those with more than 2048 keys are another launch's."""
    rng = np.random.default_rng(len(long))
    c = cache_of(head_dim=d, page_size=ps, num_kv_heads=16,
                 num_pages=30000 // ps, max_pages=4096 // ps)
    lens = rng.integers(0, 120, 80)
    lens[rng.permutation(80)[:len(long)]] = long
    new = np.minimum(lens, rng.integers(20, 31, 80))
    x = Batch(c, lens.tolist(), new.tolist(), group=group, seed=21,
              pad=80 * 30 - int(new.sum()))
    heads = [0, 16 * group // 2, 16 * group - 1]
    o, lse = x.run(dtype)
    check((o[:, heads], lse[heads]), x.want(heads), d)


def test_two_streams_at_once():
    """Calls that overlap, each with the binding's own workspace."""
    c = cache_of(head_dim=128, num_kv_heads=8, num_pages=700, max_pages=600)
    a = Batch(c, [8000, 2000], [40, 1], group=4, seed=22)
    b = Batch(c, [5, 9000], [5, 3], group=4, seed=23)
    want = a.run(), b.run()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for x, s in zip((a, b), streams):
            q = x.q.cuda()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(x.run(q=q, stream=s))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(got):
        assert torch.equal(o, want[i % 2][0])
        assert torch.equal(lse, want[i % 2][1])


def test_calls_back_to_back_on_two_streams():
    """Every buffer is there before the first call, so that the calls of one
    stream are in flight while the other's run, each with a workspace of the
    binding: the results are those of the calls alone."""
    c = cache_of(head_dim=128, num_kv_heads=8, page_size=64, num_pages=400,
                 max_pages=300)
    calls, want = [], []
    for seed, (lens, new) in enumerate((([15000, 2000], [300, 1]),
                                        ([5, 17000, 3000], [5, 150, 3]))):
        b = Batch(c, lens, new, group=4, seed=25 + seed)
        want.append(b.run())
        calls.append((b, [b.q.cuda()] + [i32(x) for x in (
            b.positions, b.cu, b.lens, b.table)] + [b.data]))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    rounds = 12
    out = [[(torch.full_like(o, 123.0), torch.full_like(lse, 123.0))
            for _ in range(rounds)] for o, lse in want]
    marks = [[[torch.cuda.Event(enable_timing=True) for _ in range(2)]
              for _ in range(rounds)] for _ in want]
    begin = torch.cuda.Event(enable_timing=True)
    begin.record()
    torch.cuda.synchronize()
    for i in range(rounds):
        for j, ((b, args), s) in enumerate(zip(calls, streams)):
            marks[j][i][0].record(s)
            ma.mesh_attn_cache_fwd(c, b.scale, *args, *out[j][i], stream=s)
            marks[j][i][1].record(s)
    torch.cuda.synchronize()
    for results, (o, lse) in zip(out, want):
        for x, y in results:
            assert torch.equal(x, o) and torch.equal(y, lse)
    # They did overlap: most calls begin before the other stream's call of the
    # same round ends, and end after it begins.
    at = [[[begin.elapsed_time(e) for e in pair] for pair in side]
          for side in marks]
    both = sum(a[0] < b[1] and b[0] < a[1] for a, b in zip(*at))
    assert both > rounds // 2, at


def test_a_captured_prompt_replays_with_other_lengths():
    """The same launches cut the sequences of one batch and leave another's whole."""
    c = cache_of(head_dim=128, num_kv_heads=16, page_size=64, num_pages=400,
                 max_pages=300)
    batches = [Batch(c, lens, new, group=2, seed=24) for lens, new in (
        ([1400, 600], [1350, 10]), ([16000, 1360], [600, 760]),
        ([1360, 0], [1360, 0]))]
    rows, d = 1360, 128
    q = torch.zeros(rows, 32, d, dtype=torch.bfloat16, device="cuda")
    positions, cu = torch.zeros(rows, **I32), torch.zeros(3, **I32)
    lens, table = torch.zeros(2, **I32), torch.zeros(2, 300, **I32)
    data = torch.zeros_like(batches[0].data)
    o = torch.zeros(rows, 32, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(32, rows, device="cuda")
    ws = torch.empty(ma.mesh_attn_cache_fwd_workspace_size(c, 32, 2, rows),
                     dtype=torch.uint8, device="cuda")

    def step():
        ma.mesh_attn_cache_fwd(c, d ** -0.5, q, positions, cu, lens, table,
                               data, o, lse, ws=ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    heads = [0, 17, 31]
    for b in batches + batches[:2]:
        q.copy_(b.q)
        for t, x in ((positions, b.positions), (cu, b.cu), (lens, b.lens),
                     (table, b.table)):
            t.copy_(i32(x))
        data.copy_(b.data)
        o.fill_(123.0)
        lse.fill_(123.0)
        graph.replay()
        torch.cuda.synchronize()
        check((o[:, heads], lse[heads]), b.want(heads), d)
        got = o.clone()
        step()
        assert torch.equal(o, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nan_in_a_short_sequence_of_many(dtype):
    """Only the heads of its KV head, and for V its 32 dims, become NaN."""
    c = cache_of(num_kv_heads=16, num_pages=1500, max_pages=32)
    b = Batch(c, [30] * 500, [1] * 500, group=2, seed=19)
    for request, head, what in ((3, 2, "k"), (9, 15, "v"), (499, 0, "k")):
        at = request * 30 + 5
        k, v = b.k[at:at + 1].cuda(), b.v[at:at + 1].cuda()
        (k if what == "k" else v)[0, head, 40] = float("nan")
        ma.mesh_attn_cache_append(c, k, v, i64(b.slots[at:at + 1]), b.data)
    o, lse = (x.isnan().cpu() for x in b.run(dtype))
    want = torch.zeros_like(o)
    want[3, 4:6] = want[9, 30:32, 32:] = want[499, :2] = True
    assert torch.equal(o, want)
    assert torch.equal(lse.T, want.all(-1))


@pytest.mark.parametrize("lens", [[2**31 - 1, 5], [192, 2**31 - 1]])
def test_lengths_past_the_table(lens):
    for share in SHARES:
        c = cache_of(num_pages=60, **share)
        b = Batch(c, lens, [2, 1], seed=14)
        check(b.run(), b.want(), 64)


def test_tables_for_a_billion_tokens():
    """max_pages at its limit: units of more keys, so that they can be counted."""
    c = cache_of(num_pages=300, page_size=256, max_pages=1 << 22)
    lens = [700, 0, 1, 5000] + [300 + i for i in range(76)]
    new = [1, 0, 1, 3] + [1] * 76
    small = Batch(cache_of(num_pages=300, page_size=256, max_pages=20), lens,
                  new, seed=15)
    want = small.want()
    table = torch.full((80, 1 << 22), -1, **I32)
    table[:, :20] = i32(small.table)
    o = torch.full((len(small.positions), 4, 64), 123.0, device="cuda")
    lse = torch.full((4, len(small.positions)), 123.0, device="cuda")
    ma.mesh_attn_cache_fwd(c, small.scale, small.q.cuda(),
                           i32(small.positions), i32(small.cu),
                           i32(small.lens), table, small.data, o, lse)
    check((o, lse), want, 64)


def test_more_rows_than_a_launch_has_workgroups_in_a_row():
    """2^26 rows and a few, sixteen to a workgroup: the last ones' grid."""
    c = cache_of(head_dim=128, num_kv_heads=1)
    rows, few = 2**26 + 21, 40
    k = torch.empty(rows, 1, 128, dtype=torch.bfloat16, device="cuda")
    slots = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    k[-few:] = torch.randn(few, 1, 128, dtype=torch.bfloat16, device="cuda")
    slots[-few:] = torch.arange(few, device="cuda") * 3
    data, want = random_bytes(c), random_bytes(c)
    ma.mesh_attn_cache_append(c, k, k, slots, data)
    ma.mesh_attn_cache_append(c, k[-few:], k[-few:], slots[-few:], want)
    assert torch.equal(data, want)
    v = torch.empty_like(k)
    ma.mesh_attn_cache_read(c, slots, data, k, v)
    wk, wv = torch.empty_like(k[-few:]), torch.empty_like(k[-few:])
    ma.mesh_attn_cache_read(c, slots[-few:], data, wk, wv)
    assert torch.equal(k[-few:], wk) and torch.equal(v[-few:], wv)
    assert not k[:-few].any() and not v[:-few].any()


def test_far_rows():
    """Q and O past 2^31 elements: the last rows, over a few keys."""
    c = cache_of(head_dim=128, num_kv_heads=1, page_size=64, num_pages=4)
    rows, hq = 140000, 128
    q = torch.zeros(rows, hq, 128, dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 2**31
    b = Batch(c, [40, 100], [1, 5], group=hq, seed=16)
    q[-6:] = b.q.cuda()
    cu = [0, rows - 5, rows]
    positions = np.full(rows, -1)
    positions[-6:] = b.positions
    o = torch.full((rows, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hq, rows), 7.0, device="cuda")
    ma.mesh_attn_cache_fwd(c, b.scale, q, i32(positions), i32(cu),
                           i32(b.lens), i32(b.table), b.data, o, lse)
    check((o[-6:], lse[:, -6:].contiguous()), b.want(), 128)
    assert not o[:-6].any() and torch.all(lse[:, :-6] == -float("inf"))


def test_fewer_bytes_of_workspace_are_refused():
    c = cache_of(num_pages=300, max_pages=256, page_size=64)
    need = ma.mesh_attn_cache_fwd_workspace_size(c, 4, 1, 1)
    assert 0 < need <= 35 << 20
    b = Batch(c, [5000], [1], seed=13)
    ws = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(ma.MeshAttnError, match="workspace"):
        b.run(ws=ws)
    # Whatever it held, and nothing behind it is written.
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    check(b.run(ws=ws[:need]), b.want(), 64)
    assert torch.all(ws[need:] == 0xFF)
    brief = cache_of(max_pages=32)
    assert ma.mesh_attn_cache_fwd_workspace_size(brief, 4, 1, 1) == 0


# -- together -----------------------------------------------------------------

ROPE = dict(head_dim=128, rotary_dim=128, num_axes=1,
            inv_freq=[10000.0 ** (-i / 64) for i in range(64)])


class Serving:
    """Buffers of a decode loop over one GPU's share of a cache."""

    def __init__(self, share, requests, rows, hkv=2, group=4):
        self.c = ma.Cache.make(cache_of(num_pages=64, page_size=16,
                                        num_kv_heads=hkv, head_dim=128,
                                        max_pages=16, **share))
        self.b, self.hkv, self.hq = requests, hkv, hkv * group
        self.data = torch.zeros(64, hkv, 16 * 136, dtype=torch.uint8,
                                device="cuda")
        self.free = torch.randperm(64).int().cuda()
        self.table = torch.full((requests, 16), -1, **I32)
        self.range = [i32([0, 64]), torch.empty(2, **I32)]
        self.lens = [torch.zeros(requests, **I32),
                     torch.empty(requests, **I32)]
        self.cu = torch.empty(requests + 1, **I32)
        self.refused = torch.empty(1, **I32)
        self.resize(rows)

    def resize(self, rows):
        self.slots = torch.empty(rows, dtype=torch.int64, device="cuda")
        self.pos = torch.empty(rows, **I32)
        self.qr = torch.empty(rows, self.hq, 128, dtype=torch.bfloat16,
                              device="cuda")
        self.kr = torch.empty(rows, self.hkv, 128, dtype=torch.bfloat16,
                              device="cuda")
        self.o = torch.empty(rows, self.hq, 128, device="cuda")
        self.lse = torch.empty(self.hq, rows, device="cuda")
        self.ws = torch.empty(max(16, ma.mesh_attn_cache_fwd_workspace_size(
            self.c, self.hq, self.b, rows)), dtype=torch.uint8, device="cuda")

    def step(self, new, q, k, v):
        ma.mesh_attn_cache_tables(
            self.c, self.lens[0], new, self.free, self.range[0], self.table,
            self.lens[1], self.cu, self.slots, self.pos, self.range[1],
            self.refused)
        self.lens[0].copy_(self.lens[1])
        self.range[0].copy_(self.range[1])
        ma.mesh_attn_rope(ROPE, self.pos, q, self.qr, k, self.kr)
        ma.mesh_attn_cache_append(self.c, self.kr, v, self.slots, self.data)
        ma.mesh_attn_cache_fwd(self.c, 128 ** -0.5, self.qr, self.pos, self.cu,
                               self.lens[0], self.table, self.data, self.o,
                               self.lse, ws=self.ws)


def projections(rows, hq, hkv, seed):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(rows, h, 128, generator=gen).to(torch.bfloat16).cuda()
            for h in (hq, hkv, hkv)]


def test_a_prompt_and_steps_on_two_gpus_merge_to_the_whole():
    """Two shares of the sequences, prompt and decode steps, merged by
    mesh_attn_lse_merge: the attention of a cache that stores everything; and
    the stored prompt read back is the tile kernels' KV buffer."""
    whole = Serving({}, 3, 0)
    parts = [Serving(dict(num_partitions=2, partition=p), 3, 0)
             for p in (0, 1)]
    for step, new in enumerate(([64, 33, 0], [1, 1, 90], [1, 1, 1],
                                [1, 0, 1])):
        rows = sum(new)
        q, k, v = projections(rows, 8, 2, step)
        for s in [whole] + parts:
            s.resize(rows)
            s.step(i32(new), q, k, v)
            assert s.refused.item() == 0
        o = torch.empty_like(whole.o)
        lse = torch.empty_like(whole.lse)
        ma.mesh_attn_lse_merge(torch.stack([s.o for s in parts]),
                               torch.stack([s.lse for s in parts]), o, lse)
        # float32 partials of the same products: 2^-14 of the values' size.
        assert (o - whole.o).abs().max() <= 2.0**-14 * 8
        assert (lse - whole.lse).abs().max() <= 2.0**-14
    assert whole.lens[0].tolist() == [67, 35, 92]
    # Request 0's first 64 tokens as a KV partition of the tile forward.
    at = torch.arange(64, device="cuda")
    slots = whole.table[0, at // 16].long() * 16 + at % 16
    k, v = torch.empty(2, 256, 2, 128, dtype=torch.bfloat16, device="cuda")
    all_slots = torch.full((256,), -1, dtype=torch.int64, device="cuda")
    all_slots[:64] = slots
    ma.mesh_attn_cache_read(whole.c, all_slots, whole.data, k, v)
    assert not k[64:].any() and not v[64:].any() and k[:64].any()
    q, _, _ = projections(256, 8, 2, 50)
    prob = dict(num_partitions=2, partition_len=256, num_q_heads=8,
                num_kv_heads=2, head_dim=128, causal=0,
                softmax_scale=128 ** -0.5)
    # Both sides see the 192 zero rows too.
    full = cache_of(num_pages=4, page_size=64, num_kv_heads=2, head_dim=128,
                    max_pages=4)
    data = torch.zeros(4, 2, 64 * 136, dtype=torch.uint8, device="cuda")
    ma.mesh_attn_cache_append(full, k, v, torch.arange(256, device="cuda"),
                              data)
    o, o2 = torch.empty(2, 256, 8, 128, device="cuda")
    lse, lse2 = torch.empty(2, 8, 256, device="cuda")
    ma.mesh_attn_tile_fwd(prob, [0], [1], q, k, v, o, lse)
    ma.mesh_attn_cache_fwd(full, 128 ** -0.5, q, i32([255] * 256),
                           i32([0, 256]), i32([256]), i32([[0, 1, 2, 3]]),
                           data, o2, lse2)
    assert (lse - lse2).abs().max() <= 2.0**-14
    assert (o - o2).abs().max() <= 2.0**-8 * v.float().abs().max()


def test_captured_steps_replay():
    """A decode step captured once serves every later step: lengths, tables and
    pages advance on the device between replays, beside eager work."""
    def build():
        torch.manual_seed(1)
        s = Serving({}, 3, 96)
        q, k, v = projections(96, 8, 2, 0)
        s.step(i32([50, 20, 26]), q, k, v)
        s.resize(3)
        return s

    steps = [projections(3, 8, 2, 100 + i) for i in range(6)]
    eager, outs = build(), []
    ones = i32([1, 1, 1])
    for q, k, v in steps:
        eager.step(ones, q, k, v)
        outs.append((eager.o.clone(), eager.lse.clone(), eager.table.clone()))
    s = build()
    q, k, v = (torch.empty_like(x) for x in steps[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step(ones, q, k, v)
    for i, step in enumerate(steps):
        for dst, src in zip((q, k, v), step):
            dst.copy_(src)
        graph.replay()
        # Eager work of the program between the replays.
        other = torch.randn(512, 512, device="cuda")
        (other @ other).sum().item()
        assert torch.equal(s.o, outs[i][0]) and torch.equal(s.lse, outs[i][1])
        assert torch.equal(s.table, outs[i][2])
