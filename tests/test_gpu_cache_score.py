"""Attention over the 4-bit cache under a score rule, and rotation and append in
one call, on the GPU: against the float64 oracle, and the whole step as it is
used."""

import numpy as np
import pytest
import torch

import paper_2512_20968_amd as ma
from oracle import cache as oc
from oracle import score as os_

from helpers import exact_angle
from score_helpers import on_gpu
from test_gpu_cache import Batch, append_inputs, cache_of, i32, i64, \
    random_bytes

pytestmark = pytest.mark.gpu


class Scored(Batch):
    """A batch under a rule (NumPy arrays)."""

    def __init__(self, c, lens, new, rule, **kw):
        super().__init__(c, lens, new, **kw)
        self.rule = rule(self) if callable(rule) else rule

    def run(self, dtype=torch.float32, q=None, ws=None, stream=None, rule=None):
        rows = self.q.shape[0]
        o = torch.full((rows, self.hq, self.c["head_dim"]), 123.0,
                       dtype=dtype, device="cuda")
        lse = torch.full((self.hq, rows), 123.0, device="cuda")
        return ma.mesh_attn_cache_score_fwd(
            self.c, self.scale, on_gpu(self.rule) if rule is None else rule,
            self.q.cuda() if q is None else q, i32(self.positions),
            i32(self.cu), i32(self.lens), i32(self.table), self.data, o, lse,
            ws=ws, stream=stream)

    def check(self, got):
        """Scores are off by the float32 products (2^-23 each of d + 16), the
        cap's tanh (2^-21 of the cap) and the bias relative to the nearest key
        (2^-21 of what can weigh, which is below 2^6); weights by twice that,
        2^-14 for exponentials and sums, 2^-8 for a bf16 O's weights and 2^-8
        for itself."""
        c = self.c
        o, lse = (x.double().cpu().numpy() for x in got)
        rows, hq, d = self.q.shape
        q = self.q.double().numpy()
        group = hq // c["num_kv_heads"]
        live = np.zeros(rows, bool)
        for b in range(len(self.lens)):
            a = min(max(int(self.cu[b]), 0), rows)
            e = min(max(int(self.cu[b + 1]), a), rows)
            if a == e:
                continue
            live[a:e] = True
            n = min(oc.stored(c, max(int(self.lens[b]), 0)),
                    c["max_pages"] * c["page_size"])
            r = np.arange(n)
            page = self.table[b, r // c["page_size"]]
            ok = (page >= 0) & (page < c["num_pages"])
            slots = np.where(ok, page * c["page_size"] + r % c["page_size"],
                             -1)
            k = torch.empty(n, c["num_kv_heads"], d, dtype=torch.bfloat16,
                            device="cuda")
            v = torch.empty_like(k)
            ma.mesh_attn_cache_read(c, i64(slots), self.data, k, v)
            k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
            kpos = np.where(ok, oc.key_positions(c, n), -1)
            sub = {x: y if x in ("cap", "slopes") else y[a:e]
                   for x, y in self.rule.items()}
            if "key_begin" in sub:
                sub["key_begin"] = np.maximum(sub["key_begin"], 0)
            elif n:
                sub["key_begin"] = np.zeros(e - a, np.int64)
            qpos = self.positions[a:e]
            args = (self.scale, sub, q[a:e], qpos, kpos)
            wo, wl = os_.cached(*args, k, v, int(self.lens[b]))
            mass, _ = os_.cached(*args, k, np.abs(v), int(self.lens[b]))
            fine = np.isfinite(k).all(-1)
            reach = self.scale * np.stack([
                np.abs(q[a:e, h]) @ np.abs(np.where(
                    fine[:, [h // group]], k[:, h // group], 0)).T
                for h in range(hq)]).max(-1, initial=0)
            err = ((d + 16) * 2.0 ** -23 * reach + 2.0 ** -14
                   + self.rule.get("cap", 0.0) * 2.0 ** -21)
            if "slopes" in self.rule:
                err += 2.0 ** -14
            go, gl = o[a:e], lse[:, a:e]
            none, nan = np.isneginf(wl), np.isnan(wl)
            np.testing.assert_array_equal(np.isneginf(gl), none)
            np.testing.assert_array_equal(np.isnan(gl), nan)
            assert (go.transpose(1, 0, 2)[none] == 0).all()
            off = np.abs(gl - wl) - err - 2.0 ** -22 * np.abs(wl)
            assert (off[~none & ~nan] <= 0).all(), off[~none & ~nan].max()
            bad = np.isnan(wo)
            np.testing.assert_array_equal(np.isnan(go), bad)
            tol = 2 * mass * err.T[:, :, None]
            if got[0].dtype is torch.bfloat16:
                tol += 2.0 ** -8 * (mass + np.abs(wo))
            off = np.where(bad, -1, np.abs(go - wo) - tol)
            assert off.max() <= 1e-30, off.max()
        assert (o[~live] == 123.0).all() and (lse[:, ~live] == 123.0).all()


def rule_of(kind, cap, slopes, seed=0):
    def make(b):
        rng = np.random.default_rng(seed)
        pos, rows = b.positions, len(b.positions)
        out = {}
        if cap:
            out["cap"] = cap
        if slopes:
            out["slopes"] = (2.0 ** -rng.uniform(0, 6, b.hq)).astype(
                np.float32)
        if kind == "window":
            out["key_begin"] = np.maximum(pos - 40 + 1, 0)
        elif kind == "prefix":
            out["key_end"] = np.maximum(pos + 1, 25)
        elif kind == "any":
            # A request's first row has the least begin of its rows.
            begin = rng.integers(-9, 60, rows)
            for a in b.cu[:-1]:
                if a < rows:
                    begin[a] = 3
            out["key_begin"] = begin
            out["key_end"] = begin + rng.integers(-3, 90, rows)
        elif kind == "none":
            out["key_begin"] = np.full(rows, 11)
            out["key_end"] = np.full(rows, 11)
        elif kind == "late":
            out["key_begin"] = np.full(rows, 5000)
        return out
    return make


RULES = [("plain", 0.0, False), ("plain", 4.0, False), ("window", 0.0, False),
         ("window", 5.0, True), ("prefix", 3.0, True), ("any", 0.0, True),
         ("any", 6.0, False), ("none", 2.0, True), ("late", 2.0, False)]


@pytest.mark.parametrize("kind,cap,slopes", RULES)
@pytest.mark.parametrize("d,ps,group,new,dtype", [
    (64, 16, 2, 1, torch.float32), (128, 64, 4, 1, torch.bfloat16),
    (128, 16, 5, 7, torch.float32), (64, 32, 3, 20, torch.bfloat16)])
def test_rules(kind, cap, slopes, d, ps, group, new, dtype):
    """Lengths around every border, one token or a chunk each."""
    lens = [1, 15, 16, 17, 31, 33, 63, 65, 96, 127, 128, 129, 160, 190]
    lens = [max(n, new) for n in lens]
    c = cache_of(head_dim=d, page_size=ps, num_pages=14 * 12, max_pages=12)
    b = Scored(c, lens, [new] * len(lens), rule_of(kind, cap, slopes),
               group=group, pad=3)
    b.check(b.run(dtype))


@pytest.mark.parametrize("share", [
    dict(num_partitions=3, partition=1),
    dict(layout=0, num_partitions=4, partition=1, partition_len=40),
    dict(num_partitions=200, partition=199)])
@pytest.mark.parametrize("kind,cap,slopes", [("window", 4.0, True),
                                             ("any", 0.0, True),
                                             ("plain", 5.0, False)])
def test_shares_of_a_mesh(share, kind, cap, slopes):
    c = cache_of(num_pages=100, **share)
    b = Scored(c, [1, 40, 41, 100, 160, 170], [1, 2, 1, 5, 1, 9],
               rule_of(kind, cap, slopes))
    b.check(b.run())
    b.check(b.run(torch.bfloat16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,group", [(1, 4), (60, 2)])
def test_long_tables_are_cut(d, new, group):
    """Long sequences are cut over workgroups and joined; windows of them read
    what they hold; equal calls give equal bits."""
    c = cache_of(head_dim=d, num_kv_heads=1, page_size=64, num_pages=400,
                 max_pages=130)
    lens = [8000, 61, 4097, 64]
    for kind, cap in (("window", 5.0), ("any", 3.0), ("plain", 0.0)):
        b = Scored(c, lens, [new] * 4, rule_of(kind, cap, True), group=group)
        got = b.run()
        b.check(got)
        again = b.run()
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("d,new,group,dtype", [
    (64, 1, 2, torch.float32), (128, 1, 4, torch.bfloat16),
    (64, 20, 3, torch.bfloat16), (128, 6, 4, torch.float32)])
@pytest.mark.parametrize("kind,cap,slopes", [("window", 4.0, True),
                                             ("any", 0.0, True)])
def test_more_short_sequences_than_waves(d, new, group, dtype, kind, cap,
                                         slopes):
    """Short tables and many requests: a wave for every sequence."""
    b, rng = 500, np.random.default_rng(d)
    c = cache_of(head_dim=d, num_kv_heads=9, num_pages=b * 8, max_pages=8)
    lens = np.maximum(rng.integers(1, 128, b), new)
    s = Scored(c, lens.tolist(), [new] * b, rule_of(kind, cap, slopes),
               group=group)
    got = s.run(dtype)
    # The oracle on a few of them.
    some = [0, 1, 250, 498, 499]
    rows = np.concatenate([np.arange(s.cu[i], s.cu[i + 1]) for i in some])
    part = Scored.__new__(Scored)
    part.c, part.hq, part.scale, part.data = c, s.hq, s.scale, s.data
    part.q, part.positions = s.q[rows], s.positions[rows]
    part.cu = np.arange(len(some) + 1) * new
    part.lens, part.table = s.lens[some], s.table[some]
    part.rule = {k: x if k in ("cap", "slopes") else x[rows]
                 for k, x in s.rule.items()}
    at = torch.tensor(rows).cuda()
    part.check((got[0][at], got[1][:, at]))


def test_no_rule_is_the_call_without():
    c = cache_of(num_pages=100)
    b = Scored(c, [5, 100, 190], [1, 9, 2], {})
    got = b.run(rule=False)  # no rule at all
    b.check(got)
    b.check(Batch.run(b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_bad_pages_and_nan(dtype):
    """Pages out of range hide their keys; NaN keys and values reach the rows
    whose range holds them and no other."""
    c = cache_of(num_pages=60)
    b = Scored(c, [100, 120, 90], [20, 3, 1], rule_of("window", 4.0, True))
    b.table[0, 4], b.table[1, 6] = -1, 60
    k, v = b.k.clone(), b.v.clone()
    k[88, 1, 3] = float("nan")        # request 0's token 88
    v[83, 0, 40] = float("inf")       # .. 83
    v[100 + 50, 1, 0] = float("nan")  # request 1's token 50: before its window
    slots = b.slots
    ma.mesh_attn_cache_append(c, k.cuda(), v.cuda(), i64(slots), b.data)
    b.check(b.run(dtype))


def test_a_steep_bias_over_a_bad_last_page():
    """The nearest keys of a request are hidden by their page: the bias of the
    others is beyond float32's smallest weight."""
    c = cache_of(num_pages=60)
    for cap in (0.0, 4.0):
        rule = {"cap": cap, "slopes": np.float32([60.0, 90.0, 0.5, 20.0])}
        b = Scored(c, [100, 96 + 16], [1, 30], rule)
        b.table[0, 6], b.table[1, 6] = -1, 60
        o, lse = b.run()
        assert torch.isfinite(lse).all()
        for r in (0, 30):  # heads 0 and 1 pick the last key with a page
            k, v = (torch.empty(1, 2, 64, dtype=torch.bfloat16, device="cuda")
                    for _ in range(2))
            s = b.table[int(r > 0), 5] * 16 + 15
            ma.mesh_attn_cache_read(c, i64([s]), b.data, k, v)
            assert (o[r, :2] - v[0, 0].float()).abs().max() <= 2.0 ** -14 * 6


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cap", [30.0, 48.0, 50.0, 55.0])
def test_a_gentle_bias_under_scores_at_the_low_end_of_the_cap(cap, dtype):
    """Every score is -cap: the weights of a thousand keys with a bias of one to
    eleven units count, however far the reference lies from them."""
    c, n = cache_of(num_pages=300, max_pages=128), 2000
    rule = {"cap": cap, "slopes": np.float32([0.005, 0.01, 0.002, 0.0])}
    b = Scored(c, [n], [3], rule)
    r = np.arange(n)
    slots = b.table[0, r // 16] * 16 + r % 16
    k = torch.ones(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(n, 2, 64, device="cuda",
                    generator=torch.Generator("cuda").manual_seed(4))
    ma.mesh_attn_cache_append(c, k, v.bfloat16(), i64(slots), b.data)
    b.q = torch.full_like(b.q, -50.0)
    b.check(b.run(dtype))


def test_keys_before_the_first_rows_begin_are_not_seen():
    c = cache_of(num_pages=60)
    b = Scored(c, [150], [4], {"key_begin": np.array([70, 10, 90, 0])})
    b.check(b.run())


def test_far_positions_keep_the_digits_of_their_bias():
    """A share whose keys are half a million positions before the rows."""
    P = 128
    c = cache_of(layout=0, num_partitions=4100, partition=2, partition_len=P,
                 num_pages=20)
    b = Scored(c, [P * 4099], [3], {"slopes": np.float32([0.5, 0.1, 2.0, 0.01]),
                                    "cap": 9.0})
    wide = b.run()
    # LSE holds half a million times the slope: compare what O is, which does not.
    o = wide[0].double().cpu().numpy()
    n = P
    r = np.arange(n)
    slots = b.table[0, r // 16] * 16 + r % 16
    k = torch.empty(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    ma.mesh_attn_cache_read(c, i64(slots), b.data, k, v)
    want, _ = os_.cached(b.scale, b.rule, b.q.double().numpy(), b.positions,
                         oc.key_positions(c, n), k.double().cpu().numpy(),
                         v.double().cpu().numpy(), P * 4099)
    assert np.abs(o - want).max() <= 2.0 ** -13 * np.abs(
        v.float().cpu().numpy()).max()


def test_slices_streams_and_workspaces():
    c = cache_of(num_pages=400, page_size=16, max_pages=200)
    b = Scored(c, [3000, 200, 77], [1, 5, 1], rule_of("window", 5.0, True))
    o, lse = b.run()
    rows = b.q.shape[0]
    wide = torch.full((rows, b.hq + 3, 64), float("nan"), dtype=torch.bfloat16,
                      device="cuda")
    wide[:, 1:1 + b.hq] = b.q.cuda()
    n = ma.mesh_attn_cache_score_fwd_workspace_size(c, b.hq, 3, rows)
    assert n > 0
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for w in (ws[:n], None):
        with torch.cuda.stream(side):
            o2, lse2 = b.run(q=wide[:, 1:1 + b.hq], ws=w)
        side.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert (ws[n:] == 255).all()


# -- rotation and append ------------------------------------------------------

def rope_of(d, rot, axes, inter, base=10000.0):
    n = rot // 2
    return dict(head_dim=d, rotary_dim=rot, num_axes=axes, interleaved=inter,
                inv_freq=[base ** (-i / n) for i in range(n)],
                axis=[i * axes // n for i in range(n)])


def undecided(y):
    """Groups (bool [.., d / 32]) with an element so near the border of two
    stored values, or a largest one so near that of two scales, that 2^-45 of
    their size decides: the oracle's own float64 angles are no better."""
    g = y.reshape(y.shape[:-1] + (-1, 32))
    top = np.abs(g).max(-1, keepdims=True)
    _, e = np.frexp(np.where(top == 0, 1, top))
    near = np.abs(top / 2.0 ** e - 0.875) < 2.0 ** -45 + 0 * g
    unit = 2.0 ** (e - 3 + (top / 2.0 ** e > 0.875))
    x = np.abs(g) / unit
    for mid in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
        near |= np.abs(x - mid) < 2.0 ** -42
    return near.any(-1)


@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("d,rot,axes,ps,hq,hkv,rows", [
    (64, 64, 1, 16, 4, 2, 1), (128, 128, 3, 64, 4, 1, 37),
    (128, 64, 2, 16, 3, 3, 50), (64, 16, 1, 256, 2, 2, 129),
    (128, 16, 1, 32, 8, 2, 33)])
def test_append_is_the_oracle_byte_for_byte(inter, d, rot, axes, ps, hq, hkv,
                                            rows):
    """The stored K is the nearest to the rotation in float64; Q is
    mesh_attn_rope's and V mesh_attn_cache_append's, bit for bit."""
    c = cache_of(head_dim=d, num_kv_heads=hkv, page_size=ps, num_pages=9)
    r = rope_of(d, rot, axes, inter)
    rng = np.random.default_rng(rows)
    slots = rng.permutation(9 * ps)[:rows]
    if rows > 5:
        slots[2], slots[3], slots[4] = -1, 9 * ps, 2**40
    x = torch.tensor(rng.standard_normal((rows, hq + 2 * hkv, d))).to(
        torch.bfloat16).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    pos = rng.integers(-2000, 10**6, (axes, rows))
    pos[:, 0] = 0
    data = random_bytes(c)
    want = data.cpu().numpy().copy()
    out = torch.full((rows, hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    before = x.clone()
    ma.mesh_attn_cache_rope_append(c, r, i32(pos), q, out, k, v, i64(slots),
                                   data)
    assert torch.equal(x, before)
    qr, kr = torch.empty_like(out), torch.empty_like(k)
    ma.mesh_attn_rope(r, i32(pos), q, qr, k, kr)
    assert torch.equal(out, qr)
    y = oc.rope(k.double().cpu().numpy(), pos, r["inv_freq"], r["axis"], rot,
                inter)
    oc.write_rows(c, want, y, v.double().cpu().numpy(), slots)
    got = data.cpu().numpy()
    if not undecided(y).any():
        np.testing.assert_array_equal(got, want)
    else:  # as values, without the undecided groups
        for i, s in enumerate(slots):
            a, b = oc.read_row(c, got, s), oc.read_row(c, want, s)
            np.testing.assert_array_equal(a[1], b[1])
            keep = ~undecided(y[i]).repeat(32, -1)
            np.testing.assert_array_equal(a[0][keep], b[0][keep])
    # In place, within the fused rows.
    data2 = random_bytes(c)
    ma.mesh_attn_cache_rope_append(c, r, i32(pos), q, q, k, v, i64(slots),
                                   data2)
    assert torch.equal(q, qr) and torch.equal(data, data2)
    assert torch.equal(x[:, hq:], before[:, hq:])


def test_append_without_a_turn_is_append():
    """Frequencies of 0, and dims behind the rotated ones: every kind of group
    (ties, infinities, NaN, subnormals) as mesh_attn_cache_append stores it."""
    c = cache_of(head_dim=128, num_kv_heads=2, page_size=16, num_pages=9)
    r = dict(head_dim=128, rotary_dim=64, num_axes=1, interleaved=0,
             inv_freq=[0.0] * 32)
    k, v = (append_inputs(128, 2, 130, s).cuda() for s in (4, 9))
    q = append_inputs(128, 2, 130, 5).cuda()
    slots = i64(np.random.default_rng(1).permutation(144)[:130])
    a, b = random_bytes(c), random_bytes(c)
    ma.mesh_attn_cache_append(c, k, v, slots, a)
    out = torch.empty_like(q)
    ma.mesh_attn_cache_rope_append(c, r, i32(np.arange(130)), q, out, k, v,
                                   slots, b)
    # 0 times an infinity or a NaN of a pair is NaN in both of its dims.
    bad = ~np.isfinite(k.double().cpu().numpy()).reshape(130, 2, 4, 32).all(-1)
    bad[:, :, :2] |= bad[:, :, 1::-1]
    a, b = a.cpu().numpy(), b.cpu().numpy()
    for i, s in enumerate(slots.tolist()):
        x, y = oc.read_row(c, a, s), oc.read_row(c, b, s)
        np.testing.assert_array_equal(x[1], y[1])
        keep = ~bad[i].repeat(32, -1)
        np.testing.assert_array_equal(x[0][keep], y[0][keep])
        assert np.isnan(y[0][~keep]).all()


def test_append_at_the_ends_of_32_bits():
    """Positions up to 2^31 - 1 and -2^31 and quick frequencies: angles off by
    2^-34 of a turn at most."""
    c = cache_of(head_dim=64, num_kv_heads=1, page_size=16, num_pages=2)
    freq = [1.0, -1.0, 3.5, 1e-3, 500.0, 0.25, 1e-9, 2.0] * 4
    r = dict(head_dim=64, rotary_dim=64, num_axes=1, interleaved=0,
             inv_freq=freq)
    pos = np.array([0, 1, 7, 2**31 - 1, -2**31, -1, 2**30 + 1, 123456789])
    rng = np.random.default_rng(2)
    k = torch.tensor(rng.standard_normal((8, 1, 64))).to(torch.bfloat16).cuda()
    data = random_bytes(c)
    q, out = k.clone(), torch.empty_like(k)
    ma.mesh_attn_cache_rope_append(c, r, i32(pos), q, out, k, k,
                                   i64(np.arange(8)), data)
    x = k.double().cpu().numpy()
    y = x.copy()
    for i in range(32):
        for j, p in enumerate(pos):
            phi = exact_angle(freq[i], int(p))
            s, co = np.sin(phi), np.cos(phi)
            y[j, 0, i] = x[j, 0, i] * co - x[j, 0, i + 32] * s
            y[j, 0, i + 32] = x[j, 0, i + 32] * co + x[j, 0, i] * s
    got = data.cpu().numpy()
    for j in range(8):
        vals = oc.read_row(c, got, j)[0][0].reshape(2, 32)
        for g, w in zip(vals, y[j, 0].reshape(2, 32)):
            code, e = oc.quantize_group(w)
            near = oc.values(code, np.array([e], np.uint8))
            # A value next to a border may go either way: within half a step
            # and 2^-30 of the pair's size.
            unit = 2.0 ** (float(e) - 127)
            a = np.abs(w) / unit
            step = np.where(a < 2, 0.5, np.where(a < 4, 1, 2)) * unit
            assert (np.abs(g - w) <= np.maximum(
                np.abs(near - w), step / 2) + 2.0 ** -28).all()


# -- the whole step -----------------------------------------------------------

def test_prompt_and_steps_under_a_rule():
    """Tables, rotation with append, attention under a window with a cap, for a
    prompt in two chunks and single tokens, captured and replayed; every step
    against the oracle on what the cache holds."""
    d, hq, hkv = 128, 4, 2
    c = cache_of(head_dim=d, num_kv_heads=hkv, num_pages=40, max_pages=12)
    r = rope_of(d, d, 1, 0)
    rng = np.random.default_rng(4)
    table = torch.full((2, 12), -1, dtype=torch.int32, device="cuda")
    lens = [i32([0, 0]), i32([0, 0])]
    free_range = [i32([0, 40]), i32([0, 40])]
    free = i32(rng.permutation(40))
    cu, refused = i32([0, 0, 0]), i32([0])
    data = random_bytes(c)
    window = 50

    def step(new, rows, bufs):
        q, k, v, pos, slots, begin, o, lse, ws = bufs
        ma.mesh_attn_cache_tables(c, lens[0], new, free, free_range[0], table,
                                  lens[1], cu, slots, pos, free_range[1],
                                  refused)
        torch.sub(pos, window - 1, out=begin)
        begin.clamp_(min=0)
        ma.mesh_attn_cache_rope_append(c, r, pos, q, q, k, v, slots, data)
        ma.mesh_attn_cache_score_fwd(c, d ** -0.5, dict(cap=7.0,
                                                        key_begin=begin), q,
                                     pos, cu, lens[1], table, data, o, lse,
                                     ws=ws)
        lens[0].copy_(lens[1])
        free_range[0].copy_(free_range[1])

    def buffers(rows):
        x = torch.tensor(rng.standard_normal((rows, hq + 2 * hkv, d))).to(
            torch.bfloat16).cuda()
        n = ma.mesh_attn_cache_score_fwd_workspace_size(c, hq, 2, rows)
        i = dict(dtype=torch.int32, device="cuda")
        return (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:],
                torch.empty(rows, **i),
                torch.empty(rows, dtype=torch.int64, device="cuda"),
                torch.empty(rows, **i),
                torch.empty(rows, hq, d, device="cuda"),
                torch.empty(hq, rows, device="cuda"),
                torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))

    def check(bufs):
        b = Scored.__new__(Scored)
        b.c, b.hq, b.scale = c, hq, d ** -0.5
        b.q = bufs[0].cpu()
        b.positions = bufs[3].cpu().numpy()
        b.cu, b.lens = cu.cpu().numpy(), lens[1].cpu().numpy()
        b.table, b.data = table.cpu().numpy(), data
        b.rule = {"cap": 7.0, "key_begin": bufs[5].cpu().numpy()}
        b.check((bufs[6], bufs[7]))

    for new in ([70, 33], [40, 1]):
        bufs = buffers(sum(new))
        step(i32(new), sum(new), bufs)
        check(bufs)
    bufs, ones = buffers(2), i32([1, 1])
    step(ones, 2, bufs)
    check(bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ones, 2, bufs)
    for _ in range(20):  # past a page's end
        bufs[0].copy_(torch.randn(2, hq, d).to(torch.bfloat16))
        bufs[1].copy_(torch.randn(2, hkv, d).to(torch.bfloat16))
        graph.replay()
        other = torch.randn(256, 256, device="cuda")
        (other @ other).sum().item()
        check(bufs)
    assert lens[0].tolist() == [70 + 40 + 21, 33 + 1 + 21]
    assert refused.item() == 0


def test_the_cache_holds_what_the_tile_sees():
    """A prompt attended by the tile call on the values read back is the cache
    call's result, under one rule."""
    d = 64
    c = cache_of(head_dim=d, num_pages=20)
    rows = 190
    b = Scored(c, [rows], [rows], rule_of("window", 5.0, True), group=2)
    k = torch.empty(rows, 2, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    ma.mesh_attn_cache_read(c, i64(b.slots), b.data, k, v)
    o, lse = b.run()
    prob = dict(num_partitions=1, partition_len=rows, num_q_heads=4,
                num_kv_heads=2, head_dim=d, causal=1, softmax_scale=b.scale)
    to, tl = torch.empty_like(o), torch.empty_like(lse)
    ma.mesh_attn_score_fwd(prob, [0], [0], on_gpu(b.rule), b.q.cuda(), k, v,
                           to, tl)
    b.check((o, lse))
    b.check((to, tl))
