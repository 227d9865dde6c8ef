"""Pins of the cache oracle: brute force, round trips, the tile oracle on the
stored values, closed forms of the rotation."""

import numpy as np
import pytest

import oracle
from oracle import cache as oc

from helpers import ExactScores


def _cache(**kw):
    c = dict(num_pages=6, page_size=16, num_kv_heads=2, head_dim=64,
             max_pages=3, layout=1, num_partitions=1, partition=0,
             partition_len=0)
    c.update(kw)
    return c


def test_values_are_the_sixteen_e2m1_numbers():
    want = []
    for code in range(16):
        s, e, m = code >> 3, (code >> 1) & 3, code & 1
        mag = m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        want.append(-mag if s else mag)
    got = oc.values(np.arange(16, dtype=np.uint8).repeat(2),
                    np.array([127], dtype=np.uint8))
    np.testing.assert_array_equal(got, np.repeat(want, 2))


@pytest.mark.parametrize("scale", [1e-30, 0.37, 1.0, 1e30])
def test_quantization_is_off_by_at_most_half_a_step(scale):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((50, 32)) * scale
    codes, scales = oc.quantize(x)
    got = oc.values(codes, scales)
    unit = 2.0 ** (scales.astype(float) - 127)
    y = np.abs(x) / unit
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    assert np.all(np.abs(got - x) <= step / 2 * unit)
    assert np.all(y.max(-1, keepdims=True) > 3.5)  # no smaller scale fits
    assert np.all(y <= 7)


def test_quantization_limits():
    x = np.zeros((6, 32))
    x[1, 3] = 2.0**-133
    x[2, 0] = np.inf
    x[3, 31] = np.nan
    x[4, 7] = 1.99 * 2.0**127
    x[5] = 7.0
    codes, scales = oc.quantize(x)
    assert scales[:, 0].tolist() == [1, 1, 255, 255, 252, 127]
    got = oc.values(codes, scales)
    assert np.all(got[:2] == 0) and np.all(np.isnan(got[2:4]))
    assert got[4, 7] == 6 * 2.0**125 and np.all(got[5] == 6)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [16, 64])
def test_layout_covers_a_block_once(d, ps):
    c = _cache(head_dim=d, page_size=ps)
    codes, scales = set(), set()
    for t in range(ps):
        for i in range(d):
            ka, va, ks, vs = oc.block_offsets(c, t, i)
            codes |= {(ka, i % 2), (va, i % 2)}
            scales |= {(ks, "k", t, i // 32), (vs, "v", t, i // 32)}
    assert len(codes) == 2 * ps * d
    assert {a for a, _ in codes} == set(range(ps * d))
    assert sorted(s[0] for s in scales) == list(range(ps * d,
                                                      oc.page_bytes(c)))


def test_write_and_read():
    rng = np.random.default_rng(6)
    c = _cache()
    data = rng.integers(0, 256, (6, 2, oc.page_bytes(c)), dtype=np.uint8)
    was = data.copy()
    k, v = rng.standard_normal((2, 5, 2, 64))
    slots = [17, 95, -1, 96, 0]
    oc.write_rows(c, data, k, v, slots)
    for r, s in enumerate(slots):
        gk, gv = oc.read_row(c, data, s)
        if 0 <= s < 96:
            np.testing.assert_array_equal(gk, oc.values(*oc.quantize(k[r])))
            np.testing.assert_array_equal(gv, oc.values(*oc.quantize(v[r])))
        else:
            assert not gk.any() and not gv.any()
    # A row is d + d/16 bytes of K and V a head; nothing else changed.
    touched = np.ones_like(data, dtype=bool)
    for s in (17, 95, 0):
        page, t = divmod(s, 16)
        for i in range(64):
            touched[page, :, oc.block_offsets(c, t, i)] = False
    np.testing.assert_array_equal(data[touched], was[touched])


@pytest.mark.parametrize("share", [
    dict(), dict(num_partitions=3, partition=2),
    dict(layout=0, num_partitions=4, partition=1, partition_len=10)])
def test_stored_counts_the_positions_of_the_share(share):
    c = _cache(**share)
    n, p, P = c["num_partitions"], c["partition"], c["partition_len"]
    for x in range(60):
        here = [y for y in range(x)
                if (y % n == p if c["layout"] == 1 else p * P <= y < p * P + P)]
        assert oc.stored(c, x) == len(here)
        np.testing.assert_array_equal(oc.key_positions(c, len(here)), here)


def test_tables_by_hand():
    # 16 tokens a page.  Request 0: 15 + 2 tokens, a page more; request 1:
    # nothing new; request 2: starts with 40 tokens, three pages.
    c = _cache(num_pages=20, max_pages=4)
    table = [[7, -1, -1, -1], [3, -1, -1, -1], [-1] * 4]
    t, lens, cu, slots, pos, rng_out, refused = oc.tables(
        c, [15, 5, 0], [2, 0, 40], [9, 11, 2, 6, 19], [1, 5], table, 44)
    assert t.tolist() == [[7, 11, -1, -1], [3, -1, -1, -1], [2, 6, 19, -1]]
    assert lens.tolist() == [17, 5, 40] and cu.tolist() == [0, 2, 2, 42]
    assert slots.tolist() == ([7 * 16 + 15, 11 * 16]
                              + [2 * 16 + i for i in range(16)]
                              + [6 * 16 + i for i in range(16)]
                              + [19 * 16 + i for i in range(8)] + [-1, -1])
    assert pos.tolist() == [15, 16] + list(range(40)) + [-1, -1]
    assert rng_out.tolist() == [5, 5] and refused == 0


def test_tables_refuse_in_request_order():
    c = _cache(num_pages=20, max_pages=2)
    t, lens, cu, slots, pos, rng_out, refused = oc.tables(
        c, [16, 16, 16, 3], [1, 17, 1, 1], [4, 5], [0, 1], -np.ones((4, 2)),
        20)
    # 0 takes the free page; 1 would need three entries; 2 finds none free; 3
    # needs none, but its table has no page.
    assert lens.tolist() == [17, 16, 16, 4] and refused == 2
    assert rng_out.tolist() == [1, 1] and cu.tolist() == [0, 1, 18, 19, 20]
    assert slots[0] == 64 and np.all(slots[1:] == -1)
    assert pos[0] == 16 and np.all(pos[1:19] == -1) and pos[19] == 3


@pytest.mark.parametrize("n", [1, 2])
def test_attention_is_the_tile_oracle_on_the_stored_values(n):
    """Queries 32 .. 63 of a 64-token sequence over striped shares, merged, as
    the tile of the stored K, V."""
    rng = np.random.default_rng(8)
    q = rng.standard_normal((32, 4, 64))
    k, v = rng.standard_normal((2, 64, 2, 64))
    kq, vq = oc.values(*oc.quantize(k)), oc.values(*oc.quantize(v))
    parts = []
    for p in range(n):
        c = _cache(num_pages=8, max_pages=4, num_partitions=n, partition=p)
        data = np.zeros((8, 2, oc.page_bytes(c)), dtype=np.uint8)
        pages = rng.permutation(8)[:4]
        where = np.arange(p, 64, n)
        slots = [pages[r // 16] * 16 + r % 16 for r in range(len(where))]
        oc.write_rows(c, data, k[where], v[where], slots)
        o, lse, _, _ = oc.attention(c, 0.125, q, np.arange(32, 64), [0, 32],
                                    [64], pages[None], data)
        parts.append((o, lse))
    prob = dict(num_partitions=2, partition_len=32, num_q_heads=4,
                num_kv_heads=2, head_dim=64, causal=1, layout=0,
                softmax_scale=0.125)
    want_o, want_l = oracle.tile_forward(prob, [1], [0, 1], q, kq, vq)
    if n == 1:
        o, lse = parts[0]
    else:
        merged = [oracle.lse_merge(np.stack([o[:, h] for o, _ in parts]),
                                   np.stack([l[h] for _, l in parts]))
                  for h in range(4)]
        o = np.stack([m[0] for m in merged], 1)
        lse = np.stack([m[1] for m in merged])
    np.testing.assert_allclose(o, want_o, atol=1e-12)
    np.testing.assert_allclose(lse, want_l, atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_rotation_of_complex_pairs(interleaved):
    rng = np.random.default_rng(9)
    x = rng.standard_normal((7, 2, 64))
    freq = 10000.0 ** (-np.arange(16) / 16)
    axis = [0] * 10 + [1] * 6
    pos = rng.integers(0, 1000, (2, 7))
    y = oc.rope(x, pos, freq, axis, 32, interleaved)
    a, b = ((slice(0, 32, 2), slice(1, 32, 2)) if interleaved
            else (slice(0, 16), slice(16, 32)))
    z = (x[..., a] + 1j * x[..., b]) * np.exp(
        1j * pos[axis].T * freq)[:, None]
    np.testing.assert_allclose(y[..., a], z.real, atol=1e-12)
    np.testing.assert_allclose(y[..., b], z.imag, atol=1e-12)
    np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
    # The inverse is the transpose.
    back = oc.rope(y, pos, freq, axis, 32, interleaved, inverse=True)
    np.testing.assert_allclose(back, x, atol=1e-12)
    w = rng.standard_normal(x.shape)
    np.testing.assert_allclose(
        (w * y).sum(), (oc.rope(w, pos, freq, axis, 32, interleaved, True)
                        * x).sum())


@pytest.mark.parametrize("shape", [(40, 1, 2, 4, 128), (40, 1, 2, 2, 64),
                                   (11, 8, 2, 4, 128), (5, 40, 1, 3, 64)])
def test_two_bf16_probabilities_miss_the_float32_bound(shape):
    """The bound that the kernel's float32 O is held to: three parts of a
    probability meet it with nothing lost, two parts, cut off or rounded, and one
    do not."""
    x = ExactScores(*shape)
    want, lse = x.want()
    # The inputs are what the cache holds, and the oracle agrees about them.
    for a in (x.k, x.v):
        np.testing.assert_array_equal(oc.values(*oc.quantize(a)), a)
    c = _cache(num_kv_heads=shape[2], head_dim=shape[4], num_pages=1)
    data = np.zeros((1, shape[2], oc.page_bytes(c)), dtype=np.uint8)
    oc.write_rows(c, data, x.k[:2], x.v[:2], [0, 1])
    o, l, _, _ = oc.attention(c, x.scale, x.q[:1], [1], [0, 1], [2],
                              np.array([[0]]), data)
    np.testing.assert_allclose(o, want[:1], rtol=1e-13)
    np.testing.assert_allclose(l, lse[:, :1], rtol=1e-13)

    def off(parts, cut):
        return (np.abs(x.with_parts(parts, cut) - want) / want).max()

    assert off(3, True) < 0.25 * x.O_BOUND
    for parts in (1, 2):
        for cut in (True, False):
            assert off(parts, cut) > 1.5 * x.O_BOUND, (parts, cut)
