"""The paged key/value cache in 4 bits, attention over it and rotary positions,
in float64 NumPy and Python loops.

A cache here is a dict: num_pages, page_size, num_kv_heads, head_dim, max_pages
and the stored positions: layout 1 (striped) stores p, p + n, p + 2n, .., layout
0 (contiguous) p P .. p P + P - 1.
"""

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32
INT32_MAX = 2**31 - 1


def stored(cache, x):
    """The stored positions below x are local tokens 0 .. stored(x) - 1."""
    n, p = cache.get("num_partitions", 1), cache.get("partition", 0)
    if cache.get("layout", 1) == 1:
        return 0 if x <= p else (x - p + n - 1) // n
    first = p * cache["partition_len"]
    return min(max(x - first, 0), cache["partition_len"])


def key_positions(cache, count):
    """Global positions of local tokens 0 .. count - 1."""
    r = np.arange(count, dtype=np.int64)
    if cache.get("layout", 1) == 1:
        return r * cache.get("num_partitions", 1) + cache.get("partition", 0)
    return cache.get("partition", 0) * cache["partition_len"] + r


# -- quantization -----------------------------------------------------------

def quantize_group(x):
    """Codes (0 .. 15) and scale code of 32 float64 values."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return np.zeros(x.size, dtype=np.uint8), 255
    amax = np.abs(x).max()
    e = -126
    if amax > 0:
        _, exp = np.frexp(amax)          # amax in [2^(exp-1), 2^exp)
        top = float(exp - 1)
        e = int(top) - 2 + (1 if amax > 1.75 * 2.0**top else 0)
        e = min(max(e, -126), 125)
    codes = np.zeros(x.size, dtype=np.uint8)
    for i, y in enumerate(x * 2.0**-e):
        dist = np.abs(E2M1 - abs(y))
        best = np.flatnonzero(dist == dist.min())
        code = next(c for c in best if c % 2 == 0) if len(best) > 1 else best[0]
        codes[i] = code + (8 if np.signbit(y) else 0)
    return codes, e + 127


def quantize(x):
    """``(codes[.., d], scales[.., d/32])`` of ``x[.., d]``."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(-1, GROUP)
    out = [quantize_group(row) for row in g]
    codes = np.array([c for c, _ in out], dtype=np.uint8).reshape(x.shape)
    scales = np.array([s for _, s in out], dtype=np.uint8)
    return codes, scales.reshape(x.shape[:-1] + (x.shape[-1] // GROUP,))


def values(codes, scales):
    """What codes and scale codes stand for, float64."""
    mag = E2M1[codes & 7]
    val = np.where(codes & 8, -mag, mag)
    scale = np.where(scales == 255, np.nan,
                     2.0 ** (scales.astype(np.float64) - 127))
    return val * np.repeat(scale, GROUP, axis=-1)


# -- layout -----------------------------------------------------------------

def block_offsets(cache, t, i):
    """Byte offsets in a (page, KV head) block of dim i of token t: (K code, V
    code, K scale, V scale); the codes are in the low four bits for even i."""
    ps, d = cache["page_size"], cache["head_dim"]
    n, rest = divmod(i, d // 16)
    return (t * (d // 2) + i // 2,
            ps * d // 2 + (t // 8) * 4 * d + n * (d // 4) + (t % 8) * (d // 32)
            + rest // 2,
            ps * d + t * (d // 32) + i // 32,
            ps * d + ps * d // 32 + (i // 32) * ps + t)


def page_bytes(cache):
    d = cache["head_dim"]
    return cache["page_size"] * (d + d // 16)


def write_rows(cache, data, k, v, slots):
    """Quantizes and writes rows of k, v [rows, Hkv, d] into data [pages, Hkv,
    page bytes] (uint8)."""
    ps, d = cache["page_size"], cache["head_dim"]
    kc, ks = quantize(k)
    vc, vs = quantize(v)
    for r, slot in enumerate(slots):
        if not 0 <= slot < cache["num_pages"] * ps:
            continue
        page, t = divmod(int(slot), ps)
        for h in range(cache["num_kv_heads"]):
            blk = data[page, h]
            for i in range(d):
                ka, va, ksa, vsa = block_offsets(cache, t, i)
                shift = 4 * (i % 2)
                blk[ka] = (blk[ka] & (0xF0 >> shift)) | (kc[r, h, i] << shift)
                blk[va] = (blk[va] & (0xF0 >> shift)) | (vc[r, h, i] << shift)
                blk[ksa] = ks[r, h, i // 32]
                blk[vsa] = vs[r, h, i // 32]


def read_row(cache, data, slot):
    """``(k, v) [Hkv, d]`` stored at a slot; zeros for one out of range."""
    ps, d, hkv = cache["page_size"], cache["head_dim"], cache["num_kv_heads"]
    if not 0 <= slot < cache["num_pages"] * ps:
        return np.zeros((hkv, d)), np.zeros((hkv, d))
    page, t = divmod(int(slot), ps)
    at = np.array([block_offsets(cache, t, i) for i in range(d)])
    shift = 4 * (np.arange(d) % 2)
    blk = data[page]
    kc = (blk[:, at[:, 0]] >> shift) & 15
    vc = (blk[:, at[:, 1]] >> shift) & 15
    return (values(kc, blk[:, at[::32, 2]]), values(vc, blk[:, at[::32, 3]]))


# -- tables -----------------------------------------------------------------

def tables(cache, lens, new_lens, free_pages, free_range, block_table, rows):
    """``(block_table, lens_out, cu_new, slots, positions, free_range_out,
    refused)`` as mesh_attn_cache_tables defines them, request by request."""
    ps = cache["page_size"]
    table = np.array(block_table, dtype=np.int64, copy=True)
    first = min(max(int(free_range[0]), 0), len(free_pages))
    last = min(max(int(free_range[1]), first), len(free_pages))
    lens_out, cu = [], [0]
    slots = np.full(rows, -1, dtype=np.int64)
    positions = np.full(rows, -1, dtype=np.int64)
    wanted = taken = refused = 0
    for b in range(len(lens)):
        have, new = max(int(lens[b]), 0), max(int(new_lens[b]), 0)
        start = cu[-1]
        cu.append(min(start + new, INT32_MAX))
        before = -(-stored(cache, have) // ps)
        ok = have + new <= INT32_MAX
        after = -(-stored(cache, have + new) // ps) if ok else before
        ok = ok and after <= cache["max_pages"]
        begin = wanted
        if ok:
            wanted += after - before
            ok = after == before or wanted <= last - first
        if not ok:
            refused += 1
            lens_out.append(int(lens[b]))
            continue
        lens_out.append(have + new)
        for j in range(after - before):
            table[b, before + j] = free_pages[first + begin + j]
        taken = max(taken, wanted) if after > before else taken
        for i in range(min(new, max(rows - start, 0))):
            x = have + i
            positions[start + i] = x
            if stored(cache, x + 1) > stored(cache, x):
                page, t = divmod(stored(cache, x), ps)
                page = table[b, page]
                if 0 <= page < cache["num_pages"]:
                    slots[start + i] = page * ps + t
    return (table, np.array(lens_out), np.array(cu), slots, positions,
            np.array([first + taken, last]), refused)


# -- attention --------------------------------------------------------------

def visible_keys(cache, table_row, length, position):
    """``(local tokens, slots)`` that a query at ``position`` sees."""
    ps = cache["page_size"]
    count = min(stored(cache, max(int(length), 0)), cache["max_pages"] * ps)
    where = key_positions(cache, count)
    out = []
    for r in range(count):
        page = int(table_row[r // ps])
        if where[r] <= position and 0 <= page < cache["num_pages"]:
            out.append((r, page * ps + r % ps))
    return out


def attention(cache, scale, q, positions, cu_new, lens, block_table, data):
    """O [rows, Hq, d], LSE [Hq, rows] and, per row and head, sum_j p_j |v_j|
    (as O) and the largest scale * sum |q_i k_ji| over the visible keys (as LSE).
    Rows of no request are NaN."""
    rows, hq, d = q.shape
    group = hq // cache["num_kv_heads"]
    o, mass = np.full((2, rows, hq, d), np.nan)
    lse, reach = np.full((2, hq, rows), np.nan)
    for b in range(len(lens)):
        stored_rows = {}
        for row in range(max(cu_new[b], 0), min(cu_new[b + 1], rows)):
            keys = visible_keys(cache, block_table[b], lens[b],
                                int(positions[row]))
            if not keys:
                o[row], mass[row] = 0.0, 0.0
                lse[:, row], reach[:, row] = -np.inf, 0.0
                continue
            for _, s in keys:
                if s not in stored_rows:
                    stored_rows[s] = read_row(cache, data, s)
            k = np.stack([stored_rows[s][0] for _, s in keys])
            v = np.stack([stored_rows[s][1] for _, s in keys])
            for h in range(hq):
                kh, vh = k[:, h // group], v[:, h // group]
                x = scale * (kh @ q[row, h])
                top = x.max()
                p = np.exp(x - top)
                total = p.sum()
                lse[h, row] = top + np.log(total)
                o[row, h] = (p @ vh) / total
                mass[row, h] = (p @ np.abs(vh)) / total
                reach[h, row] = scale * (np.abs(kh) @ np.abs(q[row, h])).max()
    return o, lse, mass, reach


# -- rotary positions ---------------------------------------------------------

def rope(x, positions, inv_freq, axis, rotary_dim, interleaved, inverse=False):
    """x [rows, heads, d] turned by positions [axes, rows]; the angles' turns
    are reduced in extended precision."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    two_pi = 2 * np.pi
    for i in range(rotary_dim // 2):
        a, b = ((2 * i, 2 * i + 1) if interleaved
                else (i, i + rotary_dim // 2))
        phi = np.asarray(positions[axis[i]], dtype=np.longdouble) \
            * np.longdouble(inv_freq[i])
        phi = np.asarray(np.remainder(
            phi, np.longdouble("6.283185307179586476925286766559")),
            dtype=np.float64)
        phi = np.where(phi > two_pi / 2, phi - two_pi, phi)
        c, s = np.cos(phi)[:, None], np.sin(phi)[:, None]
        if inverse:
            s = -s
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
