"""Refusals of the cache and rotary calls, on the CPU: the C entry points
check their arguments before anything is launched, the binding its tensors."""

import ctypes
import re

import pytest
import torch

import paper_2512_20968_amd as ma
from paper_2512_20968_amd import _binding as b

INVALID, UNSUPPORTED, TOO_SMALL = (b.MA_ERR_INVALID_ARG, b.MA_ERR_UNSUPPORTED,
                                   b.MA_ERR_WORKSPACE_TOO_SMALL)
A = 0x10000  # a 16-byte aligned address that is never read


def _cache(**kw):
    c = dict(num_pages=8, page_size=16, num_kv_heads=2, head_dim=64,
             max_pages=4)
    c.update(kw)
    return ma.Cache.make(c)


BAD_CACHES = [
    (dict(num_pages=0), INVALID, "num_pages"),
    (dict(page_size=8), UNSUPPORTED, "page_size"),
    (dict(page_size=48), UNSUPPORTED, "page_size"),
    (dict(page_size=512), UNSUPPORTED, "page_size"),
    (dict(num_kv_heads=0), INVALID, "num_kv_heads"),
    (dict(num_kv_heads=1025), INVALID, "num_kv_heads"),
    (dict(head_dim=96), UNSUPPORTED, "head_dim"),
    (dict(head_dim=256), UNSUPPORTED, "head_dim"),
    (dict(max_pages=0), INVALID, "max_pages"),
    (dict(max_pages=2**26 + 1), INVALID, "max_pages"),
    (dict(layout=2), INVALID, "layout"),
    (dict(num_partitions=0), INVALID, "partition"),
    (dict(num_partitions=2, partition=2), INVALID, "partition"),
    (dict(partition=-1), INVALID, "partition"),
    (dict(layout=0, partition_len=0), INVALID, "partition_len"),
]


def _read(c, rows=4, args=(A, A, A, A)):
    return ma.load_library().mesh_attn_cache_read(ctypes.byref(c), rows, *args,
                                                  None)


@pytest.mark.parametrize("kw,status,text", BAD_CACHES)
def test_bad_caches(kw, status, text):
    c = _cache(**kw)
    assert _read(c) == status
    assert text in ma.mesh_attn_last_error()
    assert ma.load_library().mesh_attn_cache_bytes(ctypes.byref(c)) == 0
    with pytest.raises(ma.MeshAttnError, match=text):
        ma.mesh_attn_cache_bytes(c)


def test_cache_bytes():
    assert ma.mesh_attn_cache_bytes(_cache()) == 8 * 2 * 16 * 68
    big = _cache(num_pages=2**31 - 1, page_size=256, num_kv_heads=1024,
                 head_dim=128)
    assert ma.mesh_attn_cache_bytes(big) == (2**31 - 1) * 1024 * 256 * 136
    assert ma.load_library().mesh_attn_cache_bytes(None) == 0


def _append(c=None, rows=4, k=A, ks=128, v=A, vs=128, slots=A, data=A):
    return ma.load_library().mesh_attn_cache_append(
        ctypes.byref(c or _cache()), rows, k, ks, v, vs, slots, data, None)


@pytest.mark.parametrize("kw,text", [
    (dict(rows=-1), "rows"), (dict(rows=2**31), "rows"),
    (dict(k=None), "k is NULL"), (dict(v=None), "v is NULL"),
    (dict(slots=None), "slots is NULL"), (dict(data=None), "data is NULL"),
    (dict(k=A + 8), "k is not 16"), (dict(v=A + 2), "v is not 16"),
    (dict(slots=A + 4), "slots is not 8"), (dict(data=A + 8), "data is not"),
    (dict(ks=120), "k_stride"), (dict(ks=132), "k_stride"),
    (dict(vs=0), "v_stride"), (dict(vs=-128), "v_stride"),
    (dict(vs=2**41), "v_stride")])
def test_append_refusals(kw, text):
    assert _append(**kw) == INVALID
    assert text in ma.mesh_attn_last_error()


def test_read_refusals():
    for i, name in enumerate(("slots", "data", "k", "v")):
        args = [A] * 4
        args[i] = None
        assert _read(_cache(), args=args) == INVALID
        assert f"{name} is NULL" in ma.mesh_attn_last_error()
    assert _read(_cache(), rows=-1) == INVALID
    assert _read(_cache(), rows=2**31) == INVALID


def test_nothing_to_do_is_accepted_without_buffers():
    c = _cache()
    assert _append(rows=0, k=None, v=None, slots=None, data=None) == b.MA_OK
    assert _read(c, rows=0, args=[None] * 4) == b.MA_OK
    assert _fwd(rows=0, q=None) == b.MA_OK
    assert _fwd(num_requests=0, cu=None) == b.MA_OK
    assert _rope(rows=0, q=None, q_out=None, positions=None) == b.MA_OK


def _tables(c=None, n=3, lens=A, new=A, free=A, num_free=5, rng=A, table=A,
            lens_out=2 * A, cu=A, rows=7, slots=A, pos=A, rng_out=2 * A,
            refused=A):
    return ma.load_library().mesh_attn_cache_tables(
        ctypes.byref(c or _cache()), n, lens, new, free, num_free, rng, table,
        lens_out, cu, rows, slots, pos, rng_out, refused, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "num_requests"), (dict(n=4097), "num_requests"),
    (dict(rows=-1), "rows"), (dict(num_free=-1), "num_free"),
    (dict(lens=None), "lens is NULL"), (dict(new=None), "new_lens is NULL"),
    (dict(free=None), "free_pages is NULL"),
    (dict(rng=None), "free_range is NULL"),
    (dict(table=None), "block_table is NULL"),
    (dict(lens_out=None), "lens_out is NULL"),
    (dict(cu=None), "cu_new is NULL"), (dict(slots=None), "slots is NULL"),
    (dict(slots=A + 4), "slots is not 8"),
    (dict(pos=A + 2), "positions is not 4"),
    (dict(rng_out=None), "free_range_out is NULL"),
    (dict(refused=None), "refused is NULL"),
    (dict(lens_out=A), "alias"), (dict(rng_out=A), "alias")])
def test_tables_refusals(kw, text):
    assert _tables(**kw) == INVALID
    assert text in ma.mesh_attn_last_error()


def _fwd(c=None, hq=4, scale=0.125, num_requests=3, rows=5, q=A, qs=256,
         positions=A, cu=A, lens=A, table=A, data=A, o=A, dtype=0, lse=A,
         ws=A, ws_bytes=1 << 30):
    return ma.load_library().mesh_attn_cache_fwd(
        ctypes.byref(c or _cache()), hq, scale, num_requests, rows, q, qs,
        positions, cu, lens, table, data, o, dtype, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,text", [
    (dict(hq=0), "num_q_heads"), (dict(hq=3), "num_q_heads"),
    (dict(hq=65536), "num_q_heads"),
    (dict(scale=0.0), "softmax_scale"), (dict(scale=-1.0), "softmax_scale"),
    (dict(scale=float("inf")), "softmax_scale"),
    (dict(scale=3e38), "softmax_scale"),
    (dict(scale=float("nan")), "softmax_scale"),
    (dict(num_requests=-1), "num_requests"),
    (dict(num_requests=4097), "num_requests"), (dict(rows=-1), "rows"),
    (dict(rows=2**31), "rows"), (dict(rows=2**29), "rows * num_q_heads"),
    (dict(dtype=2), "o_dtype"),
    (dict(qs=255), "q_stride"), (dict(qs=260), "q_stride"),
    (dict(q=None), "q is NULL"), (dict(q=A + 8), "q is not 16"),
    (dict(positions=None), "positions is NULL"),
    (dict(cu=None), "cu_new is NULL"), (dict(lens=None), "lens is NULL"),
    (dict(table=None), "block_table is NULL"),
    (dict(data=A + 4), "data is not 16"), (dict(o=None), "o is NULL"),
    (dict(o=A + 2), "o is not 16"), (dict(lse=None), "lse is NULL")])
def test_fwd_refusals(kw, text):
    assert _fwd(**kw) == INVALID
    assert text in ma.mesh_attn_last_error()


def _size(c, hq, n, rows):
    return ma.mesh_attn_cache_fwd_workspace_size(c, hq, n, rows)


def test_fwd_workspace():
    c = _cache(num_pages=4096, max_pages=4096)
    need = _size(c, 4, 3, 5)
    assert 0 < need <= 35 << 20
    assert _fwd(c, ws_bytes=need - 1) == TOO_SMALL
    assert _fwd(c, ws=None, ws_bytes=need) == INVALID
    assert _fwd(c, ws=A + 8, ws_bytes=need) == INVALID
    assert _size(_cache(), 4, 3, 5) == 0
    assert _size(c, 3, 3, 5) == _size(c, 4, -1, 5) == _size(c, 4, 3, -1) == 0
    assert _size(_cache(page_size=5), 4, 3, 5) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 16, 40])
def test_fwd_workspace_never_shrinks(d, group):
    c = _cache(head_dim=d, num_kv_heads=2, num_pages=9000, max_pages=4096)
    sizes = {(n, r): _size(c, 2 * group, n, r)
             for n in (1, 2, 3, 7, 16, 64, 300, 4096)
             for r in (1, 2, 3, 8, 17, 64, 1000, 4096, 100000)}
    for (n, r), s in sizes.items():
        assert 0 < s <= 35 << 20
        for (n2, r2), s2 in sizes.items():
            if n2 >= n and r2 >= r:
                assert s2 >= s


def _rope_desc(freq=None, axis=None, **kw):
    d = dict(head_dim=64, rotary_dim=32, num_axes=1, interleaved=0)
    d.update(kw)
    n = max(d["rotary_dim"] // 2, 1)
    r = ma.Rope(**d)
    if freq is None:
        freq = [0.5] * n
    if freq:
        r.inv_freq = (ctypes.c_double * len(freq))(*freq)
    if axis is not None:
        r.axis = (ctypes.c_int32 * len(axis))(*axis)
    return r


def _rope(r=None, rows=4, positions=A, hq=2, q=A, qs=128, q_out=2 * A, qos=128,
          hk=0, k=None, ks=0, k_out=None, kos=0, dtype=0, inverse=0):
    return ma.load_library().mesh_attn_rope(
        ctypes.byref(r or _rope_desc()), rows, positions, hq, q, qs, q_out,
        qos, hk, k, ks, k_out, kos, dtype, inverse, None)


@pytest.mark.parametrize("kw,status,text", [
    (dict(r=_rope_desc(head_dim=40)), UNSUPPORTED, "head_dim"),
    (dict(r=_rope_desc(head_dim=272)), UNSUPPORTED, "head_dim"),
    (dict(r=_rope_desc(rotary_dim=0)), UNSUPPORTED, "rotary_dim"),
    (dict(r=_rope_desc(rotary_dim=24)), UNSUPPORTED, "rotary_dim"),
    (dict(r=_rope_desc(rotary_dim=80)), UNSUPPORTED, "rotary_dim"),
    (dict(r=_rope_desc(num_axes=0)), INVALID, "num_axes"),
    (dict(r=_rope_desc(num_axes=9)), INVALID, "num_axes"),
    (dict(r=_rope_desc(num_axes=2)), INVALID, "axis is NULL"),
    (dict(r=_rope_desc(num_axes=2, axis=[0] * 15 + [2])), INVALID, "axis[15]"),
    (dict(r=_rope_desc(axis=[-1] * 16)), INVALID, "axis[0]"),
    (dict(r=_rope_desc(interleaved=2)), INVALID, "interleaved"),
    (dict(r=_rope_desc(freq=[])), INVALID, "inv_freq is NULL"),
    (dict(r=_rope_desc(freq=[1.0] * 15 + [float("nan")])), INVALID,
     "inv_freq[15]"),
    (dict(r=_rope_desc(freq=[-2.0**31] * 16)), INVALID, "inv_freq[0]"),
    (dict(inverse=2), INVALID, "inverse"), (dict(dtype=2), INVALID, "dtype"),
    (dict(rows=-1), INVALID, "rows"), (dict(hq=0), INVALID, "q_heads"),
    (dict(hk=-1), INVALID, "k_heads"),
    (dict(qs=120), INVALID, "q_stride"), (dict(qs=132), INVALID, "q_stride"),
    (dict(qos=64), INVALID, "q_out_stride"),
    (dict(hk=1, k=A, k_out=A, ks=32, kos=64), INVALID, "k_stride"),
    (dict(q_out=A, qos=256), INVALID, "in place"),
    (dict(hk=1, k=A, k_out=A, ks=128, kos=64), INVALID, "in place"),
    (dict(q=None), INVALID, "q is NULL"),
    (dict(q=A + 8), INVALID, "q is not 16"),
    (dict(q_out=None), INVALID, "q_out is NULL"),
    (dict(positions=None), INVALID, "positions is NULL"),
    (dict(hk=1, ks=64, kos=64, k_out=A), INVALID, "k is NULL")])
def test_rope_refusals(kw, status, text):
    assert _rope(**kw) == status
    assert text in ma.mesh_attn_last_error()


def test_binding_refuses_cpu_tensors_and_bad_mappings():
    c = _cache()
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    slots = torch.zeros(4, dtype=torch.int64)
    data = torch.zeros(8, 2, 16 * 68, dtype=torch.uint8)
    with pytest.raises(ValueError, match="k must be on a GPU"):
        ma.mesh_attn_cache_append(c, x, x, slots, data)
    with pytest.raises(ValueError, match="slots must be on a GPU"):
        ma.mesh_attn_cache_read(c, slots, data, x, x)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_cache_fwd(c, 0.1, x, slots, slots, slots, slots, data, x,
                               x)
    rope = dict(head_dim=64, rotary_dim=32, inv_freq=[1.0] * 16)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_rope(rope, slots, x, x)
    with pytest.raises(TypeError, match="lens must be a torch.Tensor"):
        ma.mesh_attn_cache_tables(c, [3], *[slots] * 10)
    with pytest.raises(ValueError, match="rotary_dim / 2"):
        ma.Rope.make(dict(rope, inv_freq=[1.0]))
    with pytest.raises(ValueError, match="rotary_dim / 2"):
        ma.Rope.make(dict(rope, axis=[0]))
    with pytest.raises(ValueError, match="go together"):
        ma.mesh_attn_rope(rope, slots, x, x, k=x)


def test_header_limit_matches_the_library():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "mesh_attn.h")).read()
    most = int(re.search(r"MA_CACHE_MAX_REQUESTS (\d+)", text).group(1))
    assert _tables(n=most + 1) == INVALID and str(most) in \
        ma.mesh_attn_last_error()
