"""Refusals of the score-rule calls and of rotation with append, on the CPU: the
C entry points check their arguments before anything is launched, the binding
its tensors."""

import ctypes
import re

import pytest
import torch

import paper_2512_20968_amd as ma
from paper_2512_20968_amd import _binding as b

INVALID, UNSUPPORTED, TOO_SMALL = (b.MA_ERR_INVALID_ARG, b.MA_ERR_UNSUPPORTED,
                                   b.MA_ERR_WORKSPACE_TOO_SMALL)
A = 0x100000  # 16-byte aligned addresses that are never read, 1 MiB apart
I32 = ctypes.POINTER(ctypes.c_int32)


def _prob(**kw):
    p = dict(num_partitions=4, partition_len=10, num_q_heads=4,
             num_kv_heads=2, head_dim=64, causal=1, layout=0,
             softmax_scale=0.125)
    p.update(kw)
    return ma.Problem.make(p)


def _list(x):
    return None if x is None else (ctypes.c_int32 * max(len(x), 1))(*x)


def _score(**kw):
    s = b.Score(kw.pop("cap", 0.0))
    for name, x in kw.items():
        setattr(s, name, x)
    return s


TILE = dict(prob=None, q_idx=[0, 1], nq=None, kv_idx=[0, 1], nkv=None,
            score=None, q=A, qs=256, k=2 * A, ks=128, v=3 * A, vs=128)


def _tile(a):
    q, kv = a["q_idx"], a["kv_idx"]
    return (a["prob"] or _prob(), _list(q),
            len(q or ()) if a["nq"] is None else a["nq"], _list(kv),
            len(kv or ()) if a["nkv"] is None else a["nkv"], a["score"],
            a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"])


def _fwd(o=4 * A, dtype=0, lse=5 * A, ws=6 * A, ws_bytes=1 << 30, **kw):
    return ma.load_library().mesh_attn_score_fwd(
        *_tile(dict(TILE, **kw)), o, dtype, lse, ws, ws_bytes, None)


def _bwd(o=4 * A, d_o=5 * A, lse=6 * A, dq=7 * A, dk=8 * A, dv=9 * A, dtype=0,
         ws=64 * A, ws_bytes=1 << 30, **kw):
    return ma.load_library().mesh_attn_score_bwd(
        *_tile(dict(TILE, **kw)), o, d_o, lse, dq, dk, dv, dtype, ws, ws_bytes,
        None)


BAD_TILES = [
    (dict(prob=_prob(num_partitions=0)), INVALID, "num_partitions"),
    (dict(prob=_prob(partition_len=0)), INVALID, "partition_len"),
    (dict(prob=_prob(partition_len=2**29)), INVALID, "2^30"),
    (dict(prob=_prob(num_q_heads=3)), INVALID, "multiple"),
    (dict(prob=_prob(num_kv_heads=0)), INVALID, "head counts"),
    (dict(prob=_prob(head_dim=96)), UNSUPPORTED, "head_dim"),
    (dict(prob=_prob(causal=2)), INVALID, "causal"),
    (dict(prob=_prob(layout=2)), INVALID, "layout"),
    (dict(prob=_prob(softmax_scale=0.0)), INVALID, "softmax_scale"),
    (dict(prob=_prob(softmax_scale=float("nan"))), INVALID, "softmax_scale"),
    (dict(prob=_prob(softmax_scale=3e38)), INVALID, "softmax_scale"),
    (dict(prob=_prob(partition_len=2**24, num_q_heads=4)), UNSUPPORTED,
     "2^27"),
    (dict(prob=_prob(num_q_heads=65536)), UNSUPPORTED, "num_q_heads"),
    (dict(q_idx=[]), INVALID, "lists"), (dict(kv_idx=[]), INVALID, "lists"),
    (dict(nq=-1), INVALID, "lists"),
    (dict(q_idx=None, nq=2), INVALID, "q_idx is NULL"),
    (dict(kv_idx=None, nkv=2), INVALID, "kv_idx is NULL"),
    (dict(q_idx=[0, 4]), INVALID, "q_idx[1]"),
    (dict(kv_idx=[-1]), INVALID, "kv_idx[0]"),
    (dict(kv_idx=[2, 1, 2]), INVALID, "duplicate"),
    (dict(q_idx=[0, 1, 2, 3, 0]), INVALID, "of 4"),
    (dict(prob=_prob(num_partitions=300, partition_len=1),
          q_idx=list(range(257))), UNSUPPORTED, "256"),
    (dict(score=_score(cap=-1.0)), INVALID, "cap"),
    (dict(score=_score(cap=float("nan"))), INVALID, "cap"),
    (dict(score=_score(cap=float("inf"))), INVALID, "cap"),
    (dict(score=_score(cap=1e-45)), INVALID, "cap"),
    (dict(score=_score(cap=3e38)), INVALID, "cap"),
    (dict(score=_score(slopes=A + 2)), INVALID, "slopes"),
    (dict(score=_score(key_begin=A + 1)), INVALID, "key_begin"),
    (dict(score=_score(key_end=A + 2)), INVALID, "key_end"),
    (dict(qs=255), INVALID, "q_stride"), (dict(qs=260), INVALID, "q_stride"),
    (dict(ks=120), INVALID, "k_stride"), (dict(vs=-128), INVALID, "v_stride"),
    (dict(ks=2**24 + 8), UNSUPPORTED, "k_stride"),
    (dict(q=None), INVALID, "q is NULL"),
    (dict(k=2 * A + 8), INVALID, "k is not 16"),
    (dict(v=None), INVALID, "v is NULL")]


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("kw,status,text", BAD_TILES)
def test_bad_tiles(call, kw, status, text):
    assert call(**kw) == status
    assert text in ma.mesh_attn_last_error()


@pytest.mark.parametrize("kw,status,text", [
    (dict(o=None), INVALID, "o is NULL"),
    (dict(o=4 * A + 4), INVALID, "o is not 16"),
    (dict(lse=None), INVALID, "lse is NULL"), (dict(dtype=2), INVALID, "dtype"),
    (dict(o=A), INVALID, "alias"), (dict(lse=3 * A), INVALID, "alias"),
    (dict(o=A - 16), INVALID, "alias"), (dict(lse=4 * A + 16), INVALID,
                                         "alias"),
    (dict(score=_score(key_end=4 * A)), INVALID, "alias"),
    (dict(score=_score(slopes=5 * A)), INVALID, "alias")])
def test_forward_refusals(kw, status, text):
    assert _fwd(**kw) == status
    assert text in ma.mesh_attn_last_error()


@pytest.mark.parametrize("kw,status,text", [
    (dict(dtype=2), INVALID, "dtype"),
    (dict(o=None), INVALID, "o is NULL"), (dict(d_o=None), INVALID, "d_o is"),
    (dict(lse=None), INVALID, "lse is NULL"),
    (dict(dq=None), INVALID, "dq is NULL"),
    (dict(dk=8 * A + 2), INVALID, "dk is not 16"),
    (dict(dv=None), INVALID, "dv is NULL"), (dict(ws=None), INVALID, "ws is"),
    (dict(ws_bytes=100), TOO_SMALL, "workspace"),
    (dict(dq=5 * A), INVALID, "alias"), (dict(dk=9 * A), INVALID, "alias"),
    (dict(ws=A), INVALID, "alias")])
def test_backward_refusals(kw, status, text):
    assert _bwd(**kw) == status
    assert text in ma.mesh_attn_last_error()


def test_workspaces():
    """Sizes serve every list of the tile's lengths: those of merged segments
    and of separate ones; a byte less is refused."""
    lib = ma.load_library()
    for d in (64, 128):
        for P, n in ((1, 256), (10, 4), (100, 30), (63, 200), (700, 3)):
            for nq, nkv in ((1, n), (n, 1), (n, n), (2, n - 1)):
                prob = _prob(num_partitions=n, partition_len=P, head_dim=d)
                need = (lib.mesh_attn_score_fwd_workspace_size(prob, nq, nkv),
                        lib.mesh_attn_score_bwd_workspace_size(prob, nq, nkv))
                assert need[1] > 0
                # An LSE that is Q: refused after the workspace's check.
                big = dict(o=100 * A, lse=A, ws=500 * A, k=1000 * A,
                           v=1500 * A, qs=4 * d, ks=2 * d, vs=2 * d,
                           prob=prob)
                for lists in ((list(range(nq)), list(range(nkv))),
                              (list(range(nq))[::-1],
                               list(range(nkv))[::-1])):
                    kw = dict(big, q_idx=lists[0], kv_idx=lists[1])
                    assert _fwd(**kw, ws_bytes=need[0]) == INVALID
                    assert "alias" in ma.mesh_attn_last_error()
                    if need[0] == 0:
                        assert _fwd(**kw, ws_bytes=0) == INVALID
                    back = dict(kw, o=200 * A, d_o=300 * A, lse=400 * A, dq=A,
                                dk=2000 * A, dv=2500 * A)
                    assert _bwd(**back, ws_bytes=need[1]) == INVALID
                    assert "alias" in ma.mesh_attn_last_error()
                    assert _bwd(**back, ws_bytes=255) == TOO_SMALL
    for kw in (dict(head_dim=96), dict(num_partitions=0)):
        assert lib.mesh_attn_score_fwd_workspace_size(_prob(**kw), 1, 1) == 0
        assert lib.mesh_attn_score_bwd_workspace_size(_prob(**kw), 1, 1) == 0
    assert lib.mesh_attn_score_fwd_workspace_size(_prob(), 0, 1) == 0
    assert lib.mesh_attn_score_bwd_workspace_size(_prob(), 1, 5) == 0
    assert lib.mesh_attn_score_bwd_workspace_size(None, 1, 1) == 0


# -- the cache ----------------------------------------------------------------

def _cache(**kw):
    c = dict(num_pages=8, page_size=16, num_kv_heads=2, head_dim=64,
             max_pages=4)
    c.update(kw)
    return ma.Cache.make(c)


def _cfwd(c=None, hq=4, scale=0.125, score=None, num_requests=3, rows=5, q=A,
          qs=256, positions=A, cu=A, lens=A, table=A, data=A, o=A, dtype=0,
          lse=A, ws=A, ws_bytes=1 << 30):
    return ma.load_library().mesh_attn_cache_score_fwd(
        c or _cache(), hq, scale, score, num_requests, rows, q, qs, positions,
        cu, lens, table, data, o, dtype, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,text", [
    (dict(hq=3), "num_q_heads"), (dict(scale=0.0), "softmax_scale"),
    (dict(score=_score(cap=-2.0)), "cap"),
    (dict(score=_score(cap=1e-45)), "cap"),
    (dict(score=_score(slopes=A + 1)), "slopes"),
    (dict(score=_score(key_begin=A + 2)), "key_begin"),
    (dict(score=_score(key_end=A + 2)), "key_end"),
    (dict(num_requests=4097), "num_requests"), (dict(rows=2**31), "rows"),
    (dict(dtype=2), "o_dtype"), (dict(qs=255), "q_stride"),
    (dict(q=None), "q is NULL"), (dict(positions=None), "positions is NULL"),
    (dict(cu=None), "cu_new is NULL"), (dict(lens=None), "lens is NULL"),
    (dict(table=None), "block_table is NULL"),
    (dict(data=A + 4), "data is not 16"), (dict(o=None), "o is NULL"),
    (dict(lse=None), "lse is NULL")])
def test_cache_refusals(kw, text):
    assert _cfwd(**kw) == INVALID
    assert text in ma.mesh_attn_last_error()


def test_cache_workspace():
    c = _cache(num_pages=4096, max_pages=4096)
    need = ma.mesh_attn_cache_score_fwd_workspace_size(c, 4, 3, 5)
    assert need == ma.mesh_attn_cache_fwd_workspace_size(c, 4, 3, 5) > 0
    assert _cfwd(c, ws_bytes=need - 1) == TOO_SMALL
    assert _cfwd(rows=0, q=None) == b.MA_OK
    assert _cfwd(num_requests=0, cu=None) == b.MA_OK


def _rope(freq=None, **kw):
    d = dict(head_dim=64, rotary_dim=32, num_axes=1, interleaved=0)
    d.update(kw)
    r = ma.Rope(**d)
    freq = [0.5] * max(d["rotary_dim"] // 2, 1) if freq is None else freq
    r.inv_freq = (ctypes.c_double * len(freq))(*freq)
    return r


def _append(c=None, r=None, rows=4, positions=A, hq=2, q=A, qs=128,
            q_out=2 * A, qos=128, k=A, ks=128, v=A, vs=128, slots=A, data=A):
    return ma.load_library().mesh_attn_cache_rope_append(
        c or _cache(), r or _rope(), rows, positions, hq, q, qs, q_out, qos, k,
        ks, v, vs, slots, data, None)


@pytest.mark.parametrize("kw,status,text", [
    (dict(c=_cache(page_size=5)), UNSUPPORTED, "page_size"),
    (dict(r=_rope(head_dim=128, rotary_dim=64)), INVALID, "of the rotation"),
    (dict(r=_rope(rotary_dim=24)), UNSUPPORTED, "rotary_dim"),
    (dict(r=_rope(num_axes=2)), INVALID, "axis is NULL"),
    (dict(r=_rope(freq=[float("nan")] * 16)), INVALID, "inv_freq[0]"),
    (dict(r=_rope(interleaved=3)), INVALID, "interleaved"),
    (dict(rows=-1), INVALID, "rows"), (dict(rows=2**31), INVALID, "rows"),
    (dict(hq=0), INVALID, "q_heads"), (dict(hq=65536), INVALID, "q_heads"),
    (dict(qs=120), INVALID, "q_stride"),
    (dict(qos=132), INVALID, "q_out_stride"),
    (dict(ks=64), INVALID, "k_stride"), (dict(vs=2**41), INVALID, "v_stride"),
    (dict(q_out=A, qos=256), INVALID, "in place"),
    (dict(positions=None), INVALID, "positions is NULL"),
    (dict(q=None), INVALID, "q is NULL"),
    (dict(q_out=A + 8), INVALID, "q_out is not 16"),
    (dict(k=None), INVALID, "k is NULL"), (dict(v=A + 2), INVALID, "v is not"),
    (dict(slots=A + 4), INVALID, "slots is not 8"),
    (dict(data=None), INVALID, "data is NULL")])
def test_append_refusals(kw, status, text):
    assert _append(**kw) == status
    assert text in ma.mesh_attn_last_error()


def test_append_of_nothing_is_accepted():
    assert _append(rows=0, positions=None, q=None, q_out=None, k=None, v=None,
                   slots=None, data=None) == b.MA_OK


# -- the binding --------------------------------------------------------------

def test_binding_refusals():
    c = _cache()
    x = torch.zeros(10, 4, 64, dtype=torch.bfloat16)
    y = torch.zeros(10, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(10, dtype=torch.int32)
    prob = _prob(num_partitions=1)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_score_fwd(prob, [0], [0], None, x, y, y, x, i)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_score_bwd(prob, [0], [0], None, x, y, y, x, x, i, x, y, y)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_cache_score_fwd(c, 0.1, None, x, i, i, i, i, i, x, i)
    rope = dict(head_dim=64, rotary_dim=32, inv_freq=[1.0] * 16)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        ma.mesh_attn_cache_rope_append(c, rope, i, x, x, y, y, i, i)
    with pytest.raises(TypeError, match="q must be a torch.Tensor"):
        ma.mesh_attn_score_fwd(prob, [0], [0], None, [1], y, y, x, i)
    with pytest.raises(ValueError, match="unknown fields"):
        ma.Score.make(dict(cap=1.0, window=3))
    with pytest.raises(TypeError, match="torch.Tensors"):
        ma.Score.make(dict(key_begin=[1, 2]))
    s = ma.Score.make(None)
    assert s.cap == 0 and not s.slopes and not s.key_begin and not s.key_end
    assert ma.Score.make(s) is s


def test_header_limit_matches_the_library():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "mesh_attn.h")).read()
    most = int(re.search(r"MA_SCORE_MAX_LIST (\d+)", text).group(1))
    prob = _prob(num_partitions=2 * most, partition_len=1)
    assert _fwd(prob=prob, q_idx=list(range(most + 1))) == UNSUPPORTED
    assert str(most) in ma.mesh_attn_last_error()
