"""Attention under a score rule at the ends of what its arguments may be, on the
GPU: wide caps, positions that float32 does not hold, products that overflow,
padding in front of a request; and how often the backward rounds."""

import numpy as np
import pytest
import torch

import paper_2512_20968_amd as ma
from oracle import cache as oc
from oracle import score as os_

from score_helpers import (E, U, Bounds, make_rule, np64, on_gpu, problem,
                           run_backward, run_forward, tile_inputs)
from test_gpu_cache import cache_of, i64
from test_gpu_cache_score import Scored

pytestmark = pytest.mark.gpu


# -- wide caps ----------------------------------------------------------------

class WideBounds(Bounds):
    """The bounds for a cap that says nothing about the scores' size: what the
    tanh is off by is relative to the score.  Of its series (|u| < 0.4) a few E;
    of 1 - 2 r, with r's exponential, reciprocal and product off by a few E each
    of at most one, 2^-21, and tanh is above 0.38: 2^-19 of the score covers
    both."""

    def __init__(self, prob, q_idx, kv_idx, rule, q, k, v):
        super().__init__(prob, q_idx, kv_idx, rule, q, k, v)
        qpos, kpos = (os_.positions(prob, x) for x in (q_idx, kv_idx))
        lo, hi = os_.ranges(prob, rule, qpos)
        s, d, hq = (prob["softmax_scale"], prob["head_dim"],
                    prob["num_q_heads"])
        for h in range(hq):
            hk = h // (hq // prob["num_kv_heads"])
            slope = float(rule["slopes"][h]) if "slopes" in rule else 0.0
            x, seen, _ = os_.scores(self.q[:, h], self.k[:, hk], s,
                                    rule["cap"], slope, qpos, kpos, lo, hi)
            far = np.abs(qpos[:, None] - kpos[None, :]) * abs(slope)
            mag = s * np.abs(self.q[:, h]) @ np.abs(self.k[:, hk]).T
            # (The nearest key is the row's own: no bias that all share.)
            e = (E * (d + 8) * mag + 2.0 ** -19 * np.abs(x + far)
                 + 8 * E * far + 2.0 ** -21)
            e = np.where(self.p[h] > 2.0 ** -40, e, 0)
            self.err[h] = e.max(1, initial=0)


WIDE_CAPS = [300.0, 1e3, 1e4, 1e5, 1e7, 1e30]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", WIDE_CAPS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_caps(cap, slopes, d, dtype):
    prob = problem(150, hq=2, hkv=1, d=d)
    rule = make_rule(prob, [0], "causal", cap, slopes, 3)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 5))
    want = WideBounds(prob, [0], [0], rule, q, k, v)
    o, lse = run_forward(prob, [0], [0], on_gpu(rule), q, k, v, dtype)
    want.check_forward(o, lse, dtype is torch.float32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", WIDE_CAPS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_under_wide_caps(cap, slopes, d, dtype):
    """LSE from the oracle, so that the backward stands by itself."""
    prob = problem(150, hq=2, hkv=1, d=d)
    rule = make_rule(prob, [0], "causal", cap, slopes, 3)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 5))
    want = WideBounds(prob, [0], [0], rule, q, k, v)
    o = torch.tensor(want.o).to(torch.bfloat16).cuda()
    lse = torch.tensor(want.lse).float().cuda()
    grads = run_backward(prob, [0], [0], on_gpu(rule), q, k, v, o, do, lse,
                         grads=dtype)
    want.check_backward(o, lse, do, *grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_caps_that_bend(dtype):
    """Scores of a few times a cap of 1000."""
    prob = problem(140, hq=2, hkv=1, d=64)
    q, k, v, do = (x.cuda() for x in
                   tile_inputs(prob, [0], [0], 9, wide=300.0))
    rule = dict(cap=1000.0)
    want = WideBounds(prob, [0], [0], rule, q, k, v)
    o, lse = run_forward(prob, [0], [0], rule, q, k, v, dtype)
    want.check_forward(o, lse, dtype is torch.float32)


@pytest.mark.parametrize("cap", [255.0, 256.0, 257.0])
def test_caps_around_the_wide_ones(cap):
    """On both sides of where the kernels change over, each other's results."""
    prob = problem(150, hq=2, hkv=1, d=128)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 5))
    rule = dict(cap=cap)
    want = Bounds(prob, [0], [0], rule, q, k, v)
    o, lse = run_forward(prob, [0], [0], rule, q, k, v)
    want.check_forward(o, lse, False)
    grads = run_backward(prob, [0], [0], rule, q, k, v, o, do, lse)
    want.check_backward(o, lse, do, *grads)


def one_request(c, rows, length, rule, group, dtype):
    """O, LSE of a request's last rows, the oracle's, and the error of a score
    that the products make."""
    b = Scored(c, [length], [rows], rule, group=group)
    o, lse = b.run(dtype)
    n = oc.stored(c, length)
    r = np.arange(n)
    page = b.table[0, r // c["page_size"]]
    slots = page * c["page_size"] + r % c["page_size"]
    d = c["head_dim"]
    k = torch.empty(n, c["num_kv_heads"], d, dtype=torch.bfloat16,
                    device="cuda")
    v = torch.empty_like(k)
    ma.mesh_attn_cache_read(c, i64(slots), b.data, k, v)
    q, k, v = np64(b.q), np64(k), np64(v)
    args = (b.scale, b.rule, q, b.positions, oc.key_positions(c, n), k)
    wo, wl = os_.cached(*args, v, length)
    mass, _ = os_.cached(*args, np.abs(v), length)
    reach = b.scale * np.stack(
        [np.abs(q[:, h]) @ np.abs(k[:, h // group]).T
         for h in range(q.shape[1])])
    err = (d + 16) * 2.0 ** -23 * reach.max(-1)
    return np64(o), np64(lse), wo, wl, mass, err


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", WIDE_CAPS)
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_caps_over_the_cache(cap, rows, d, dtype):
    """As over a tile; 2^-14 for the exponentials and sums."""
    c = cache_of(head_dim=d, num_pages=40, max_pages=20)
    o, lse, wo, wl, mass, err = one_request(c, rows, 300, dict(cap=cap), 2,
                                            dtype)
    # Scores that weigh 2^-40 of the row or more lie within 28 of its LSE.
    err = err + 2.0 ** -19 * (np.abs(wl) + 28) + 2.0 ** -14
    assert (np.abs(lse - wl) <= err).all(), np.abs(lse - wl).max()
    tol = 2 * mass * err.T[:, :, None]
    if dtype is torch.bfloat16:
        tol += U * (mass + np.abs(wo))
    assert (np.abs(o - wo) <= tol).all(), (np.abs(o - wo) - tol).max()


# -- positions that float32 does not hold ------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_a_billion_positions_apart(d, dtype):
    """128 rows of which the first 100 are 2^30 positions before all keys and
    the others among them: biases of far keys differ by their distances from
    each other.  The weights' error leaves out what all keys of a row share."""
    n = 2 ** 30 // 100
    prob = problem(100, n=n, hq=2, hkv=1, d=d, causal=0)
    lists = [0, n - 1], [n - 1]
    q, k, v, _ = (x.cuda() for x in tile_inputs(prob, *lists, 2))
    rule = dict(slopes=np.float32([0.5, 0.03]))
    want = Bounds(prob, *lists, rule, q, k, v)
    qpos, kpos = (os_.positions(prob, x) for x in lists)
    far = np.abs(qpos[:, None] - kpos[None, :]).min(1)
    near = 4 * E * rule["slopes"][:, None].astype(float) * far
    want.err = want.err - near
    o, lse = run_forward(prob, *lists, on_gpu(rule), q, k, v, dtype)
    tol = 2 * want.err.T[:, :, None] * want.a + 16 * E * want.a
    if dtype is torch.bfloat16:
        tol += U * (want.a + np.abs(want.o))
    assert (np.abs(np64(o) - want.o) <= 1.1 * tol).all()
    assert (np.abs(np64(lse) - want.lse) <= 1.1 * (want.err + near)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 6.0])
def test_gradients_of_rows_a_billion_positions_apart(d, cap):
    """Partitions of 100 rows at both ends of 2^30 positions: rows 64 .. 127 are
    of both, and the later ones see keys beside them."""
    n = 2 ** 30 // 100
    prob = problem(100, n=n, hq=2, hkv=1, d=d)
    lists = [0, n - 1], [n - 1, 0]
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, *lists, 2))
    qpos = os_.positions(prob, lists[0])
    rule = dict(slopes=np.float32([0.5, 0.03]), key_begin=qpos // 100 * 100)
    if cap:
        rule["cap"] = cap
    want = Bounds(prob, *lists, rule, q, k, v)
    dev = on_gpu(rule)
    o, lse = run_forward(prob, *lists, dev, q, k, v)
    want.check_forward(o, lse, False)
    grads = run_backward(prob, *lists, dev, q, k, v, o, do, lse)
    want.check_backward(o, lse, do, *grads)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 6.0])
def test_most_striped_partitions_with_a_bias(d, cap):
    """Rows and keys almost 2^18 positions apart, each beside a key of another partition:
    the nearest one's bias is exact."""
    n = 2 ** 18 - 3
    prob = problem(200, n=n, hq=2, hkv=1, d=d, causal=0, layout=1)
    lists = [5, n - 1], [7, n - 4]
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, *lists, 2))
    rule = dict(slopes=np.float32([0.5, 2.0 ** -18]))
    if cap:
        rule["cap"] = cap
    want = Bounds(prob, *lists, rule, q, k, v)
    dev = on_gpu(rule)
    o, lse = run_forward(prob, *lists, dev, q, k, v)
    want.check_forward(o, lse, False)
    grads = run_backward(prob, *lists, dev, q, k, v, o, do, lse)
    want.check_backward(o, lse, do, *grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cache_of_a_million_partitions(dtype):
    """Stored keys 2^20 positions apart, the rows right behind the last one: the
    nearest key's bias is exact."""
    n = 2 ** 20
    c = cache_of(num_pages=40, max_pages=20, num_partitions=n, partition=n - 1)
    rule = dict(slopes=np.float32([0.5, 0.3, 0.2, 2.0 ** -20]))
    o, lse, wo, wl, mass, err = one_request(c, 3, 192 * n + 3, rule, 2, dtype)
    err = err + 2.0 ** -14
    assert (np.abs(lse - wl) <= err + 8 * E * np.abs(wl)).all()
    tol = 2 * mass * err.T[:, :, None]
    if dtype is torch.bfloat16:
        tol += U * (mass + np.abs(wo))
    assert (np.abs(o - wo) <= tol).all()


# -- products that overflow ---------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (5.0, False),
                                        (0.0, True), (300.0, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_hidden_products_that_overflow_reach_nobody(cap, slopes, d, dtype):
    """Padding rows and keys that hold finite numbers whose products are
    infinite, or infinite with both signs: results are those of zeros there."""
    prob = problem(330, hq=4, hkv=2, d=d)
    at = np.arange(330)
    hole = (at % 110) >= 90  # rows and keys of no document
    lo = at // 110 * 110
    rule = make_rule(prob, [0], "causal", cap, slopes, 1)
    rule.update(key_begin=np.where(hole, 0, lo),
                key_end=np.where(hole, 0, at + 1))
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 1))
    for x in (q, k, v, do):
        x[hole] = 0
    dev = on_gpu(rule)
    o, lse = run_forward(prob, [0], [0], dev, q, k, v, dtype)
    ob = o.to(torch.bfloat16)
    grads = run_backward(prob, [0], [0], dev, q, k, v, ob, do, lse, dtype)
    for large in (1e38, 1e20, 2.0 ** 64):
        for which in range(5):  # each by itself, then all of them
            ins = [x.clone() for x in (q, k, v, do)]
            for i, x in enumerate(ins):
                if which in (i, 4):
                    sign = torch.ones(d, device="cuda")
                    sign[i::3] = -1
                    x[hole] = (large * sign).to(torch.bfloat16)
            o2, lse2 = run_forward(prob, [0], [0], dev, *ins[:3], dtype)
            assert torch.equal(o, o2) and torch.equal(lse, lse2)
            got = run_backward(prob, [0], [0], dev, *ins[:3], ob, ins[3], lse,
                               dtype)
            for a, b in zip(grads, got):
                assert torch.equal(a, b), (large, which)


# -- padding in front ---------------------------------------------------------

@pytest.mark.parametrize("window", [0, 40])
def test_padding_in_front_of_a_request(window):
    """Rows with begin = end = 0 in front: the rows behind them have the results
    that they have without them."""
    c = cache_of(num_pages=40, max_pages=20)
    b = Scored(c, [300], [30], {})
    begin = np.maximum(b.positions - window + 1, 0) if window else (
        b.positions * 0)
    end = b.positions + 1
    begin[:7] = end[:7] = 0
    b.rule = dict(cap=4.0, key_begin=begin, key_end=end)
    b.check(b.run())
    o, lse = b.run()
    assert (o[:7] == 0).all() and torch.isneginf(lse[:, :7]).all()


# -- how often the backward rounds -------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (5.0, False),
                                        (0.0, True), (300.0, True)])
def test_the_scores_gradient_is_rounded_once(cap, slopes, d):
    """dS enters its products rounded to bf16 once: an error of 2^-8 / sqrt(3) of
    the last power of two, 0.54^(1/2) 2^-8 / sqrt(3) = 0.00166 of a value of any
    size in the root mean square, each apart from the others.  dQ and dK in
    float32 are then off by 0.00166 of the root of the sum of the squared terms; a
    second rounding would make that 1.41 times as much."""
    prob = problem(400, hq=2, hkv=1, d=d)
    rule = make_rule(prob, [0], "causal", cap, slopes, 3)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 5))
    want = Bounds(prob, [0], [0], rule, q, k, v)
    o = torch.tensor(want.o).to(torch.bfloat16).cuda()
    lse = torch.tensor(want.lse).float().cuda()
    grads = run_backward(prob, [0], [0], on_gpu(rule), q, k, v, o, do, lse,
                         grads=torch.float32)
    q, k, v, o, do = (np64(x) for x in (q, k, v, o, do))
    exact = os_.backward(prob, [0], [0], rule, q, k, v, o, np64(lse), do)
    s, step = prob["softmax_scale"], 0.00166
    own = [np.zeros(q.shape), np.zeros(k.shape)]
    for h in range(2):
        ds = s * want.p[h] * want.grad[h] * (
            do[:, h] @ v[:, 0].T - np.sum(do[:, h] * o[:, h], 1)[:, None])
        own[0][:, h] = ds ** 2 @ k[:, 0] ** 2
        own[1][:, 0] += (ds ** 2).T @ q[:, h] ** 2
    for name, got, x, e in zip(("dq", "dk"), grads, exact, own):
        off = np.sqrt(np.sum((np64(got) - x) ** 2))
        assert off < 1.2 * step * np.sqrt(np.sum(e)), (
            name, off / (step * np.sqrt(np.sum(e))))
