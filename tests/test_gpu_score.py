"""Tile attention under a score rule on the GPU, forward and backward, against
the float64 oracle within counted roundings (score_helpers)."""

import numpy as np
import pytest
import torch

import paper_2512_20968_amd as ma
from oracle import score as os_

from score_helpers import (Bounds, bf16, make_rule, np64, on_gpu, problem,
                           run_backward, run_forward, tile_inputs)

pytestmark = pytest.mark.gpu


def check(prob, q_idx, kv_idx, rule, ins, dtype=torch.bfloat16, backward=True):
    q, k, v, do = (x.cuda() for x in ins)
    want = Bounds(prob, q_idx, kv_idx, rule, q, k, v)
    dev = on_gpu(rule)
    o, lse = run_forward(prob, q_idx, kv_idx, dev, q, k, v, dtype)
    want.check_forward(o, lse, dtype is torch.float32)
    if backward:
        ob = o.to(torch.bfloat16)
        # float32 gradients beside a float32 O, bf16 ones beside a bf16 O.
        grads = run_backward(prob, q_idx, kv_idx, dev, q, k, v, ob, do, lse,
                             grads=dtype)
        want.check_backward(ob, lse, do, *grads)
        if dtype is torch.float32:  # bf16 ones are their roundings
            for a, b in zip(grads, run_backward(prob, q_idx, kv_idx, dev, q, k,
                                                v, ob, do, lse)):
                assert torch.equal(a.to(torch.bfloat16), b)


# -- sizes, rules, layouts ----------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [1, 2, 31, 33, 63, 64, 65, 127, 128, 129, 200,
                               257, 400])
def test_lengths(P, d):
    prob = problem(P, hq=2, hkv=1, d=d)
    rule = make_rule(prob, [0], "causal", 8.0, True, P)
    check(prob, [0], [0], rule, tile_inputs(prob, [0], [0], P))


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("kind", ["causal", "docs", "blocks", "prefix",
                                  "window", "any", "none"])
@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16),
                                     (128, torch.float32)])
def test_rules(kind, cap, slopes, d, dtype):
    prob = problem(301, hq=6, hkv=2, d=d)
    rule = make_rule(prob, [0], kind, cap, slopes, 5)
    check(prob, [0], [0], rule, tile_inputs(prob, [0], [0], 6), dtype)


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("P,n,q_idx,kv_idx", [
    (70, 4, [2], [0, 1, 2, 3]),      # segments that merge, or strides of 4
    (70, 4, [3, 0], [3, 1, 2]),      # lists out of order
    (1, 9, [8, 2, 5], list(range(9))),
    (129, 3, [0, 1, 2], [2]),        # keys behind most rows
    (40, 7, [1, 6, 3], [0, 5, 6]),
])
def test_tiles(P, n, q_idx, kv_idx, layout, causal):
    for kind, cap, slopes, d in (("causal", 0.0, True, 64),
                                 ("docs", 6.0, False, 128),
                                 ("any", 4.0, True, 64)):
        prob = problem(P, n=n, hq=4, hkv=4, d=d, causal=causal, layout=layout)
        rule = make_rule(prob, q_idx, kind, cap, slopes, P + n)
        check(prob, q_idx, kv_idx, rule,
              tile_inputs(prob, q_idx, kv_idx, n))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 1), (12, 4), (40, 8)])
def test_heads(hq, hkv):
    for d in (64, 128):
        prob = problem(150, hq=hq, hkv=hkv, d=d)
        rule = make_rule(prob, [0], "prefix", 7.0, True, hq)
        check(prob, [0], [0], rule, tile_inputs(prob, [0], [0], hq))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_rows_over_many_keys_are_cut(d, dtype):
    """Rows of one partition over the keys of many: the keys are cut into parts
    whose results are merged; equal calls give equal bits."""
    prob = problem(100, n=30, hq=2, hkv=1, d=d)
    q_idx, kv_idx = [29], list(range(30))
    assert ma.mesh_attn_score_fwd_workspace_size(prob, 1, 30) > 0
    for kind, cap in (("causal", 0.0), ("any", 6.0), ("none", 2.0)):
        rule = make_rule(prob, q_idx, kind, cap, True, 3)
        ins = tile_inputs(prob, q_idx, kv_idx, 8)
        check(prob, q_idx, kv_idx, rule, ins, dtype)
        q, k, v, do = (x.cuda() for x in ins)
        dev = on_gpu(rule)
        a = run_forward(prob, q_idx, kv_idx, dev, q, k, v)
        b = run_forward(prob, q_idx, kv_idx, dev, q, k, v)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        g = [run_backward(prob, q_idx, kv_idx, dev, q, k, v, a[0], do, a[1])
             for _ in range(2)]
        assert all(torch.equal(x, y) for x, y in zip(*g))


def test_many_rows_over_few_keys():
    prob = problem(60, n=20, hq=2, hkv=2, d=128, causal=0)
    q_idx, kv_idx = list(range(20)), [7]
    rule = make_rule(prob, q_idx, "window", 3.0, True, 3)
    check(prob, q_idx, kv_idx, rule, tile_inputs(prob, q_idx, kv_idx, 8))


def test_no_rule_is_the_tile():
    """Without a rule and with whole blocks, the results of mesh_attn_tile_fwd
    and _bwd within both's roundings."""
    prob = problem(512, n=2, hq=4, hkv=2, d=128)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0, 1], [0, 1], 4))
    o, lse = run_forward(prob, [0, 1], [0, 1], None, q, k, v)
    to, tl = torch.empty_like(o), torch.empty_like(lse)
    ma.mesh_attn_tile_fwd(prob, [0, 1], [0, 1], q, k, v, to, tl)
    want = Bounds(prob, [0, 1], [0, 1], {}, q, k, v)
    want.check_forward(o, lse, False)
    want.check_forward(to, tl, False)
    grads = run_backward(prob, [0, 1], [0, 1], None, q, k, v, o, do, lse)
    want.check_backward(o, lse, do, *grads)


# -- far positions, large scores ---------------------------------------------

@pytest.mark.parametrize("layout", [0, 1])
def test_far_keys_keep_the_digits_of_their_bias(layout):
    """Keys a million positions from their rows: only differences of their
    biases decide."""
    n = 2 ** 14
    prob = problem(64, n=n, hq=2, hkv=1, d=64, causal=0, layout=layout)
    q_idx, kv_idx = [n - 1], [1, 0] if layout == 0 else [3]
    ins = tile_inputs(prob, q_idx, kv_idx, 2)
    rule = dict(slopes=np.float32([0.5, 0.03]) / (n if layout else 1))
    check(prob, q_idx, kv_idx, rule, ins, torch.float32, backward=False)


@pytest.mark.parametrize("cap", [0.5, 20.0, 1000.0])
def test_scores_far_over_the_cap(cap):
    prob = problem(140, hq=2, hkv=1, d=64)
    q, k, v, do = tile_inputs(prob, [0], [0], 9, wide=300.0)
    check(prob, [0], [0], dict(cap=cap), (q, k, v, do), torch.float32)


def test_infinite_scores_are_the_cap():
    prob = problem(70, hq=1, hkv=1, d=64)
    q, k, v, _ = (x.cuda() for x in tile_inputs(prob, [0], [0], 9))
    q[:], k[:] = 1, 1
    k[::2, 0, 3] = float("inf")
    o, lse = run_forward(prob, [0], [0], dict(cap=3.0), q, k, v)
    x = np.full(70, 3 * np.tanh(8 / 3))
    x[::2] = 3.0
    w = np.tril(np.exp(np.broadcast_to(x, (70, 70))))
    np.testing.assert_allclose(np64(lse)[0], np.log(w.sum(1)), atol=1e-5)
    assert np.isfinite(np64(o)).all()


# -- what is not finite -------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_hidden_infinities_and_nan_reach_nobody(d, dtype):
    """Padding rows of Q, dO and padding keys of K, V full of NaN and
    infinities, between documents: results are those of zeros there."""
    prob = problem(330, hq=4, hkv=2, d=d)
    at = np.arange(330)
    hole = (at % 110) >= 90  # rows and keys of no document
    lo = at // 110 * 110
    rule = dict(cap=5.0, key_begin=np.where(hole, 0, lo),
                key_end=np.where(hole, 0, at + 1))
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 1))
    for x in (q, k, v, do):
        x[hole] = 0
    dev = on_gpu(rule)
    o, lse = run_forward(prob, [0], [0], dev, q, k, v, dtype)
    ob = o.to(torch.bfloat16)
    grads = run_backward(prob, [0], [0], dev, q, k, v, ob, do, lse)
    junk = [float("nan"), float("inf"), -float("inf")]
    for i, x in enumerate((q, k, v, do)):
        for j, r in enumerate(np.flatnonzero(hole)):
            x[r, :, j % d] = junk[(i + j) % 3]
            if j % 3 == 0:
                x[r] = float("nan")
    o2, lse2 = run_forward(prob, [0], [0], dev, q, k, v, dtype)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert (np64(o)[hole] == 0).all() and np.isneginf(np64(lse)[:, hole]).all()
    grads2 = run_backward(prob, [0], [0], dev, q, k, v, ob, do, lse)
    for a, b in zip(grads, grads2):
        assert torch.equal(a, b)
    assert (np64(grads[0])[hole] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_seen_values_that_are_not_finite_reach_their_rows_alone(d):
    prob = problem(200, hq=2, hkv=1, d=d)
    rule = make_rule(prob, [0], "window", 4.0, False, 1)
    q, k, v, _ = (x.cuda() for x in tile_inputs(prob, [0], [0], 1))
    v[50, 0, 3], v[120, 0, d - 1] = float("inf"), float("nan")
    v[121, 0, 0] = -float("inf")
    k[77, 0, 9] = float("nan")
    o, lse = run_forward(prob, [0], [0], on_gpu(rule), q, k, v, torch.float32)
    wo, wl = os_.forward(prob, [0], [0], rule, np64(q), np64(k), np64(v))
    o, lse = np64(o), np64(lse)
    np.testing.assert_array_equal(np.isnan(lse), np.isnan(wl))
    seen_nan = np.isnan(wl)
    assert np.isnan(o.transpose(1, 0, 2)[seen_nan]).all()
    clean = ~seen_nan
    a, b = o.transpose(1, 0, 2)[clean], wo.transpose(1, 0, 2)[clean]
    np.testing.assert_array_equal(np.isposinf(a), np.isposinf(b))
    np.testing.assert_array_equal(np.isneginf(a), np.isneginf(b))
    np.testing.assert_array_equal(np.isnan(a), np.isnan(b))


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_what_is_not_finite_stay_with_their_pairs(d):
    """A NaN in dO's row 60 and one in K's row 100: the rows and keys that see
    them, and no others, have gradients that are not finite."""
    prob = problem(200, hq=1, hkv=1, d=d)
    rule = make_rule(prob, [0], "window", 4.0, False, 1)  # 40 keys
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 1))
    dev = on_gpu(rule)
    o, lse = run_forward(prob, [0], [0], dev, q, k, v)
    do[60, 0, 5] = float("nan")
    k[100, 0, 7] = float("inf")
    dq, dk, dv = (np64(x)[:, 0] for x in run_backward(
        prob, [0], [0], dev, q, k, v, o, do, lse))
    rows, keys = np.zeros(200, bool), np.zeros(200, bool)
    rows[60] = True
    rows[100:140] = True
    keys[21:61] = True
    assert (~np.isfinite(dq).all(1) == rows).all()
    bad = ~np.isfinite(dk).all(1)
    assert bad[keys].all()
    # dK of keys beside key 100 is finite: its score is the cap, its weight too.
    assert not bad[~keys].any()
    assert (~np.isfinite(dv).all(1))[keys].all()
    assert not (~np.isfinite(dv).all(1))[~keys].any()


# -- differences --------------------------------------------------------------

@pytest.mark.parametrize("kind,cap,slopes", [("docs", 4.0, False),
                                             ("prefix", 0.0, True),
                                             ("window", 3.0, True)])
def test_gradients_against_differences_of_the_forward(kind, cap, slopes):
    """<grad, step> against differences of the kernel's own float32 forward.
    bf16 inputs move by powers of two along the step, so that the difference is
    one of exact inputs; the gradient is off by 2^-7 of the absolute sum, the
    difference by its second order (bounded from two step sizes) and by 2^-18 of
    the sum of |O dO| over the step."""
    prob = problem(96, hq=2, hkv=1, d=64)
    rule = make_rule(prob, [0], kind, cap, slopes, 2)
    rng = np.random.default_rng(3)
    ins = [np.round(np64(x) * 16) / 16 for x in
           tile_inputs(prob, [0], [0], 3, wide=1.0)]
    q, k, v = (np.clip(x, -3, 3) for x in ins[:3])
    do = bf16(ins[3]).cuda()
    dev = on_gpu(rule)

    def loss(args):
        o, _ = run_forward(prob, [0], [0], dev, *(bf16(x).cuda()
                                                  for x in args),
                           torch.float32)
        return np.sum(np64(o) * np64(do)), np.sum(np.abs(np64(o) * np64(do)))

    q0, k0, v0 = (bf16(x).cuda() for x in (q, k, v))
    o, lse = run_forward(prob, [0], [0], dev, q0, k0, v0)
    grads = run_backward(prob, [0], [0], dev, q0, k0, v0, o, do, lse)
    for which, g in enumerate(grads):
        sign = np.where(rng.random(g.shape) < 0.5, -1.0, 1.0)
        sign[rng.random(g.shape) < 0.75] = 0
        est = []
        for h in (2.0 ** -5, 2.0 ** -4):
            f = []
            for s in (h, -h):
                args = [q, k, v]
                args[which] = args[which] + s * sign
                assert (np64(bf16(args[which])) == args[which]).all()
                f.append(loss(args))
            est.append(((f[0][0] - f[1][0]) / (2 * h),
                        2.0 ** -18 * f[0][1] / h))
        got, total = np.sum(np64(g) * sign), np.sum(np.abs(np64(g) * sign))
        curve = abs(est[0][0] - est[1][0])
        assert abs(got - est[0][0]) <= (2.0 ** -7 * total + curve + est[0][1]
                                        + est[1][1]), which


# -- strides, streams, workspaces, graphs ------------------------------------

@pytest.mark.parametrize("d", [64, 128])
def test_slices_of_a_fused_projection(d):
    prob = problem(210, hq=4, hkv=2, d=d)
    rule = make_rule(prob, [0], "docs", 5.0, True, 2)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 7))
    dev = on_gpu(rule)
    o, lse = run_forward(prob, [0], [0], dev, q, k, v)
    grads = run_backward(prob, [0], [0], dev, q, k, v, o, do, lse)
    fused = torch.full((210, 9, d), float("nan"), dtype=torch.bfloat16,
                       device="cuda")
    fused[:, :4], fused[:, 5:7], fused[:, 7:] = q, k, v
    parts = fused[:, :4], fused[:, 5:7], fused[:, 7:]
    o2, lse2 = run_forward(prob, [0], [0], dev, *parts)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(grads, run_backward(prob, [0], [0], dev, *parts, o, do,
                                        lse)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_the_widest_strides_pass_32_bits(d):
    prob = problem(205, hq=2, hkv=1, d=d)
    rule = on_gpu(make_rule(prob, [0], "docs", 5.0, True, 2))
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 7))
    o, lse = run_forward(prob, [0], [0], rule, q, k, v)
    grads = run_backward(prob, [0], [0], rule, q, k, v, o, do, lse)
    wide = torch.empty(205, 2 ** 24, dtype=torch.bfloat16, device="cuda")
    parts = [wide[:, at:at + n * d].view(205, n, d)
             for at, n in ((0, 2), (2 ** 23, 1), (2 ** 24 - d, 1))]
    for x, y in zip(parts, (q, k, v)):
        x.copy_(y)
    o2, lse2 = run_forward(prob, [0], [0], rule, *parts)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for x, y in zip(grads, run_backward(prob, [0], [0], rule, *parts, o, do,
                                        lse)):
        assert torch.equal(x, y)


def test_other_streams_and_workspaces():
    """Calls on a stream of their own, with a workspace and without; a
    workspace's old contents do not matter, and nothing behind it is touched."""
    prob = problem(300, n=3, hq=2, hkv=1, d=64)
    q_idx, kv_idx = [2], [0, 1, 2]
    rule = on_gpu(make_rule(prob, q_idx, "any", 5.0, True, 2))
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, q_idx, kv_idx, 7))
    o, lse = run_forward(prob, q_idx, kv_idx, rule, q, k, v)
    grads = run_backward(prob, q_idx, kv_idx, rule, q, k, v, o, do, lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    nf = ma.mesh_attn_score_fwd_workspace_size(prob, 1, 3)
    nb = ma.mesh_attn_score_bwd_workspace_size(prob, 1, 3)
    for ws in (None, 255):
        wf = wb = None
        if ws:
            wf, wb = (torch.full((n + 256,), ws, dtype=torch.uint8,
                                 device="cuda") for n in (nf, nb))
            torch.cuda.synchronize()
        o2, lse2 = run_forward(prob, q_idx, kv_idx, rule, q, k, v, stream=side,
                               ws=None if wf is None else wf[:nf])
        side.synchronize()
        g2 = run_backward(prob, q_idx, kv_idx, rule, q, k, v, o, do, lse,
                          stream=side, ws=None if wb is None else wb[:nb])
        side.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert all(torch.equal(a, b) for a, b in zip(grads, g2))
        if ws:
            assert (wf[nf:] == ws).all() and (wb[nb:] == ws).all()


def test_results_stay_inside_their_buffers():
    prob = problem(77, hq=3, hkv=3, d=64)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 7))
    rule = on_gpu(make_rule(prob, [0], "any", 0.0, True, 2))
    n = 77 * 3 * 64
    big = [torch.full((n + 512,), 9.0, dtype=torch.bfloat16, device="cuda")
           for _ in range(4)]
    o, dq, dk, dv = (x[256:256 + n].view(77, 3, 64) for x in big)
    lse = torch.full((77 * 3 + 256,), 9.0, device="cuda")
    l3 = lse[128:128 + 231].view(3, 77)
    ma.mesh_attn_score_fwd(prob, [0], [0], rule, q, k, v, o, l3)
    ma.mesh_attn_score_bwd(prob, [0], [0], rule, q, k, v, o, do, l3, dq, dk,
                           dv)
    for x in big:
        assert (x[:256] == 9).all() and (x[256 + n:] == 9).all()
    assert (lse[:128] == 9).all() and (lse[359:] == 9).all()


def test_a_captured_step_replays_with_other_ranges():
    """Forward and backward in a graph; before every replay the ranges, the
    inputs and eager work of the same leaves change."""
    prob = problem(260, hq=4, hkv=2, d=64)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], 1))
    rule = on_gpu(make_rule(prob, [0], "docs", 5.0, True, 1))
    o = torch.empty_like(q)
    lse = torch.empty(4, 260, device="cuda")
    grads = [torch.empty_like(x) for x in (q, k, v)]
    wf = torch.empty(max(ma.mesh_attn_score_fwd_workspace_size(prob, 1, 1),
                         16), dtype=torch.uint8, device="cuda")
    wb = torch.empty(ma.mesh_attn_score_bwd_workspace_size(prob, 1, 1),
                     dtype=torch.uint8, device="cuda")

    def step():
        ma.mesh_attn_score_fwd(prob, [0], [0], rule, q, k, v, o, lse, ws=wf)
        ma.mesh_attn_score_bwd(prob, [0], [0], rule, q, k, v, o, do, lse,
                               *grads, ws=wb)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        kind = ("docs", "any", "none", "prefix")[seed]
        new = on_gpu(make_rule(prob, [0], kind, 5.0, True, seed + 9))
        for name in ("slopes", "key_begin", "key_end"):
            rule[name].copy_(new[name])
        for a, b in zip((q, k, v, do), tile_inputs(prob, [0], [0], seed + 9)):
            a.copy_(b)
        graph.replay()
        got = [x.clone() for x in (o, lse, *grads)]
        torch.cuda.synchronize()
        step()
        for a, b in zip(got, (o, lse, *grads)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    prob = problem(400, hq=4, hkv=1, d=128)
    sets = []
    for i in range(2):
        q, k, v, do = (x.cuda() for x in tile_inputs(prob, [0], [0], i))
        rule = on_gpu(make_rule(prob, [0], "docs", 5.0 + i, False, i))
        o, lse = run_forward(prob, [0], [0], rule, q, k, v)
        g = run_backward(prob, [0], [0], rule, q, k, v, o, do, lse)
        sets.append((rule, q, k, v, do, o, lse, g, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (rule, q, k, v, do, o, lse, g, s) in enumerate(sets):
            with torch.cuda.stream(s):
                a = run_forward(prob, [0], [0], rule, q, k, v)
                b = run_backward(prob, [0], [0], rule, q, k, v, o, do, lse)
            got[i].append((a, b))
    torch.cuda.synchronize()
    for i, (_, _, _, _, _, o, lse, g, _) in enumerate(sets):
        for a, b in got[i]:
            assert torch.equal(a[0], o) and torch.equal(a[1], lse)
            assert all(torch.equal(x, y) for x, y in zip(b, g))


# -- a mesh's partials --------------------------------------------------------

def test_partials_of_two_gpus_merge_to_the_whole():
    """float32 partials over each half of the keys, merged, are the whole
    tile's result; the two halves' dQ sum to it."""
    prob = problem(130, n=4, hq=4, hkv=2, d=64, layout=1)
    q_idx, kv = [1, 2], [0, 1, 2, 3]
    rule = make_rule(prob, q_idx, "prefix", 6.0, True, 3)
    q, k, v, do = (x.cuda() for x in tile_inputs(prob, q_idx, kv, 4))
    dev = on_gpu(rule)
    parts = [run_forward(prob, q_idx, kv[a:a + 2], dev, q,
                         k[130 * a:130 * (a + 2)], v[130 * a:130 * (a + 2)],
                         torch.float32) for a in (0, 2)]
    o = torch.empty(260, 4, 64, device="cuda")
    lse = torch.empty(4, 260, device="cuda")
    ma.mesh_attn_lse_merge(torch.stack([p[0] for p in parts]),
                           torch.stack([p[1] for p in parts]), o, lse)
    want = Bounds(prob, q_idx, kv, rule, q, k, v)
    want.check_forward(o, lse, True)


@pytest.mark.parametrize("seed", range(6))
def test_drawn_tiles(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 6))
    P = int(rng.integers(1, 250))
    hkv = int(rng.integers(1, 4))
    prob = problem(P, n=n, hq=hkv * int(rng.integers(1, 4)), hkv=hkv,
                   d=int(rng.choice([64, 128])), causal=int(rng.integers(2)),
                   layout=int(rng.integers(2)))
    q_idx, kv_idx = (list(map(int, rng.permutation(n)[:rng.integers(1, n + 1)]))
                     for _ in range(2))
    kind = str(rng.choice(["causal", "docs", "prefix", "window", "any"]))
    rule = make_rule(prob, q_idx, kind, float(rng.choice([0, 3, 30])),
                     bool(rng.integers(2)), seed)
    check(prob, q_idx, kv_idx, rule, tile_inputs(prob, q_idx, kv_idx, seed),
          torch.float32 if seed % 2 else torch.bfloat16)
