"""Pins of the float64 oracle of attention under a score rule: against the
plain attention of the tile oracle, torch's automatic gradients and differences,
and closed forms."""

import numpy as np
import pytest
import torch

import oracle
from oracle import score as os_

from score_helpers import documents, make_rule, np64, problem, tile_inputs

RULES = [("causal", 0.0, False), ("docs", 5.0, False), ("prefix", 0.0, True),
         ("any", 3.0, True), ("window", 2.0, True)]


def setup(kind, cap, slopes, seed=3, n=2, layout=1):
    prob = problem(12, n=n, hq=4, hkv=2, d=64, layout=layout)
    q_idx, kv_idx = [1, 0], [0, 1]
    rule = make_rule(prob, q_idx, kind, cap, slopes, seed)
    return prob, q_idx, kv_idx, rule, tile_inputs(prob, q_idx, kv_idx, seed)


@pytest.mark.parametrize("causal,layout", [(0, 0), (1, 0), (1, 1)])
def test_no_rule_is_plain_attention(causal, layout):
    prob = problem(16, n=2, hq=4, hkv=2, d=64, causal=causal, layout=layout)
    q, k, v, _ = (np64(x) for x in tile_inputs(prob, [0, 1], [1, 0], 1))
    o, lse = os_.forward(prob, [0, 1], [1, 0], {}, q, k, v)
    ro, rl = oracle.tile_forward(prob, [0, 1], [1, 0], q, k, v)
    np.testing.assert_allclose(o, ro, atol=1e-12)
    np.testing.assert_allclose(lse, rl, atol=1e-12)


@pytest.mark.parametrize("kind,cap,slopes", RULES)
def test_gradients_are_torchs(kind, cap, slopes):
    prob, qi, ki, rule, (q, k, v, do) = setup(kind, cap, slopes)
    q, k, v = (x.double().requires_grad_() for x in (q, k, v))
    qpos, kpos = (torch.tensor(os_.positions(prob, x)) for x in (qi, ki))
    lo, hi = (torch.tensor(x) for x in os_.ranges(prob, rule, qpos.numpy()))
    x = torch.einsum("qhd,khd->hqk", q, k.repeat_interleave(2, 1))
    x = x * prob["softmax_scale"]
    if cap:
        x = cap * torch.tanh(x / cap)
    if slopes:
        far = (qpos[:, None] - kpos).abs()
        x = x - torch.tensor(rule["slopes"]).double()[:, None, None] * far
    seen = (lo[:, None] <= kpos) & (kpos < hi[:, None])
    some = seen.any(1)
    p = torch.softmax(x.masked_fill(~seen, -1e300), -1) * some[:, None]
    o = torch.einsum("hqk,khd->qhd", p, v.repeat_interleave(2, 1))
    o.backward(do.double())
    ro, rl = os_.forward(prob, qi, ki, rule, np64(q.detach()),
                         np64(k.detach()), np64(v.detach()))
    np.testing.assert_allclose(ro, o.detach().numpy(), atol=1e-12)
    got = os_.backward(prob, qi, ki, rule, *(np64(x.detach())
                                             for x in (q, k, v)), ro, rl,
                       np64(do))
    for a, b in zip(got, (q.grad, k.grad, v.grad)):
        np.testing.assert_allclose(a, b.numpy(), atol=1e-12)


@pytest.mark.parametrize("kind,cap,slopes", RULES)
def test_gradients_are_differences(kind, cap, slopes):
    prob, qi, ki, rule, ins = setup(kind, cap, slopes)
    q, k, v, do = (np64(x) for x in ins)
    o, lse = os_.forward(prob, qi, ki, rule, q, k, v)
    grads = os_.backward(prob, qi, ki, rule, q, k, v, o, lse, do)
    rng = np.random.default_rng(0)
    for which in range(3):
        step = rng.standard_normal((q, k, v)[which].shape)
        f = []
        for sign in (1e-5, -1e-5):
            args = [q, k, v]
            args[which] = args[which] + sign * step
            f.append(np.sum(os_.forward(prob, qi, ki, rule, *args)[0] * do))
        want = (f[0] - f[1]) / 2e-5
        got = np.sum(grads[which] * step)
        # Differences of second order: 1e-10 of the third derivative.
        assert abs(want - got) <= 1e-5 * max(1.0, abs(want))


def test_closed_forms():
    """Equal scores: the mean of the seen values; a cap's limit; a bias that
    picks the nearest key."""
    prob = problem(8, hq=1, hkv=1, causal=0)
    v = np.random.default_rng(0).standard_normal((8, 1, 64))
    zero = np.zeros((8, 1, 64))
    lo, hi = np.arange(8) // 2, np.arange(8) // 2 + 3
    o, lse = os_.forward(prob, [0], [0], dict(key_begin=lo, key_end=hi), zero,
                         zero, v)
    for i in range(8):
        np.testing.assert_allclose(o[i, 0], v[lo[i]:hi[i], 0].mean(0))
        np.testing.assert_allclose(lse[0, i], np.log(min(hi[i], 8) - lo[i]))
    big = np.full((8, 1, 64), 1e4)
    _, lse = os_.forward(prob, [0], [0], dict(cap=2.0), big, big, v)
    np.testing.assert_allclose(lse, 2.0 + np.log(8))
    o, lse = os_.forward(prob, [0], [0], dict(slopes=[200.0]), zero, zero, v)
    np.testing.assert_allclose(o[:, 0], v[:, 0])
    np.testing.assert_allclose(lse, 0, atol=1e-12)


def test_hidden_values_reach_nobody():
    prob = problem(4, hq=1, hkv=1)
    q = np.ones((4, 1, 64))
    k, v = q.copy(), q.copy()
    k[3], v[2, 0, 5] = np.nan, np.inf
    o, lse = os_.forward(prob, [0], [0], {}, q, k, v)
    assert np.isfinite(o[:2]).all() and np.isfinite(lse[0, :3]).all()
    assert np.isinf(o[2, 0, 5]) and np.isnan(o[3]).any()
    assert np.isfinite(np.delete(o[2, 0], 5)).all()


def test_cached_is_the_tile_with_windows():
    prob = problem(20, hq=2, hkv=1)
    q, k, v, _ = (np64(x) for x in tile_inputs(prob, [0], [0], 5))
    pos = np.arange(20)
    rule = dict(cap=4.0, slopes=[0.1, 0.3], key_begin=np.maximum(pos - 4, 0))
    o, lse = os_.forward(prob, [0], [0], rule, q, k, v)
    rows = slice(13, 20)
    sub = dict(rule, key_begin=rule["key_begin"][rows])
    co, cl = os_.cached(prob["softmax_scale"], sub, q[rows], pos[rows], pos,
                        k, v, 20)
    np.testing.assert_allclose(co, o[rows], atol=1e-12)
    np.testing.assert_allclose(cl, lse[:, rows], atol=1e-12)


def test_documents_cover_what_they_say():
    lo, hi = documents(50, np.random.default_rng(1), prefix=True)
    assert (lo[:45] <= np.arange(45)).all() and (hi[:45] > np.arange(45)).all()
    assert (lo[45:] == hi[45:]).all()
