"""Attention under a score rule, in float64 NumPy: capped scores, a distance
bias and ranges of keys, over a tile or over the stored rows of a cache.

A rule is a dict with any of cap (0: none), slopes [Hq], key_begin [rows],
key_end [rows].  A problem is the mapping the library takes.
"""

import numpy as np


def positions(prob, idx):
    """Positions of the rows of a buffer that stacks the partitions idx."""
    n, P = prob["num_partitions"], prob["partition_len"]
    r = np.arange(P, dtype=np.int64)
    return np.concatenate([r * n + p if prob.get("layout", 0) else p * P + r
                           for p in idx])


def ranges(prob, rule, qpos):
    total = prob["num_partitions"] * prob["partition_len"]
    lo = rule.get("key_begin")
    hi = rule.get("key_end")
    lo = np.zeros(len(qpos), np.int64) if lo is None else np.asarray(lo)
    if hi is None:
        hi = qpos + 1 if prob["causal"] else np.full(len(qpos), total)
    return lo.astype(np.int64), np.asarray(hi).astype(np.int64)


def scores(q, k, scale, cap, slope, qpos, kpos, lo, hi):
    """(x, seen, derivative of the cap) of one head's rows and keys."""
    with np.errstate(invalid="ignore", over="ignore"):
        x = (q @ k.T) * scale
        grad = np.ones_like(x)
        if cap:
            t = np.tanh(x / cap)
            x, grad = cap * t, 1 - t * t
        x = x - slope * np.abs(qpos[:, None] - kpos[None, :])
    seen = (lo[:, None] <= kpos[None, :]) & (kpos[None, :] < hi[:, None])
    return x, seen, grad


def attend(x, seen, v):
    """(O, LSE) of one head; products with hidden keys are left out."""
    x = np.where(seen, x, -np.inf)
    with np.errstate(invalid="ignore", divide="ignore"):
        top = np.max(x, axis=1, initial=-np.inf)
        ref = np.where(np.isneginf(top), 0.0, top)
        w = np.where(seen, np.exp(x - ref[:, None]), 0.0)
        total = w.sum(1)
        lse = ref + np.log(total)
        bad = ~np.isfinite(v)
        o = w @ np.where(bad, 0.0, v)
        if bad.any():
            for j in np.flatnonzero(bad.any(1)):
                o[seen[:, j]] += np.where(bad[j], v[j], 0.0)
        o = np.where(total[:, None] == 0, 0.0, o / total[:, None])
    return o, lse


def _each_head(prob, rule):
    hq, hkv = prob["num_q_heads"], prob["num_kv_heads"]
    slopes = rule.get("slopes")
    for h in range(hq):
        yield h, h // (hq // hkv), 0.0 if slopes is None else float(slopes[h])


def forward(prob, q_idx, kv_idx, rule, q, k, v):
    """O [rows, Hq, d] and LSE [Hq, rows]."""
    qpos, kpos = positions(prob, q_idx), positions(prob, kv_idx)
    lo, hi = ranges(prob, rule, qpos)
    o = np.zeros(q.shape)
    lse = np.zeros((q.shape[1], q.shape[0]))
    for h, hk, slope in _each_head(prob, rule):
        x, seen, _ = scores(q[:, h], k[:, hk], prob["softmax_scale"],
                            rule.get("cap", 0.0), slope, qpos, kpos, lo, hi)
        o[:, h], lse[h] = attend(x, seen, v[:, hk])
    return o, lse


def backward(prob, q_idx, kv_idx, rule, q, k, v, o, lse, do):
    """dQ, dK, dV from the final O and LSE."""
    qpos, kpos = positions(prob, q_idx), positions(prob, kv_idx)
    lo, hi = ranges(prob, rule, qpos)
    s = prob["softmax_scale"]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h, hk, slope in _each_head(prob, rule):
        x, seen, grad = scores(q[:, h], k[:, hk], s, rule.get("cap", 0.0),
                               slope, qpos, kpos, lo, hi)
        z = np.where(np.isneginf(lse[h]), 0.0, lse[h])
        p = np.exp(np.where(seen, x - z[:, None], -np.inf))
        d = np.sum(do[:, h] * o[:, h], 1)
        ds = p * grad * (do[:, h] @ v[:, hk].T - d[:, None])
        dq[:, h] = s * ds @ k[:, hk]
        dk[:, hk] += s * ds.T @ q[:, h]
        dv[:, hk] += p.T @ do[:, h]
    return dq, dk, dv


def cached(scale, rule, q, qpos, kpos, k, v, length):
    """O [rows, Hq, d], LSE [Hq, rows] of one request's rows over stored keys
    k, v [keys, Hkv, d] at positions kpos, those below its length; no row sees
    keys before the first row's key_begin."""
    rows, hq, _ = q.shape
    lo = rule.get("key_begin")
    hi = rule.get("key_end")
    lo = np.zeros(rows, np.int64) if lo is None else np.asarray(lo, np.int64)
    hi = qpos + 1 if hi is None else np.asarray(hi, np.int64)
    if rows:
        lo = np.maximum(lo, lo[0])
    hi = np.minimum(hi, length)
    group = hq // k.shape[1]
    o, lse = np.zeros(q.shape), np.full((hq, rows), -np.inf)
    for h in range(hq):
        slope = 0.0 if rule.get("slopes") is None else float(rule["slopes"][h])
        x, seen, _ = scores(q[:, h], k[:, h // group], scale,
                            rule.get("cap", 0.0), slope, qpos, kpos, lo, hi)
        o[:, h], lse[h] = attend(x, seen, v[:, h // group])
    return o, lse
