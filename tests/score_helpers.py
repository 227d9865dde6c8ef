"""Inputs, calls and error bounds of the tests of the score-rule operators.

The bounds count what the kernels round, step by step.  U = 2^-8 is half a step
of bf16 relative to the value, E = 2^-24 of float32.  A score's error D is that
of a float32 dot product of d terms, of the cap (its tanh off by 2^-23, the cap's
product and the sums with it by a few E), of the bias and of the exponent;
weights are then off by the factor e^D.  With A_i = sum_j P_ij |v_j|:
  O (bf16)     U A (weights) + U |O| (result) + 2 D A
  O (float32)  2 D A + 16 E A
  LSE          D + 8 E |LSE|
  dV           sum_i P |dO| (U + D_i) + U |dV|
  dK, dQ       s sum P T' |dP - D| |q| (2 U + D_i + 2^-20), the products' own
               errors s sum P T' |q| E (d + 8) (|dO| |v| + |dO| |o|), + U |dK|
(two roundings of dS: its factor P T', and itself).  Second-order terms and the
float32 sums over the keys are covered by a tenth on top and by
2^-20 of the absolute sums.
"""

import numpy as np
import torch

import paper_2512_20968_amd as ma
from oracle import score as os_

U, E = 2.0 ** -8, 2.0 ** -24


def problem(P, n=1, hq=4, hkv=2, d=64, causal=1, layout=0):
    return dict(num_partitions=n, partition_len=P, num_q_heads=hq,
                num_kv_heads=hkv, head_dim=d, causal=causal, layout=layout,
                softmax_scale=float(np.float32(d ** -0.5)))


def bf16(x):
    return torch.tensor(np.asarray(x)).to(torch.float32).to(torch.bfloat16)


def tile_inputs(prob, q_idx, kv_idx, seed, wide=2.0):
    rng = np.random.default_rng(seed)
    P, d = prob["partition_len"], prob["head_dim"]
    rq, rk = len(q_idx) * P, len(kv_idx) * P
    q = bf16(rng.standard_normal((rq, prob["num_q_heads"], d)) * wide)
    k = bf16(rng.standard_normal((rk, prob["num_kv_heads"], d)))
    v = bf16(rng.standard_normal((rk, prob["num_kv_heads"], d)))
    do = bf16(rng.standard_normal((rq, prob["num_q_heads"], d)))
    return q, k, v, do


def documents(total, rng, causal=True, prefix=False, pad=True):
    """key_begin, key_end of every position of packed documents."""
    lo, hi = np.zeros(total, np.int64), np.zeros(total, np.int64)
    stop = total - total // 10 if pad else total
    x = 0
    while x < stop:
        y = min(x + int(rng.integers(1, max(total // 3, 2))), stop)
        lo[x:y] = x
        hi[x:y] = np.arange(x, y) + 1 if causal else y
        if prefix:
            hi[x:y] = np.maximum(hi[x:y], x + (y - x + 2) // 3)
        x = y
    return lo, hi


def make_rule(prob, q_idx, kind, cap, slopes, seed):
    """A rule of a kind as a dict of NumPy arrays."""
    rng = np.random.default_rng(seed + 1000)
    qpos = os_.positions(prob, q_idx)
    total = prob["num_partitions"] * prob["partition_len"]
    rule = {}
    if cap:
        rule["cap"] = cap
    if slopes:
        rule["slopes"] = (2.0 ** -rng.uniform(0, 6, prob["num_q_heads"])
                          ).astype(np.float32)
    if kind == "docs":
        lo, hi = documents(total, rng)
    elif kind == "blocks":
        lo, hi = documents(total, rng, causal=False, pad=False)
    elif kind == "prefix":
        lo, hi = documents(total, rng, prefix=True)
    elif kind == "window":
        rule["key_begin"] = np.maximum(qpos - max(total // 5, 1) + 1, 0)
        return rule
    elif kind == "any":  # ranges in no order, beyond the ends and empty ones
        lo = rng.integers(-5, total + 5, total)
        hi = lo + rng.integers(-3, total + 5, total)
    elif kind == "none":
        lo, hi = np.full(total, 7), np.full(total, 7)
    else:
        return rule
    rule["key_begin"], rule["key_end"] = lo[qpos], hi[qpos]
    return rule


def on_gpu(rule):
    out = {}
    for name, x in rule.items():
        if name == "cap":
            out[name] = x
        else:
            dt = torch.float32 if name == "slopes" else torch.int32
            out[name] = torch.tensor(np.asarray(x)).to(dt).cuda()
    return out


def np64(t):
    return t.double().cpu().numpy()


class Bounds:
    """The oracle's results and how far a kernel's may be from them."""

    def __init__(self, prob, q_idx, kv_idx, rule, q, k, v):
        self.args = prob, q_idx, kv_idx, rule
        self.q, self.k, self.v = np64(q), np64(k), np64(v)
        self.o, self.lse = os_.forward(*self.args, self.q, self.k, self.v)
        qpos, kpos = (os_.positions(prob, x) for x in (q_idx, kv_idx))
        lo, hi = os_.ranges(prob, rule, qpos)
        cap, s = rule.get("cap", 0.0), prob["softmax_scale"]
        d, hq = prob["head_dim"], prob["num_q_heads"]
        self.p, self.grad, self.err = [], [], np.zeros((hq, len(qpos)))
        a = np.zeros(self.o.shape)
        for h in range(hq):
            hk = h // (hq // prob["num_kv_heads"])
            slope = float(rule["slopes"][h]) if "slopes" in rule else 0.0
            x, seen, grad = os_.scores(self.q[:, h], self.k[:, hk], s, cap,
                                       slope, qpos, kpos, lo, hi)
            z = np.where(np.isneginf(self.lse[h]), 0, self.lse[h])
            p = np.exp(np.where(seen, x - z[:, None], -np.inf))
            mag = s * np.abs(self.q[:, h]) @ np.abs(self.k[:, hk]).T
            far = np.abs(qpos[:, None] - kpos[None, :]) * abs(slope)
            near = np.where(seen, far, np.inf).min(1, initial=np.inf)
            near = np.where(np.isinf(near), 0, near)
            dist = np.maximum(far - near[:, None], 0)
            # What can weigh: terms that are 2^-40 of the row's need not be exact.
            e = (E * (d + 8) * mag + cap * 2.0 ** -21 + 8 * E * dist
                 + 8 * E * np.abs(x + far) + 2.0 ** -21)
            e = np.where(p > 2.0 ** -40, e, 0)
            self.err[h] = e.max(1, initial=0) + 4 * E * near
            self.p.append(p)
            self.grad.append(grad)
            a[:, h] = p @ np.abs(self.v[:, hk])
        self.a = a

    def check_forward(self, o, lse, f32):
        o, lse = np64(o), np64(lse)
        e = self.err.T[:, :, None]
        tol = 2 * e * self.a + 16 * E * self.a
        if not f32:
            tol += U * (self.a + np.abs(self.o))
        none = np.isneginf(self.lse)
        assert (np.isneginf(lse) == none).all()
        assert (o.transpose(1, 0, 2)[none] == 0).all()
        off = np.abs(o - self.o) - 1.1 * tol
        assert off.max(initial=-1) <= 1e-30, off.max()
        z = np.where(none, 0, self.lse)
        off = np.abs(np.where(none, 0, lse) - z) - 1.1 * (
            self.err + 8 * E * np.abs(z))
        assert off.max(initial=-1) <= 1e-30, off.max()

    def check_backward(self, o, lse, do, dq, dk, dv):
        prob, _, _, rule = self.args
        s, d, hq = (prob["softmax_scale"], prob["head_dim"],
                    prob["num_q_heads"])
        group = hq // prob["num_kv_heads"]
        o, do = np64(o), np64(do)
        want = os_.backward(*self.args, self.q, self.k, self.v, o, np64(lse),
                            do)
        tol = [np.zeros(x.shape) for x in want]
        for h in range(hq):
            hk = h // group
            q, k, v = self.q[:, h], self.k[:, hk], self.v[:, hk]
            z = np64(lse)[h]
            z0 = np.where(np.isneginf(self.lse[h]), 0, self.lse[h])
            p = self.p[h] * np.exp(z0 - np.where(np.isneginf(z), 0, z)
                                   )[:, None]
            e = self.err[h][:, None] + 8 * E * np.abs(z0)[:, None]
            dd = np.sum(do[:, h] * o[:, h], 1)
            pt = p * self.grad[h]
            part = np.abs(do[:, h] @ v.T - dd[:, None])
            own = E * (d + 8) * (
                np.abs(do[:, h]) @ np.abs(v).T
                + np.sum(np.abs(do[:, h] * o[:, h]), 1)[:, None])
            w = pt * (part * (2 * U + e + 2.0 ** -20) + own)
            # 1 - tanh^2 is off by 2^-21 of one.
            w += p * part * 2.0 ** -21
            tol[0][:, h] += s * w @ np.abs(k)
            tol[1][:, hk] += s * w.T @ np.abs(q)
            tol[2][:, hk] += (p * (U + e + 2.0 ** -20)).T @ np.abs(do[:, h])
        for name, got, x, t in zip(("dq", "dk", "dv"), (dq, dk, dv), want,
                                   tol):
            last = U if got.dtype is torch.bfloat16 else 16 * E
            off = np.abs(np64(got) - x) - 1.1 * (t + last * np.abs(x))
            assert off.max(initial=-1) <= 1e-30, (name, off.max())


def run_forward(prob, q_idx, kv_idx, rule, q, k, v, dtype=torch.bfloat16,
                **kw):
    rows, hq = len(q_idx) * prob["partition_len"], prob["num_q_heads"]
    o = torch.full((rows, hq, prob["head_dim"]), 3.0, dtype=dtype,
                   device="cuda")
    lse = torch.full((hq, rows), 3.0, device="cuda")
    return ma.mesh_attn_score_fwd(prob, q_idx, kv_idx, rule, q, k, v, o, lse,
                                  **kw)


def run_backward(prob, q_idx, kv_idx, rule, q, k, v, o, do, lse,
                 grads=torch.bfloat16, **kw):
    out = [torch.full(x.shape, 3.0, dtype=grads, device="cuda")
           for x in (q, k, v)]
    return ma.mesh_attn_score_bwd(prob, q_idx, kv_idx, rule, q, k, v, o, do,
                                  lse, *out, **kw)
