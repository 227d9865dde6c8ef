"""Rotary positions on the GPU against the float64 oracle."""

import numpy as np
import pytest
import torch

import paper_2512_20968_amd as ma
from oracle import cache as oc

from helpers import exact_angle

pytestmark = pytest.mark.gpu


def _rope(d, rot, axes, inter, base=10000.0):
    n = rot // 2
    return dict(head_dim=d, rotary_dim=rot, num_axes=axes, interleaved=inter,
                inv_freq=[base ** (-i / n) for i in range(n)],
                axis=[i * axes // n for i in range(n)])


def _check(x, y, pos, r, inverse):
    """A component is two products with rounded factors and one sum: off by at
    most 2^-21 of the pair's size (angles good to 2^-24), and half a step of
    bf16, 2^-8 of itself."""
    want = oc.rope(x.double().cpu().numpy(), pos, r["inv_freq"], r["axis"],
                   r["rotary_dim"], r["interleaved"], inverse)
    mag = x.double().abs().cpu().numpy()
    n = r["rotary_dim"] // 2
    pair = mag.copy()
    a, b = ((slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if r["interleaved"]
            else (slice(0, n), slice(n, 2 * n)))
    pair[..., a] = pair[..., b] = np.hypot(mag[..., a], mag[..., b])
    tol = pair * 2.0**-21
    if x.dtype == torch.bfloat16:
        tol += np.abs(want) * 2.0**-8
    got = y.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol)
    np.testing.assert_array_equal(got[..., 2 * n:],
                                  x.double().cpu().numpy()[..., 2 * n:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("d,rot,axes", [
    (16, 16, 1), (64, 64, 1), (128, 128, 3), (128, 64, 2), (80, 48, 3),
    (256, 256, 8), (64, 32, 1), (240, 16, 2)])
@pytest.mark.parametrize("inverse", [0, 1])
def test_rope(dtype, inter, d, rot, axes, inverse):
    gen = torch.Generator().manual_seed(d + rot)
    r = _rope(d, rot, axes, inter)
    for rows, hq, hk in ((1, 1, 1), (7, 3, 2), (65, 8, 0), (130, 2, 5)):
        x = torch.randn(rows, hq + hk + 1, d, generator=gen).to(dtype).cuda()
        pos = np.random.default_rng(rows).integers(-2000, 2**31, (axes, rows))
        pos[:, 0] = 0
        p = torch.tensor(pos).int().cuda()
        q, k = x[:, :hq], x[:, hq:hq + hk]
        yq = torch.full((rows, hq, d), 9.0, dtype=dtype, device="cuda")
        yk = torch.full((rows, hk, d), 9.0, dtype=dtype, device="cuda")
        pos = p.cpu().numpy().astype(np.int64)
        if hk:
            ma.mesh_attn_rope(r, p, q, yq, k, yk, inverse=inverse)
            _check(k, yk, pos, r, inverse)
        else:
            ma.mesh_attn_rope(r, p, q, yq, inverse=inverse)
        _check(q, yq, pos, r, inverse)
        assert torch.equal(yq[0, :, rot:], q[0, :, rot:])
        # In place, within the fused rows; their other heads stay.
        z = x.clone()
        ma.mesh_attn_rope(r, p, z[:, :hq], z[:, :hq],
                          *((z[:, hq:hq + hk],) * 2 if hk else ()),
                          inverse=inverse)
        assert torch.equal(z[:, :hq], yq)
        if hk:
            assert torch.equal(z[:, hq:hq + hk], yk)
        assert torch.equal(z[:, hq + hk:], x[:, hq + hk:])


def test_every_quadrant_and_far_positions():
    """Frequencies of whole eighths of a turn, negative ones and ones past a
    turn, at positions up to the ends of 32 bits."""
    n = 16
    freq = [2 * np.pi * i / 8 for i in range(8)] + [
        -1.0, -1e-9, 0.0, 1.0, 7.5, 1e3, 2.0**31 - 1, 1e-300]
    r = dict(head_dim=32, rotary_dim=32, num_axes=1, interleaved=0,
             inv_freq=freq, axis=[0] * n)
    pos = np.array([0, 1, 2, 3, 5, 7, 8, 1000003, 2**31 - 1, -1, -3, -2**31])
    x = torch.randn(len(pos), 2, 32, generator=torch.Generator().manual_seed(1))
    x = x.cuda()
    y = torch.empty_like(x)
    ma.mesh_attn_rope(r, torch.tensor(pos).int().cuda(), x, y)
    # The oracle's extended precision holds 2^31 * f to 2^-64 of it: enough
    # below f of about 2^10, so the two largest frequencies are left out.
    want = oc.rope(x.double().cpu().numpy(), pos[None], freq, [0] * n, 32,
                   False)
    keep = [i for i in range(32) if i % 16 not in (13, 14)]
    err = np.abs(y.double().cpu().numpy() - want)[..., keep]
    assert err.max() <= 2.0**-20 * 4


def test_gradient_is_the_inverse_turn():
    """<w, R x> differs from <R^-1 w, x> by rounding alone, and R^-1 R is the
    identity: the backward of the tile's float32 dQ, dK."""
    gen = torch.Generator().manual_seed(2)
    r = _rope(128, 128, 3, 0)
    pos = torch.randint(0, 10**6, (3, 200), generator=gen).int().cuda()
    x, w = torch.randn(2, 200, 4, 128, generator=gen).cuda()
    y, z, back = (torch.empty_like(x) for _ in range(3))
    ma.mesh_attn_rope(r, pos, x, y)
    ma.mesh_attn_rope(r, pos, w, z, inverse=1)
    ma.mesh_attn_rope(r, pos, y, back, inverse=1)
    a = (w.double() * y.double()).sum().item()
    b = (z.double() * x.double()).sum().item()
    size = (w.double().norm() * x.double().norm()).item()
    assert abs(a - b) <= 2.0**-20 * size
    assert (back - x).abs().max().item() <= 2.0**-19 * x.abs().max().item() * 2
    # Against differences: the loss <w, R x> along a random direction.
    d = torch.randn(x.shape, generator=gen).cuda()
    moved = torch.empty_like(x)
    ma.mesh_attn_rope(r, pos, x + 0.5 * d, moved)
    diff = ((w.double() * (moved.double() - y.double())).sum() / 0.5).item()
    grad = (z.double() * d.double()).sum().item()
    assert abs(diff - grad) <= 2.0**-19 * (w.double().norm().item()
                                           * (x.double().norm()
                                              + d.double().norm()).item() * 4)


def test_captured_and_on_another_stream():
    r = _rope(64, 64, 1, 1)
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    x = torch.randn(33, 4, 64, device="cuda").to(torch.bfloat16)
    want, y = torch.empty_like(x), torch.zeros_like(x)
    ma.mesh_attn_rope(r, pos, x, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ma.mesh_attn_rope(r, pos, x, y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
    side = torch.cuda.Stream()
    z = torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    ma.mesh_attn_rope(r, pos, x, z, stream=side)
    side.synchronize()
    assert torch.equal(z, want)


def test_more_rows_than_a_launch_counts_threads():
    """33.6 million rows, two to a workgroup of 256 threads: past 2^32 threads."""
    rows = 2**25 + 2**10 + 3
    r = _rope(256, 256, 1, 0)
    x = torch.zeros(rows, 1, 256, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2**32
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    tail = torch.randn(700, 1, 256, generator=torch.Generator().manual_seed(5))
    x[-700:] = tail.to(torch.bfloat16).cuda()
    pos[-700:] = torch.arange(700, device="cuda").int() * 1009
    y, p = x[-700:].clone(), pos[-700:].clone()
    ma.mesh_attn_rope(r, pos, x, x)
    want = torch.empty_like(y)
    ma.mesh_attn_rope(r, p, y, want)
    assert torch.equal(x[-700:], want)
    assert not x[:1000].any() and not x[-2000:-700].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_frequencies_at_far_positions(dtype):
    """Frequencies far past a turn, up to the limit, against angles of exact
    integers; tolerances as _check's."""
    freq = [7.5, 100.0, 1e3, 1e4, 1e6, 1.2e8, -2.0**30, 2.0**31 - 1]
    r = dict(head_dim=16, rotary_dim=16, inv_freq=freq)
    pos = [0, 1, 77, 1000003, 2**30 + 1, 2**31 - 1, -1, -12345, -2**31]
    x = torch.randn(len(pos), 3, 16,
                    generator=torch.Generator().manual_seed(3))
    x = x.to(dtype).cuda()
    y = torch.empty_like(x)
    ma.mesh_attn_rope(r, torch.tensor(pos).int().cuda(), x, y)
    phi = np.array([[exact_angle(f, t) for f in freq] for t in pos])[:, None]
    z = x.double().cpu().numpy()
    a, b = z[..., :8], z[..., 8:]
    want = np.concatenate([a * np.cos(phi) - b * np.sin(phi),
                           b * np.cos(phi) + a * np.sin(phi)], -1)
    tol = np.tile(np.hypot(a, b), 2) * 2.0**-21
    if dtype == torch.bfloat16:
        tol += np.abs(want) * 2.0**-8
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= tol)
