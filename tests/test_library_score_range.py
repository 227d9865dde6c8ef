"""What the score-rule calls refuse of arguments at the ends of their ranges, on
the CPU."""

import pytest

import paper_2512_20968_amd as ma
from paper_2512_20968_amd import _binding as b

from test_library_score import _bwd, _cfwd, _fwd, _prob, _score


@pytest.mark.parametrize("call", [_fwd, _bwd, _cfwd])
def test_caps(call):
    """Up to 2^100, as long as the scores' factor is a normal float32."""
    for cap in (2.0 ** 101, 1.3e30, 1e37):
        assert call(score=_score(cap=cap)) == b.MA_ERR_INVALID_ARG
        assert "cap" in ma.mesh_attn_last_error()
    small = dict(scale=1e-20) if call is _cfwd else dict(
        prob=_prob(softmax_scale=1e-20))
    assert call(score=_score(cap=1e20), **small) == b.MA_ERR_INVALID_ARG
    assert "cap" in ma.mesh_attn_last_error()
    # The largest one passes: refused for what is checked after it.
    assert call(score=_score(cap=2.0 ** 100), qs=255) == b.MA_ERR_INVALID_ARG
    assert "q_stride" in ma.mesh_attn_last_error()


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_slopes_of_very_many_striped_partitions(call):
    """Positions of 64 rows of a partition span 64 n: more than 2^24 of them is
    more than a float32 holds.  Contiguous partitions, and rules without a bias,
    have no such limit."""
    for n, kw, status in ((2 ** 18 + 1, {}, b.MA_ERR_UNSUPPORTED),
                          (2 ** 20, {}, b.MA_ERR_UNSUPPORTED),
                          (2 ** 18, {}, b.MA_ERR_INVALID_ARG),
                          (2 ** 20, dict(layout=0), b.MA_ERR_INVALID_ARG)):
        prob = _prob(num_partitions=n, **dict(dict(layout=1), **kw))
        # (An odd stride: refused after the check in question.)
        assert call(prob=prob, score=_score(slopes=0x100000), qs=255) == status
        assert ("2^18" in ma.mesh_attn_last_error()) == (
            status == b.MA_ERR_UNSUPPORTED)
    prob = _prob(num_partitions=2 ** 20, layout=1)
    assert call(prob=prob, score=_score(cap=1.0),
                qs=255) == b.MA_ERR_INVALID_ARG
