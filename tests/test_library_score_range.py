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
