"""What the score-rule calls refuse of arguments at the ends of their ranges, on
the CPU."""

import pytest
import torch

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


def test_a_rule_from_tensors():
    """The structure's own constructor takes what a mapping holds, keeps the
    tensors alive, and has them checked by the calls."""
    slopes, begin = torch.ones(4), torch.zeros(10, dtype=torch.int32)
    rule = ma.Score(cap=30.0, slopes=slopes, key_begin=begin, key_end=None)
    assert rule.cap == 30.0 and rule.slopes == slopes.data_ptr()
    assert rule.key_begin == begin.data_ptr() and rule.key_end is None
    assert rule.tensors[0] is slopes and rule.tensors[1] is begin
    assert ma.Score.make(rule) is rule
    same = ma.Score.make(dict(cap=30.0, slopes=slopes, key_begin=begin))
    assert bytes(same) == bytes(rule)
    assert ma.Score().cap == 0.0
    with pytest.raises(TypeError, match="torch.Tensors"):
        ma.Score(slopes=[1.0])
    with pytest.raises(TypeError, match="torch.Tensors"):
        ma.Score(1.0, slopes.data_ptr())
    with pytest.raises(TypeError):
        ma.Score(window=3)


def test_pointers_set_by_hand_are_refused():
    rule = ma.Score(cap=1.0)
    rule.key_end = 0x100000
    with pytest.raises(ValueError, match="key_end of a score rule must come"):
        b._score_args(rule, 10, 4, 0)
    assert b._score_args(ma.Score(cap=1.0), 10, 4, 0).cap == 1.0
