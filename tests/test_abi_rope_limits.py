"""Rotary frequencies at the ends of the double range: finite ones, or a refusal."""
import math

import pytest

import paper_2111_05972_amd as pkg


# a stretched base past the largest double, one below the least, a stretch that no frequency can be divided by
@pytest.mark.parametrize("rot,scaling,stretch", [(4, pkg.TPL_ROPE_BASE, 1e200), (4, pkg.TPL_ROPE_BASE, 1e-200), (8, pkg.TPL_ROPE_LINEAR, 5e-324),
                                                 (8, pkg.TPL_ROPE_PARTS, 5e-324)])
def test_frequencies_that_are_no_numbers_are_refused(rot, scaling, stretch):
    with pytest.raises(pkg.TpLayerError) as e:
        pkg.tp_layer_rope_frequencies(rot, 10000.0, scaling, stretch, 1.0)
    assert e.value.status == pkg.TPL_EINVAL


@pytest.mark.parametrize("rot,scaling,stretch", [(128, pkg.TPL_ROPE_BASE, 1e200), (4, pkg.TPL_ROPE_BASE, 1e100), (8, pkg.TPL_ROPE_LINEAR, 1e-300), (8, pkg.TPL_ROPE_PARTS, 1e300)])
def test_far_stretches_are_taken(rot, scaling, stretch):
    freq, factor = pkg.tp_layer_rope_frequencies(rot, 10000.0, scaling, stretch, 1.0)
    assert all(math.isfinite(f) and f > 0 for f in freq) and math.isfinite(factor)
