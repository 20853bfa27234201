"""Arguments that the policy's operators cannot answer rightly, refused before a device is touched."""
import math

import pytest

from test_policy_arguments import _scores, _scores_back, _text


@pytest.mark.parametrize("scale", [math.nextafter(2.0 ** 127, math.inf) * (1 + 1e-6), 3e38])
def test_scales_whose_exponents_no_float_holds(scale):
    """Exponents are taken to the base 2: scale times log2 e has to be finite."""
    assert _scores(scale=scale) == -1 and "scale" in _text()
    assert _scores_back(scale=scale) == -1 and "scale" in _text()
