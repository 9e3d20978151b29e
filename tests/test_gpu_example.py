"""The example trains: every operator of a step together, through autograd."""
import math
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_field_policy_learns():
    import field_policy
    preference, missed = field_policy.main(steps=60, say=lambda *_: None)
    assert abs(preference[0] - math.log(2)) < 1e-3                  # model and reference are the same at first
    assert sum(preference[-10:]) < 0.6 * sum(preference[:10])
    assert sum(missed[-10:]) < sum(missed[:10])
