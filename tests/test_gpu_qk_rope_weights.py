"""Weights of the norm that are not finite: of a feature that is not rotated one reaches that feature alone, of one that is its pair."""

import numpy as np
import pytest

from tests.test_gpu_qk_rope import Rope

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D, R, interleaved", [(128, 64, False), (128, 96, True), (64, 16, False), (64, 48, True), (128, 0, False)])
def test_weights_that_are_not_finite(D, R, interleaved):
    r = Rope(2, 5, 19, D, R, interleaved, far=900, weights=(True, True))
    r.positions[r.positions == 0] = 1  # (a sine of 0 times an infinity is NaN in the formula, too)
    clean = r.forward()
    for i, (feature, value) in enumerate(((D - 5, np.inf), (R + 3, -np.inf))):
        r.w[i][feature] = value
    r.w[0][D - 6] = np.nan
    got = r.forward()
    for i, feature in enumerate((D - 5, R + 3)):
        rest = [f for f in range(D) if f != feature and (i or f != D - 6)]
        assert np.array_equal(got[i][..., rest], clean[i][..., rest])
        # the weights of these features are near 1: the sign of a result without the infinity is that of x
        assert np.array_equal(got[i][..., feature], np.sign(clean[i][..., feature]) * r.w[i][feature])
    assert np.all(np.isnan(got[0][..., D - 6]))


@pytest.mark.parametrize("D, R, interleaved", [(128, 64, False), (64, 48, True)])
def test_a_weight_of_a_rotated_feature(D, R, interleaved):
    r = Rope(2, 5, 19, D, R, interleaved, far=900)
    r.positions[r.positions == 0] = 1
    clean = r.forward()
    pair = [6, 7] if interleaved else [3, 3 + R // 2]
    r.w[0][pair[0]] = np.inf
    got = r.forward()
    rest = [f for f in range(D) if f not in pair]
    assert np.array_equal(got[0][..., rest], clean[0][..., rest]) and np.array_equal(got[1], clean[1])
    assert np.all(np.isinf(got[0][..., pair]))
