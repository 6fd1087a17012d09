"""The oracle's rows of zeros: codes 0 and scale 0, also where nothing is added to their mean square."""
import numpy as np
import pytest

from oracle import attention_oracle as orc


@pytest.mark.parametrize("eps", [0.0, 1e-5])
@pytest.mark.parametrize("normalize", [True, False])
def test_rows_of_zeros(eps, normalize):
    codes, scales, y = orc.rmsnorm_quantize([[0.0, 0.0], [3.0, 4.0]], residual=[[0.0, 0.0], [-3.0, -4.0]], eps=eps, normalize=normalize)
    assert not codes.any() and not scales.any() and not y.any()
    # zeros because of gamma, not of the row
    codes, scales, _ = orc.rmsnorm_quantize([[3.0, 4.0]], gamma=[0.0, 0.0], eps=eps, normalize=normalize)
    assert not codes.any() and scales[0] == 0
    assert np.isnan(orc.rmsnorm_quantize([[np.nan, 0.0]], eps=eps, normalize=normalize)[1][0])
