"""Single tokens and a few of them over values near float32's smallest and largest numbers: the sum of the weights does not depend on what the
values' scales are."""
import numpy as np
import pytest

from test_gpu_attention_unseen import check_seen
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv,new", [([700], [1]), ([5000], [1]), ([700, 90], [3, 1]), ([700], [40]), ([9000], [40])])
@pytest.mark.parametrize("exponent", [-121, -100, 90, 115])
def test_many_keys_of_one_size(bits, kv, new, exponent):
    p = Problem(kv, new, 8, 2, 64, bits, 16, seed=31)
    p.scales[1] = np.float32(2.0 ** exponent)
    p.check(absolute=True)
    check_seen(p, p.run(), True, 0)
    p.Q[:] = 0.0   # all scores alike: the mean
    check_seen(p, p.run(), True, 0)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kv,new", [([64], [1]), ([700], [1]), ([5000, 3], [1, 1]), ([700], [3]), ([700], [40]), ([5000], [40])])
@pytest.mark.parametrize("low,high", [(-110, 20), (-120, 110), (-60, 70)])
def test_scales_far_from_each_other(bits, kv, new, low, high):
    """Every other key's value is 2^130 and more of its neighbour's; all scores are alike, so that it is half of the mean."""
    p = Problem(kv, new, 8, 2, 64, bits, 16, seed=32)
    p.Q[:] = 0.0
    p.scales[1, :, :, 0::2] = np.float32(2.0 ** low)
    p.scales[1, :, :, 1::2] = np.float32(2.0 ** high)
    check_seen(p, p.run(), True, 0)
    # and with scores of their own
    p = Problem(kv, new, 8, 2, 64, bits, 16, seed=33, q_size=3.0)
    p.scales[1, :, :, 0::2] = np.float32(2.0 ** low)
    p.scales[1, :, :, 1::2] = np.float32(2.0 ** high)
    check_seen(p, p.run(), True, 0)
