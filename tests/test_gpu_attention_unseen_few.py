"""test_gpu_attention_unseen for single tokens and a few of them: rows that do not see an altered key keep every bit."""
import pytest

from test_gpu_attention_unseen import FACTORS, both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("bits,d,page", [(8, 128, 16), (4, 64, 16), (8, 80, 1), (4, 256, 64)])
def test_a_few_tokens(bits, d, page, factor):
    both([130, 47, 9], [4, 2, 1], 8, 2, d, bits, page, 0, [128], factor)
    both([130, 47, 9], [4, 2, 1], 8, 2, d, bits, page, 0, list(range(60, 77)), factor, window=50, keys_too=True)
    both([3000, 47, 9], [4, 2, 1], 8, 2, d, bits, page, 0, [2998], factor)
