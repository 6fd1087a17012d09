"""Rows of zeros have codes 0 and scale 0, also where nothing is added to their mean square."""
import pytest
import torch

import paper_2601_19675_amd as ptq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 7, 64, 2048, 4096, 20000])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_zero_rows(dtype, n, eps):
    x = torch.zeros((3, n), dtype=dtype, device="cuda")
    x[1] = 2.0
    ones, nothing = torch.ones(n, dtype=dtype, device="cuda"), torch.zeros(n, dtype=dtype, device="cuda")
    for gamma, residual, row_is_zero in ((None, None, False), (ones, None, False), (None, torch.zeros_like(x), False), (None, -x, True), (nothing, None, True),
                                         (nothing, -x, True)):
        codes = torch.full((3, -(-n // 16) * 16), 9, dtype=torch.int8, device="cuda")[:, :n]
        scales = torch.full((3,), 7.0, device="cuda")
        ptq.ptq_rmsnorm_quantize(x, codes, scales, gamma=gamma, residual=residual, eps=eps)
        assert not codes[[0, 2]].any() and (scales[[0, 2]] == 0).all()
        if row_is_zero:
            assert not codes[1].any() and scales[1] == 0
        else:   # every value is the largest; the mean square is 4
            assert (codes[1] == 127).all()
            assert abs(scales[1].item() - 2 / 127 / (4 + eps) ** 0.5) <= 2.0 ** -23 / 127
