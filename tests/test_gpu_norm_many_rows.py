"""Backward of the norm where every block takes several rows in turn (512
blocks of four rows up to 2048 columns, of one row above): the check of
test_gpu_norm.py with its bounds, over the three kinds of row (a wave, four
waves with the next row on its way, sixteen waves without)."""

import pytest

from test_gpu_norm import test_norm_backward as check_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(2049, 31), (4500, 96), (2500, 1536), (8200, 40), (513, 2056), (1100, 5120),
                                       (1600, 8192), (1100, 8200), (700, 16400), (520, 32763)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_sum", [False, True])
def test_several_rows_a_block(rows, cols, dtype, with_sum):
    check_backward(rows, cols, dtype, with_sum)
