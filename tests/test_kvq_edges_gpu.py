"""Calls on the 4-bit cache at the edges of their arguments: windows as large as an int."""
import pytest
import torch

from tests import test_kvq_gpu as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4])
@pytest.mark.parametrize("d,hq,hk,lens,new", [(128, 4, 1, [3, 40, 0], [5, 5, 2]), (128, 8, 1, [20, 70], [40, 12]), (256, 2, 2, [9], [60])])
def test_attend_largest_window(d, hq, hk, lens, new, window):
    # sequences with more queries than tokens among them: their first rows stand before position 0
    base._attend_case(d, hq, hk, 16, torch.bfloat16, lens, new, window=window, seed=d)
