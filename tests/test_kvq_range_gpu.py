"""Attention over the 4-bit cache at the ends of the numbers' range, for one query token (up to 32 rows of a sequence and KV head) and
for prompts. Tolerances are test_kvq_prompt_gpu's, none of them absolute."""
import pytest

from tests import test_kvq_prompt_gpu as prompt

pytestmark = pytest.mark.gpu

# few rows: 8 and 16 of them at a time; and one prompt
SHAPES = [(64, 2, 1, [70, 33], [1, 1]), (128, 8, 2, [200, 40], [1, 1]), (128, 10, 1, [200, 40], [2, 1]), (256, 4, 1, [90], [3]), (128, 4, 1, [90], [20])]


@pytest.mark.parametrize("size", [1e35, 1e30, 1e-30, 1e-35])
@pytest.mark.parametrize("d,hq,hk,lens,new", SHAPES)
def test_queries_and_keys_of_opposite_sizes(d, hq, hk, lens, new, size):
    prompt._range_case(d, hq, hk, lens, new, 1 / size, 1.0, size, seed=d + hq)
