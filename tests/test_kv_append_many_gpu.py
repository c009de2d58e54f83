"""Append to a cache of 16-bit values of so many tokens (20 for each multiprocessor) that a warp takes a whole token, in all its forms.
Tolerances: test_kv_gpu."""
import pytest
import torch

from tests.test_kv_gpu import Case, check_append

pytestmark = pytest.mark.gpu


def case(heads, d, bs, dtype, **kw):
    """In a prompt, a longer one behind text, and a single token."""
    most = torch.cuda.get_device_properties(0).multi_processor_count * 20
    first = most // 2
    return Case([first, most - first + 40, 7], [first, most - first + 5, 1], heads, d, bs, dtype, **kw)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(5, 3), (1, 1), (9, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_dims_heads_and_types(d, hq, hk, dtype):
    check_append(case(hk, d, 16, dtype, seed=d + hq), hq, True, d, False)


@pytest.mark.parametrize("rotary,interleaved,norm", [(16, False, True), (32, True, False), (48, False, False), (64, True, True), (0, False, True), (0, False, False)])
@pytest.mark.parametrize("token_major", [False, True])
def test_transforms(rotary, interleaved, norm, token_major):
    check_append(case(2, 64, 32, torch.bfloat16, token_major=token_major), 4, norm, rotary, interleaved)
    check_append(case(2, 128, 48, torch.float16, layers=2, layer=1, token_major=token_major), 3, norm, rotary, interleaved, positions=True, in_place=True)


@pytest.mark.parametrize("d", [64, 256])
def test_keys_and_values_only(d):
    check_append(case(3, d, 16, torch.bfloat16), 0, True, 32, True)
    check_append(case(3, d, 16, torch.float16), 0, False, 0, False)
