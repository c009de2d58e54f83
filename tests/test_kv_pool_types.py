"""A cache of 16-bit values is of the type of the rows that are written to it or read from it: calls that mix types are refused before
anything is enqueued. Tensors are stood in for, so no GPU is needed."""
import pytest
import torch

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200._lib import RempBlockTables, RempKvqBatch

PTR = 1 << 20  # stands for device memory; never dereferenced


class Rows:
    def __init__(self, dtype, shape=(4, 2, 128), is_cuda=True):
        self.dtype, self.shape, self.is_cuda, self.nbytes = dtype, shape, is_cuda, 1 << 40

    def data_ptr(self):
        return PTR

    def numel(self):
        return 1

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def stride(self, i=None):
        strides = (self.shape[1] * self.shape[2], self.shape[2], 1)
        return strides if i is None else strides[i]


def pool(dtype):
    return remp.make_kv_pool(Rows(dtype), 8, 2, 128, 16)


def calls(cache, dtype):
    batch = RempKvqBatch(RempBlockTables(0, 4, PTR, PTR), PTR, 4, 2, None)  # no sequences: what is not refused does nothing
    rows, floats = Rows(dtype), Rows(torch.float32, (4, 2))
    yield lambda: remp.remp_kv_append(cache, batch, None, rows, rows, None, stream=1)
    yield lambda: remp.remp_kv_append(cache, batch, rows, rows, rows, rows, stream=1)
    yield lambda: remp.remp_kv_attend(cache, batch, rows, rows, 1.0, rows, stream=1)
    yield lambda: remp.remp_kv_weigh(cache, batch, rows, floats, Rows(torch.float32, (0, 2, 64)), 1.0, stream=1)


@pytest.mark.parametrize("held,given", [(torch.float16, torch.bfloat16), (torch.bfloat16, torch.float16)])
def test_rows_of_another_type(held, given):
    for call in calls(pool(held), given):
        with pytest.raises(remp.RempError) as e:
            call()
        assert e.value.status == remp.REMP_ERR_INVALID_ARG and str(held) in str(e.value)


@pytest.mark.parametrize("held,given", [(torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16), (torch.uint8, torch.float16), (torch.int16, torch.bfloat16)])
def test_rows_of_the_same_type_and_pools_of_bytes(held, given):
    for call in calls(pool(held), given):
        call()


@pytest.mark.parametrize("held", [torch.float32, torch.float64, torch.float8_e4m3fn])
def test_pools_of_other_numbers(held):
    with pytest.raises(remp.RempError):
        pool(held)


def test_pools_on_the_host():
    with pytest.raises(remp.RempError):
        remp.make_kv_pool(torch.zeros(8, dtype=torch.bfloat16), 8, 2, 128, 16)
