"""Many short sequences with more than 16 rows each (more than 24 for weights): the kernels for few rows take them row block by row block,
and keep 16 bits of a probability whatever the rows (`few`). Tolerances: test_kv_gpu."""
import math

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import Case, check, check_weights

pytestmark = pytest.mark.gpu


def short(heads, d, dtype, longest, most, seed=0, **kw):
    """As many sequences as fill the GPU, of 0 to `longest` tokens and 0 to `most` new ones."""
    rng = np.random.default_rng(seed)
    n = torch.cuda.get_device_properties(0).multi_processor_count // heads + 2
    lens = rng.integers(0, longest + 1, n)
    lens[0] = longest
    new = np.minimum(rng.integers(0, most + 1, n), lens)
    new[0] = min(most, longest)
    return Case(lens, new, heads, d, 16, dtype, seed=seed, **kw)


@pytest.mark.parametrize("d,longest,most", [(64, 200, 9), (64, 70, 17), (128, 200, 8), (128, 60, 20), (256, 90, 7), (256, 30, 12)])
@pytest.mark.parametrize("hq,hk", [(8, 2), (5, 1), (4, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention(d, longest, most, hq, hk, dtype):
    c = short(hk, d, dtype, longest, most, seed=d + hq)
    check(c, hq, few=True)
    check(c, hq, window=33, first=2, few=True)


@pytest.mark.parametrize("d,longest,most", [(64, 120, 9), (128, 200, 8), (128, 40, 30), (256, 90, 7)])
@pytest.mark.parametrize("hq,hk", [(8, 2), (5, 1)])
@pytest.mark.parametrize("fresh", [False, True])
def test_weights(d, longest, most, hq, hk, fresh):
    c = short(hk, d, torch.bfloat16, longest, most, seed=d + hq)
    check_weights(c, hq, fresh=fresh)
    check_weights(c, hq, window=33, first=2, fresh=fresh)


def test_a_table_that_names_longer_sequences():
    """The host sees the table's width only; another kernel, the same results within the tolerance."""
    for width in (None, 100):
        check(short(2, 128, torch.bfloat16, 60, 8, width=width), 8, few=True)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_up_to_64_rows_before_the_first_position(d):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([5, 40, 0, 1], [40, 60, 3, 33], 2, d, 16, torch.bfloat16, error=word)
    _, out, lse = check(c, 2, few=True)
    assert int(word) == 2 and (out[:35] == 0).all() and (lse[:35] == -math.inf).all() and (out[100:103] == 0).all() and (out[103:135] == 0).all()


@pytest.mark.parametrize("lens,queries", [([300, 100], 10), ([1500], 5)])
def test_a_wait_of_up_to_64_rows_that_runs_out_is_reported_and_the_next_call_is_right(lens, queries):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case(lens, [queries] * len(lens), 2, 128, 16, torch.bfloat16, error=word)
    q, w = c.queries(12), remp.make_kv_workspace()
    good, out = torch.empty_like(q), torch.empty_like(q)
    remp.remp_kv_attend(c.pool, c.batch, q, good, 0.1, w)
    try:
        remp.remp_kvq_set_wait_limit(0)
        remp.remp_kv_attend(c.pool, c.batch, q, out, 0.1, w)
        torch.cuda.synchronize()
    finally:
        remp.remp_kvq_set_wait_limit(-1)
    assert int(word) == 16 and out.isnan().all()
    word.zero_()
    remp.remp_kv_attend(c.pool, c.batch, q, out, 0.1, w)
    assert int(word) == 0 and torch.equal(out, good)
