"""Attention over a cache of 16-bit values: values V of any size, for few and for many rows of a sequence. Probabilities and sums are
scaled by powers of two, so a V scaled by one gives outputs scaled by it, bit for bit, as long as nothing overflows or falls
below the normal numbers of 32 bits; and a mean of equal values is that value."""
import math

import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import Case

pytestmark = pytest.mark.gpu

# queries of a sequence, query heads, KV heads: 8, 16, 24, 40, 160 and 320 rows
ROWS = [(1, 8, 1), (2, 16, 2), (3, 8, 1), (5, 8, 1), (20, 16, 2), (40, 8, 1)]


def attend(c, q, window=0, first=0):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    remp.remp_kv_attend(c.pool, c.batch, q, out, c.d ** -0.5, remp.make_kv_workspace(), window=window, first=first, lse=lse)
    return out, lse


@pytest.mark.parametrize("queries,hq,hk", ROWS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_outputs_follow_the_size_of_the_values(queries, hq, hk, d):
    for lens in ([queries, queries + 1, 100 + queries, 900], [9001]):
        c = Case(lens, [queries] * len(lens), hk, d, 16, torch.bfloat16, seed=queries + d)
        q, v = c.queries(hq), c.cache.data[:, 1].clone()
        assert float(v.abs().max()) < 64
        want, _ = attend(c, q)
        for power in (-60, 60, 121):
            c.cache.data[:, 1] = v * 2.0 ** power
            assert torch.equal(attend(c, q)[0], want * 2.0 ** power), power


@pytest.mark.parametrize("queries,hq,hk", ROWS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_mean_of_equal_values_is_that_value(queries, hq, hk, d, dtype):
    """Scores of 0 give probabilities that are equal powers of two."""
    most = torch.finfo(dtype).max
    lens = [queries, 40 + queries, 5000]
    c = Case(lens, [queries] * 3, hk, d, 16, dtype)
    c.cache.data[:, 0] = 0
    c.cache.data[:, 1] = most
    c.cache.data[:, 1, ..., 1::2] = -most
    out, lse = attend(c, c.queries(hq))
    assert (out[..., 0::2] == most).all() and (out[..., 1::2] == -most).all()
    seen = torch.cat([torch.arange(n - queries + 1, n + 1) for n in lens]).cuda().double()
    assert ((lse.double() - seen.log()[:, None]).abs() <= 2.0 ** -18 + 2.0 ** -22 * seen.log()[:, None]).all()


def test_scores_that_rise_by_much_and_large_values():
    """The reference moves from block to block; V is as large as its type allows."""
    for queries, hq in ((1, 8), (2, 8), (5, 8), (40, 8)):
        c = Case([1500], [queries], 1, 128, 16, torch.bfloat16)
        for pos in range(1500):
            c.cache.slots(0, 0)[c.tables[0, pos // 16], pos % 16] *= 0.2 + 4 * pos / 1500
        q, v = c.queries(hq, 3.0), c.cache.data[:, 1].clamp(-1, 1).clone()
        c.cache.data[:, 1] = v
        want, _ = attend(c, q)
        c.cache.data[:, 1] = v * 2.0 ** 127
        assert torch.equal(attend(c, q)[0], want * 2.0 ** 127)
