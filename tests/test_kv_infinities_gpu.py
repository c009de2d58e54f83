"""Attention over a cache of 16-bit values: an infinity in V reaches the rows that see it as an infinity of its sign, two of both signs
as NaN, and only in its own dim."""
import math

import pytest
import torch

from tests.test_kv_gpu import Case
from tests.test_kv_values_gpu import ROWS, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("queries,hq,hk", ROWS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_infinities_that_every_row_sees(queries, hq, hk, d, dtype):
    lens = [queries, 30 + queries, 700]
    c = Case(lens, [queries] * 3, hk, d, 16, dtype, seed=queries + d)
    q, v = c.queries(hq), c.cache.slots(0, 1)
    # dims 3, 5 and 7 are 0 first: what the others give must stay
    v[..., 3], v[..., 5], v[..., 7] = 0, 0, 0
    want, want_lse = attend(c, q)
    for s, n in enumerate(lens):
        v[c.tables[s, 0], 0, :, 3] = math.inf
        v[c.tables[s, 0], 0, :, 5] = -math.inf
        if s:
            v[c.tables[s, 0], 0, :, 7] = math.inf
            v[c.tables[s, 1], 7, :, 7] = -math.inf
    out, lse = attend(c, q)
    assert (out[..., 3] == math.inf).all() and (out[..., 5] == -math.inf).all()
    assert (out[:queries, :, 7] == 0).all() and out[queries:, :, 7].isnan().all()
    others = [i for i in range(d) if i not in (3, 5, 7)]
    assert torch.equal(out[..., others], want[..., others]) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_probabilities_that_are_powers_of_two(dtype):
    """Scores of 0: a probability is one number of the cache's type, and nothing is left of it for a second."""
    for queries, hq in ((1, 8), (2, 8), (3, 8), (5, 8), (20, 8)):
        for d in (64, 128, 256):
            c = Case([500], [queries], 1, d, 16, dtype)
            c.cache.data[:, 0] = 0
            v = c.cache.slots(0, 1)
            v[c.tables[0, 1], 3] = math.inf
            v[c.tables[0, 2], 5, :, 0::2] = math.inf
            v[c.tables[0, 2], 5, :, 1::2] = -math.inf
            out, _ = attend(c, c.queries(hq))
            assert (out[..., 0::2] == math.inf).all() and out[..., 1::2].isnan().all()


@pytest.mark.parametrize("dtype,score", [(torch.bfloat16, -48.0), (torch.float16, -20.0)])
def test_probabilities_far_below_the_largest(dtype, score):
    """2^-69 and 2^-29 of it: still above 0 as two numbers of the cache's type."""
    for queries, hq in ((1, 8), (2, 8), (5, 8), (20, 8)):
        for d in (64, 128, 256):
            c = Case([300], [queries], 1, d, 16, dtype)
            c.cache.data[:, 0] = 0
            k, v, block, q = c.cache.slots(0, 0), c.cache.slots(0, 1), c.tables[0, 2], torch.zeros_like(c.queries(hq))
            q[..., 0] = 4.0
            k[block, 5, :, 0] = score / 4 * d ** 0.5
            v[block, 5, :, 0::2] = math.inf
            out, _ = attend(c, q)
            assert (out[..., 0::2] == math.inf).all() and torch.isfinite(out[..., 1::2]).all()
