"""How many bits a probability keeps on its way to the values of a cache of 16-bit values: 16 and more for up to 64 rows of a sequence and
KV head (queries times query heads of a KV head), whatever other sequences of the batch have. Tolerances: test_kv_gpu, without
the half step that it allows for a probability in the cache's type (`few`); at most 1500 keys."""
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import HALF_STEP, Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("queries,hq,hk", [(17, 1, 1), (12, 4, 2), (25, 2, 2), (4, 16, 2)])
def test_up_to_32_rows_of_64_dims(dtype, queries, hq, hk):
    check(Case([queries, 40, 300, 1000], [queries, 1, queries, queries - 1], hk, 64, 16, dtype, seed=queries), hq, few=True)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("queries,hq,hk", [(17, 1, 1), (24, 1, 1), (4, 40, 8), (32, 2, 2), (33, 1, 1), (7, 14, 2), (9, 7, 1), (64, 1, 1), (1, 64, 1)])
def test_up_to_64_rows(d, dtype, queries, hq, hk):
    check(Case([queries, queries + 40, 300, 1000, 1], [queries, 1, queries, queries // 2, 0], hk, d, 16, dtype, seed=queries + d), hq, few=True)
    check(Case([queries + 40, 1400], [queries] * 2, hk, d, 32, dtype, seed=queries + d), hq, window=200, first=5, few=True)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_beside_those_of_a_prompt(d):
    """Sequences with few rows keep their bits in a batch with a prompt; so do the last few rows of a prompt."""
    c = Case([777, 1000, 33, 900], [1, 300, 1, 5], 2, d, 16, torch.bfloat16, seed=d)
    q, scale = c.queries(8), d ** -0.5
    out = torch.empty_like(q)
    remp.remp_kv_attend(c.pool, c.batch, q, out, scale, remp.make_kv_workspace())
    for s, (mine, want, _, weight, terms, _) in enumerate(c.exact(q, scale, 0, 0)):
        extra = HALF_STEP[torch.bfloat16] if s == 1 else 0.0
        tol = HALF_STEP[torch.bfloat16] * want.abs() + (2 * (terms * 2.0 ** -18 + 2.0 ** -20) + 2.0 ** -14 + extra) * weight + 2.0 ** -26
        assert ((out[mine].double() - want).abs() <= tol).all(), s


def test_keys_in_parts():
    for d in (64, 128, 256):
        check(Case([1500], [20], 1, d, 16, torch.bfloat16, seed=d), 2, few=True)
        check(Case([1500, 1200], [5, 3], 1, d, 16, torch.bfloat16, seed=d), 8, window=700, few=True)
