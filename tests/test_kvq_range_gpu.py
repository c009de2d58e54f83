"""Attention over the 4-bit cache at the ends of the numbers' range, for one query token (up to 32 rows of a sequence and KV head) and
for prompts. Tolerances are test_kvq_prompt_gpu's, none of them absolute."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import test_kvq_gpu as base
from tests import test_kvq_prompt_gpu as prompt

pytestmark = pytest.mark.gpu

# few rows: 8 and 16 of them at a time; and one prompt
SHAPES = [(64, 2, 1, [70, 33], [1, 1]), (128, 8, 2, [200, 40], [1, 1]), (128, 10, 1, [200, 40], [2, 1]), (256, 4, 1, [90], [3]), (128, 4, 1, [90], [20])]


@pytest.mark.parametrize("size", [1e35, 1e30, 1e-30, 1e-35])
@pytest.mark.parametrize("d,hq,hk,lens,new", SHAPES)
def test_queries_and_keys_of_opposite_sizes(d, hq, hk, lens, new, size):
    prompt._range_case(d, hq, hk, lens, new, 1 / size, 1.0, size, seed=d + hq)


@pytest.mark.parametrize("size", [1e31, 1e35])
@pytest.mark.parametrize("d,n", [(64, 1), (128, 1), (128, 40), (256, 33)])
def test_scores_that_are_all_very_low(d, n, size):
    # far apart too: the highest takes it all
    rng = np.random.default_rng(d)
    lens, new, tables, start, batch = base._batch([100], [n], 16, 7, rng)
    pool = base._filled(7, 1, d, 16, rng)
    key = size / d / 1024 * 2.0 ** rng.permutation(np.arange(100) % 7)
    for p in range(100):
        pool.write(0, 0, tables[0, p // 16], p, np.full((1, d), -2.0 ** np.round(np.log2(key[p])), dtype=np.float32))
    buf, dev = base._dev_pool(pool)
    q = torch.full((n, 1, d), 1024.0, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(n, 1, device="cuda")
    remp.remp_kvq_attend(dev, batch, q, out, 1.0, remp.make_kvq_workspace(), lse=lse)
    k, v = (pool.rows(0, kv, tables[0], 100) for kv in (0, 1))
    want, want_lse, _, size, _ = base.ref.attend(q.double().cpu().numpy(), k, v, 100 - n, 1.0, 0)
    assert (want_lse < -1e30).all()
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= 2.0 ** -9 * np.abs(want) + 2.0 ** -10 * size[..., None]).all()
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= 2e-5 * np.abs(want_lse)).all()


@pytest.mark.parametrize("size", [1e-5, 1e-10, 1e-12, 1e-14, 1e7, 1e18])
@pytest.mark.parametrize("d,hq,hk,lens,new", SHAPES)
def test_values_of_any_size(d, hq, hk, lens, new, size):
    prompt._range_case(d, hq, hk, lens, new, 1.0, size, 1.0, seed=d + hq)


def test_values_without_a_step():
    # groups of one value: the step is 0, and only the minimum counts
    rng = np.random.default_rng(1)
    lens, new, tables, start, batch = base._batch([300], [1], 16, 19, rng)
    for size in (2.0 ** 60, 1.0, 2.0 ** -60):
        pool = base._filled(19, 1, 128, 16, rng)
        for p in range(300):
            pool.write(0, 1, tables[0, p // 16], p, np.full((1, 128), size * (1 + p % 3), dtype=np.float32))
        buf, dev = base._dev_pool(pool)
        q = torch.randn(1, 4, 128, device="cuda").bfloat16()
        out, lse = torch.empty_like(q), torch.empty(1, 4, device="cuda")
        remp.remp_kvq_attend(dev, batch, q, out, 128 ** -0.5, remp.make_kvq_workspace(), lse=lse)
        prompt._check_range(out, lse, q, pool, lens, new, tables, 128 ** -0.5)
