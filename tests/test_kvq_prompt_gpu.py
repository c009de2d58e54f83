"""Attention of prompts over the 4-bit cache: what the matrix kernel does when a wait runs out, when a thread block walks many
blocks of keys, and at the ends of the numbers' range. Helpers and tolerances are those of test_kvq_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import test_kvq_gpu as base

pytestmark = pytest.mark.gpu


@pytest.fixture
def wait_limit():
    yield remp.remp_kvq_set_wait_limit
    torch.cuda.synchronize()
    remp.remp_kvq_set_wait_limit(-1)


# (head_dim, query heads, KV heads, lengths, query tokens): units of several blocks of keys, one and two matrices; one unit in parts
WAITS = [(128, 32, 32, [400] * 12, [40] * 12), (64, 24, 24, [300] * 8, [200] * 8), (256, 20, 20, [330] * 9, [35] * 9), (128, 1, 1, [900], [200])]


@pytest.mark.parametrize("d,hq,hk,lens,new", WAITS)
@pytest.mark.parametrize("tries", [0, 1, 2])
def test_a_wait_that_runs_out_gives_nan_and_is_reported(wait_limit, d, hq, hk, lens, new, tries):
    rng = np.random.default_rng(d)
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    blocks = int((-(-np.asarray(lens) // 16)).sum())
    lens, new, tables, start, batch = base._batch(lens, new, 16, blocks, rng, error=error)
    buf, pool = base._dev_pool(base._filled(blocks, hk, d, 16, rng))
    q = torch.randn(int(start[-1]), hq, d, device="cuda").bfloat16()
    ws = remp.make_kvq_workspace()
    want, got, again = (torch.full_like(q, 7.0) for _ in range(3))
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    remp.remp_kvq_attend(pool, batch, q, want, d ** -0.5, ws)
    assert int(error) == 0 and torch.isfinite(want).all()
    wait_limit(tries)
    remp.remp_kvq_attend(pool, batch, q, got, d ** -0.5, ws, lse=lse)
    torch.cuda.synchronize()
    bad = torch.isnan(got)
    assert torch.equal(bad.any(-1), bad.all(-1)) and torch.equal(bad.any(-1), torch.isnan(lse))
    assert torch.equal(got[~bad], want[~bad])  # a row is right or NaN
    assert int(error) in ((16,) if bad.any() else (0, 16))
    if tries == 0:
        assert bad.all()
    # the workspace is as it was, and the limit too
    wait_limit(-1)
    error.zero_()
    remp.remp_kvq_attend(pool, batch, q, again, d ** -0.5, ws)
    assert torch.equal(again, want) and int(error) == 0
