"""Appending many tokens to the 4-bit cache: from 20 tokens for each SM on a warp takes a whole token, group of heads by group, and
above 160 a warp takes several tokens. Bytes and queries are compared exactly, as in test_kvq_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import test_kvq_gpu as base

pytestmark = pytest.mark.gpu


def _lengths(total, seqs, seed):
    """Prompts of uneven lengths that add up to `total`, some with tokens before them."""
    rng = np.random.default_rng(seed)
    cut = np.sort(rng.choice(np.arange(1, total), seqs - 1, replace=False))
    new = np.diff(np.concatenate([[0], cut, [total]]))
    return new + rng.integers(0, 30, seqs) * (rng.random(seqs) < 0.5), new


@pytest.mark.parametrize("d,hq,hk", [(64, 40, 18), (128, 20, 10), (128, 3, 1), (256, 9, 5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("norm,rotary,interleaved", [(True, 1.0, False), (True, 0.5, True), (False, 0.25, False)])
def test_append_prompts(d, hq, hk, dtype, norm, rotary, interleaved):
    lens, new = _lengths(3300, 9, d + hq)
    base._append_case(d, hq, hk, 16, dtype, norm, int(d * rotary), interleaved, lens, new, d + hq)


def test_append_more_tokens_than_warps():
    lens, new = _lengths(25000, 40, 1)
    base._append_case(64, 2, 1, 32, torch.bfloat16, True, 64, False, lens, new, 1)


def test_append_more_groups_than_warps():
    lens, new = _lengths(2900, 5, 2)
    base._append_case(256, 30, 2, 16, torch.float16, True, 128, True, lens, new, 2)


@pytest.mark.parametrize("d,h", [(64, 33), (128, 9), (256, 9)])
def test_append_prompts_in_place(d, h):
    lens, new = _lengths(3300, 7, d)
    lens, new, tables, start, batch = base._batch(lens, new, 16, int((-(-lens // 16)).sum()), np.random.default_rng(d))
    pool = base.ref.Pool(1, int((-(-lens // 16)).sum()), h, d, 16)
    (b1, d1), (b2, d2) = base._dev_pool(pool), base._dev_pool(pool)
    x = torch.randn(3300, 3 * h, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).bfloat16()
    rope = torch.from_numpy(base._rope(int(lens.max()), d, np.random.default_rng(1))).cuda()
    w = torch.rand(d, device="cuda") + 0.5
    apart, y = torch.empty(3300, h, d, dtype=x.dtype, device="cuda"), x.clone()
    remp.remp_kvq_append(d1, batch, x[:, :h], x[:, h:2 * h], x[:, 2 * h:], apart, q_norm=w, k_norm=w, rope=rope)
    remp.remp_kvq_append(d2, batch, y[:, :h], y[:, h:2 * h], y[:, 2 * h:], y[:, :h], q_norm=w, k_norm=w, rope=rope)
    assert torch.equal(b1, b2) and torch.equal(y[:, :h], apart) and torch.equal(y[:, h:], x[:, h:])
