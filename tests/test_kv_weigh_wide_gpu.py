"""Weights of cached positions from many rows of a sequence against formulas in 64 bits (tolerances: test_kv_gpu)."""
import math

import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import Case, check_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("queries,hq,hk", [(33, 1, 1), (32, 8, 4), (64, 2, 2), (17, 7, 1), (128, 2, 1), (257, 1, 1), (40, 16, 2), (129, 32, 8)])
def test_rows(d, dtype, queries, hq, hk):
    lens = [queries, queries + 1, queries + 100, 700, 64, 0]
    check_weights(Case(lens, [queries, 1, queries, queries // 2, 0, 0], hk, d, 16, dtype, seed=queries + d), hq)


@pytest.mark.parametrize("window,first,fresh", [(1, 0, False), (20, 4, False), (20, 4, True), (128, 129, False), (300, 40, True), (0, 0, True), (2 ** 31 - 1, 3, False),
                                                (500, 200, False)])
@pytest.mark.parametrize("token_major", [False, True])
def test_windows(window, first, fresh, token_major):
    check_weights(Case([150, 1000, 40, 97], [150, 60, 0, 20], 2, 128, 32, torch.bfloat16, token_major=token_major, layers=2, layer=1), 8, window, first, fresh)


@pytest.mark.parametrize("bs", [16, 48, 256])
def test_blocks_and_a_pool_with_few_heads(bs):
    check_weights(Case([500, 300], [50, 300], 1, 128, bs, torch.float16), 2)
    check_weights(Case([1], [1], 1, 64, bs, torch.float16, spare=0), 64)


def test_long_sequences():
    check_weights(Case([20000, 50], [40, 40], 1, 64, 16, torch.bfloat16), 4)
    check_weights(Case([3000] * 40, [35] * 40, 4, 128, 16, torch.bfloat16), 4)


def test_bad_blocks_short_rows_and_rows_without_keys():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([300, 64], [40, 64], 2, 128, 16, torch.float16, error=word)
    c.tables[0, 2], c.tables[0, 9] = 10 ** 6, -1
    c.rebatch()
    check_weights(c, 4)
    assert int(word) == 8
    word.zero_()
    check_weights(Case([100, 60], [40, 60], 2, 128, 16, torch.float16, error=word), 4, stride=50)
    assert int(word) == 2
    c = Case([20, 90], [40, 1], 1, 64, 16, torch.bfloat16)
    q, got = c.queries(2), torch.full((2, 1, 90), 5.0, device="cuda")
    remp.remp_kv_weigh(c.pool, c.batch, q, torch.full((41, 2), -math.inf, device="cuda"), got, 1.0)
    assert (got[0, :, :20] == 0).all() and (got[0, :, 20:] == 5).all() and (got[1, :, 89] == 0).all() and (got[1, :, :89] == 5).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_slots_that_nobody_sees_hold_anything(bad):
    c = Case([300, 133], [40, 50], 2, 128, 16, torch.bfloat16)
    for s, n in enumerate(c.lens):
        for pos in range(c.tables.shape[1] * 16):
            block = c.tables[s, pos // 16]
            if block >= 0 and (pos >= n or 3 <= pos <= n - c.new[s] - 50):
                c.cache.slots(0, 0)[block, pos % 16] = bad
                c.cache.slots(0, 1)[block, pos % 16] = bad
    for fresh in (False, True):
        q, lse = c.queries(8), torch.empty(90, 8, device="cuda")
        remp.remp_kv_attend(c.pool, c.batch, q, torch.empty_like(q), 0.1, remp.make_kv_workspace(), window=50, first=3, lse=lse)
        got = torch.full((2, 2, 303), 1.0, device="cuda")
        remp.remp_kv_weigh(c.pool, c.batch, q, lse, got, 0.1, window=50, first=3, fresh=fresh)
        assert torch.isfinite(got).all()
        for s, n in enumerate(c.lens):
            hidden = got[s, :, 3:n - c.new[s] - 49]
            assert (hidden == (0.0 if fresh else 1.0)).all()


def test_the_same_every_time_and_rows_that_sum_to_one():
    c = Case([3000, 777], [40, 20], 2, 128, 16, torch.bfloat16)
    q, lse, outs = c.queries(4), torch.empty(60, 4, device="cuda"), []
    remp.remp_kv_attend(c.pool, c.batch, q, torch.empty_like(q), 0.1, remp.make_kv_workspace(), lse=lse)
    for _ in range(3):
        outs.append(torch.zeros(2, 2, 3000, device="cuda"))
        remp.remp_kv_weigh(c.pool, c.batch, q, lse, outs[-1], 0.1)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    # every query head's row sums to 1
    sums = torch.stack([outs[0][0].sum(-1), outs[0][1].sum(-1)]).double()
    want = torch.tensor([[80.0, 80.0], [40.0, 40.0]], device="cuda")
    assert ((sums - want).abs() <= want * 2.0 ** -14).all()


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([300, 100], [60, 60], 2, 128, 16, torch.bfloat16, error=word)
    q = c.queries(8)
    lse, got, good = torch.zeros(120, 8, device="cuda"), torch.zeros(2, 2, 300, device="cuda"), torch.zeros(2, 2, 300, device="cuda")
    remp.remp_kv_weigh(c.pool, c.batch, q, lse, good, 0.1, fresh=True)
    try:
        remp.remp_kvq_set_wait_limit(0)
        remp.remp_kv_weigh(c.pool, c.batch, q, lse, got, 0.1, fresh=True)
        torch.cuda.synchronize()
    finally:
        remp.remp_kvq_set_wait_limit(-1)
    assert int(word) == 16 and got[0].isnan().all() and got[1, :, :100].isnan().all()
    word.zero_()
    remp.remp_kv_weigh(c.pool, c.batch, q, lse, got, 0.1, fresh=True)
    got[1, :, 100:] = 0
    assert int(word) == 0 and torch.equal(got, good)
