"""Attention of many queries over a cache of 16-bit values against formulas in 64 bits (tolerances: test_kv_gpu)."""
import math

import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("queries,hq,hk", [(17, 1, 1), (128, 2, 2), (129, 1, 1), (33, 8, 1), (256, 4, 4), (300, 7, 1), (64, 32, 2)])
def test_rows(d, dtype, queries, hq, hk):
    check(Case([queries, queries + 1, queries + 200, 900, 41], [queries, 1, queries, queries // 2, 0], hk, d, 16, dtype, seed=queries + d), hq)


@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (16, 3), (100, 4), (127, 128), (128, 129), (129, 300), (500, 4), (64, 1000), (1000, 0),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("d", [128, 256])
def test_windows_and_first_tokens(window, first, d):
    check(Case([200, 1500, 333, 150], [200, 130, 1, 150], 2, d, 16, torch.bfloat16, seed=window % 89), 4, window=window, first=first)


@pytest.mark.parametrize("bs", [16, 32, 48, 112, 256])
@pytest.mark.parametrize("token_major", [False, True])
def test_blocks_and_orders(bs, token_major):
    check(Case([500, 77, 130], [60, 77, 20], 3, 128, bs, torch.bfloat16, token_major=token_major, layers=2, layer=1), 6)
    check(Case([500, 77, 130], [60, 77, 20], 3, 64, bs, torch.float16, token_major=token_major), 3, window=70, first=20)


@pytest.mark.parametrize("lens,queries,hq,hk", [([9000], 20, 1, 1), ([5000], 3, 16, 2), ([700] * 90, 18, 2, 2), ([4000, 40], 300, 4, 1), ([20000], 1, 32, 1)])
def test_keys_in_parts(lens, queries, hq, hk):
    """Units that share the GPU: few of them, and a few more than fill it."""
    for d in (64, 128, 256):
        check(Case(lens, [min(queries, n) for n in lens], hk, d, 16, torch.bfloat16, seed=d), hq)


def test_prompts_from_nothing_and_behind_text():
    check(Case([1000, 2100, 1], [1000, 700, 1], 2, 128, 16, torch.bfloat16), 16)
    check(Case([1000, 2100, 1], [1000, 700, 1], 2, 128, 16, torch.float16), 16, window=300, first=4)


def test_rows_before_the_first_position_and_bad_blocks():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([20, 300, 0], [50, 90, 3], 2, 128, 16, torch.bfloat16, error=word)
    _, out, lse = check(c, 4)
    assert int(word) == 2 and (out[:30] == 0).all() and (lse[:30] == -math.inf).all()
    word.zero_()
    c = Case([200, 300], [40, 90], 2, 128, 16, torch.bfloat16, error=word)
    c.tables[0, 2], c.tables[1, 0], c.tables[1, 18] = 10 ** 6, -5, 2 ** 31 - 1
    c.rebatch()
    check(c, 4)
    assert int(word) == 8


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_slots_that_nobody_sees_hold_anything(bad):
    c = Case([300, 133], [30, 20], 2, 128, 16, torch.bfloat16)
    window, first = 50, 3
    for s, (n, m) in enumerate(zip(c.lens, c.new)):
        for pos in range(c.tables.shape[1] * 16):
            block = c.tables[s, pos // 16]
            if block >= 0 and (pos >= n or first <= pos <= n - m - window):
                c.cache.slots(0, 0)[block, pos % 16] = bad
                c.cache.slots(0, 1)[block, pos % 16] = bad
    check(c, 8, window=window, first=first)


def test_references_that_move():
    """Scores that grow along the keys, and rows of very different sizes."""
    c = Case([1500, 400], [100, 60], 1, 128, 16, torch.bfloat16)
    for s, n in enumerate(c.lens):
        for pos in range(int(n)):
            c.cache.slots(0, 0)[c.tables[s, pos // 16], pos % 16] *= 0.2 + 4 * pos / int(n)
    q = c.queries(4)
    q *= torch.logspace(-3, 1, 160, device="cuda")[torch.randperm(160, device="cuda")][:, None, None].bfloat16()
    check(c, 4, q=q)
    check(c, 4, size=30.0)


def test_strides_of_rows():
    c = Case([50, 70], [30, 70], 2, 128, 16, torch.bfloat16)
    wide = torch.randn(100, 3, 8, 160, generator=c.gen, device="cuda").bfloat16()
    out = torch.full((100, 8, 160), 3.0, device="cuda", dtype=torch.bfloat16)
    check(c, 4, q=wide[:, 1, 2:6, 16:144], out=out[:, 1:5, 16:144])
    assert (out[:, 0] == 3).all() and (out[:, 5:] == 3).all() and (out[..., :16] == 3).all() and (out[..., 144:] == 3).all()
    check(c, 4, q=wide[:1, 0, :4, :128].expand(100, 4, 128))


def test_results_do_not_depend_on_the_run():
    c = Case([3000, 10, 777], [40, 10, 20], 2, 128, 16, torch.bfloat16)
    q, w, outs = c.queries(16), remp.make_kv_workspace(), []
    for _ in range(3):
        out = torch.empty_like(q)
        remp.remp_kv_attend(c.pool, c.batch, q, out, 0.1, w)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("lens,queries", [([300, 100], 60), ([5000], 40)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(lens, queries):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case(lens, [queries] * len(lens), 2, 128, 16, torch.bfloat16, error=word)
    q, w = c.queries(8), remp.make_kv_workspace()
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
