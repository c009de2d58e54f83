"""Pages between the first tokens and the window, which no row of a call sees, may be given back: what the table names there is not looked
at, by few rows and by many, and not reported."""
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests.test_kv_gpu import Case

pytestmark = pytest.mark.gpu

# queries, query heads, KV heads: 8 to 320 rows
ROWS = [(1, 8, 1), (2, 16, 2), (4, 16, 2), (5, 8, 1), (20, 16, 2), (40, 8, 1)]


@pytest.mark.parametrize("window,first", [(50, 4), (20, 0), (130, 17), (300, 129), (1, 16)])
@pytest.mark.parametrize("bs", [16, 48])
@pytest.mark.parametrize("queries,hq,hk", ROWS)
@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1])
def test_pages_that_no_row_sees(window, first, bs, queries, hq, hk, bad):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = [900, 260 + queries, 20 + queries, queries]
    c = Case(lens, [queries] * 4, hk, 128, bs, torch.bfloat16, error=word, seed=window)
    q, scale, positions = c.queries(hq), 0.1, 907

    def calls():
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        remp.remp_kv_attend(c.pool, c.batch, q, out, scale, remp.make_kv_workspace(), window=window, first=first, lse=lse)
        assert int(word) == 0, "attention"
        added = []
        for fresh in (False, True):
            weights = torch.full((4, hk, positions), 1.5, device="cuda")
            remp.remp_kv_weigh(c.pool, c.batch, q, lse, weights, scale, window=window, first=first, fresh=fresh)
            assert int(word) == 0, "weights"
            added.append(weights)
        return out, lse, *added

    want = calls()
    hidden = 0
    for s, n in enumerate(lens):
        for i in range(c.tables.shape[1]):
            if i * bs >= n or (i * bs >= first and (i + 1) * bs <= n - queries - window + 1):
                hidden += i * bs < n
                c.tables[s, i] = bad
    assert hidden > 0
    c.rebatch()
    for got, old in zip(calls(), want):
        assert torch.equal(got, old)


def test_pages_that_some_row_sees_are_reported():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    for queries, hq in ((1, 8), (5, 8), (20, 8)):
        for at in (0, (600 - queries - 50 + 1) // 16, 599 // 16):
            c = Case([600], [queries], 1, 128, 16, torch.bfloat16, error=word)
            c.tables[0, at] = -1
            c.rebatch()
            q, lse = c.queries(hq), torch.zeros(queries, hq, device="cuda")
            remp.remp_kv_attend(c.pool, c.batch, q, torch.empty_like(q), 0.1, remp.make_kv_workspace(), window=50, first=4)
            assert int(word) == 8
            for fresh in (False, True):
                word.zero_()
                remp.remp_kv_weigh(c.pool, c.batch, q, lse, torch.zeros(1, 1, 600, device="cuda"), 0.1, window=50, first=4, fresh=fresh)
                assert int(word) == 8
            word.zero_()
