"""Calls on the 4-bit cache at the edges of their arguments: windows as large as an int, positions before the sequence, workspaces and
streams, rows with strides of 0."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import test_kvq_gpu as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4])
@pytest.mark.parametrize("d,hq,hk,lens,new", [(128, 4, 1, [3, 40, 0], [5, 5, 2]), (128, 8, 1, [20, 70], [40, 12]), (256, 2, 2, [9], [60])])
def test_attend_largest_window(d, hq, hk, lens, new, window):
    # sequences with more queries than tokens among them: their first rows stand before position 0
    base._attend_case(d, hq, hk, 16, torch.bfloat16, lens, new, window=window, seed=d)


@pytest.mark.parametrize("hq,lens,new,bits", [(4, [3, 40], [5, 1], 2), (4, [40, 0], [1, 1], 2), (8, [3, 90], [5, 40], 2), (8, [80, 90], [1, 40], 0),
                                              (4, [40, 0, 7], [1, 0, 7], 0)])
def test_attend_reports_positions_before_the_sequence(hq, lens, new, bits):
    rng = np.random.default_rng(0)
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, new, tables, start, batch = base._batch(lens, new, 16, 20, rng, error=error)
    pool = base._filled(20, 1, 128, 16, rng)
    buf, dev = base._dev_pool(pool)
    q = torch.randn(int(start[-1]), hq, 128, device="cuda").bfloat16()
    out = torch.empty_like(q)
    remp.remp_kvq_attend(dev, batch, q, out, 128 ** -0.5, remp.make_kvq_workspace())
    base._check(out, None, q, pool, 0, lens, new, tables, 128 ** -0.5, 0, torch.bfloat16)
    assert int(error) == bits


def test_workspace_is_ready_for_any_stream():
    x = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x @ x
        ws = remp.make_kvq_workspace()
        assert side.query()  # zeroed, whichever stream comes next
    assert not ws.any()


def test_rows_repeated_by_strides_of_zero():
    # inputs that are broadcast: one key for all heads, one value for all tokens, one query for all heads
    rng = np.random.default_rng(4)
    d, hk, n = 128, 4, 6
    lens, new, tables, start, batch = base._batch([20, 9], [4, 2], 16, 4, rng)
    k, v, q = (torch.randn(*s, d, device="cuda").bfloat16() for s in ((n, 1), (1, hk), (n, 1)))
    wide = [k.expand(n, hk, d), v.expand(n, hk, d), q.expand(n, 2 * hk, d)]
    outs = []
    for kk, vv, qq in (wide, [x.contiguous() for x in wide]):
        p = base.ref.Pool(1, 4, hk, d, 16)
        buf, dev = base._dev_pool(base._filled(4, hk, d, 16, np.random.default_rng(1)))
        turned, out = torch.empty(n, 2 * hk, d, dtype=k.dtype, device="cuda"), torch.empty(n, 2 * hk, d, dtype=k.dtype, device="cuda")
        remp.remp_kvq_append(dev, batch, qq, kk, vv, turned)
        remp.remp_kvq_attend(dev, batch, qq, out, d ** -0.5, remp.make_kvq_workspace())
        outs.append((buf, turned, out))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_strides_of_single_heads_and_tokens_do_not_matter():
    rng = np.random.default_rng(5)
    d = 64
    lens, new, tables, start, batch = base._batch([20], [1], 16, 2, rng)
    buf, dev = base._dev_pool(base._filled(2, 1, d, 16, rng))
    row = torch.randn(d, device="cuda").bfloat16()
    odd = row.as_strided((1, 1, d), (3, 5, 1))  # what slices of padded tensors can look like
    out = torch.zeros(d, dtype=row.dtype, device="cuda")
    remp.remp_kvq_append(dev, batch, odd, odd, odd, out.as_strided((1, 1, d), (3, 5, 1)))
    assert torch.equal(out, row)
