"""Calls on the 4-bit cache at the edges of their arguments: windows as large as an int, positions before the sequence, workspaces and
streams."""
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
