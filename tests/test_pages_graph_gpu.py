"""Page management inside a CUDA graph: one launch, and the steps that take scratch from the library's pool."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200.synth import Shape, Topo
from tests import kvq_reference as ref
from tests import test_pages_gpu as pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kids,max_len,spare", [(10, 12, 100, 30), (64, 300, 900, 4000)])
def test_fork_free_compact_and_copy_in_a_graph(n, kids, max_len, spare):
    bs = 16
    rng, lens, tables, refs, blocks = pages._state(n, kids, max_len, bs, spare, n)
    parents, children = rng.integers(0, n, kids).astype(np.int32), (n + rng.permutation(kids)).astype(np.int32)
    done = (rng.random(n + kids) < 0.5).astype(np.int32)
    T, m = Topo(2, 1), Shape(2, 2, 16, bs, 2)
    start = [torch.randint(0, 256, (remp.remp_shard_bytes(T, m, r, blocks),), dtype=torch.uint8, device="cuda") for r in range(2)]
    # the plain statement
    l1, t1, r1, p1, res1 = ref.fork(lens, tables, bs, parents, children, refs)
    l2, t2, r2, res2 = ref.free(l1, t1, bs, done, r1)
    t3, r3, p3, res3 = ref.compact(l2, t2, bs, r2, blocks // 2)
    pools = [b.cpu().numpy().reshape(2, 2, blocks, -1).copy() for b in start]
    for b in pools:
        for pairs, count in ((p1, res1[0]), (p3, res3[0])):
            b[:, :, pairs[:count, 1]] = b[:, :, pairs[:count, 0]]
    # the calls, once captured and replayed on fresh inputs
    dl, dt, dr = pages._d(lens), pages._d(tables), pages._d(refs)
    par, chi, fin = pages._d(parents), pages._d(children), pages._d(done)
    pairs, moves = torch.empty(kids, 2, dtype=torch.int32, device="cuda"), torch.empty(blocks // 2, 2, dtype=torch.int32, device="cuda")
    results = [torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(3)]
    bufs = [b.clone() for b in start]
    shards = remp.make_shards(bufs, [blocks] * 2)

    def calls():
        remp.remp_pages_fork(dl, dt, bs, par, chi, dr, dr, pairs, results[0])
        remp.remp_pages_copy(T, m, shards, pairs, results[0])
        remp.remp_pages_free(dl, dt, bs, fin, dr, dl, dt, dr, results[1])
        remp.remp_pages_compact(dl, dt, bs, dr, dt, dr, moves, results[2])
        remp.remp_pages_copy(T, m, shards, moves, results[2])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        for x, y in ((dl, lens), (dt, tables), (dr, refs)):
            x.copy_(pages._d(y))
        for x, y in zip(bufs, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in ((dl, l2), (dt, t3), (dr, r3), (pairs, p1), (moves, p3)):
            assert np.array_equal(got.cpu().numpy(), want)
        assert [r.tolist() for r in results] == [res1, res2, res3]
        for got, want in zip(bufs, pools):
            assert np.array_equal(got.cpu().numpy().reshape(want.shape), want)


FIRST = """
import torch, paper_2606_18741_b200 as remp
n, width, blocks = 200, 30, 6000
i = dict(dtype=torch.int32, device="cuda")
lens, tables = torch.full((n,), width * 16, **i), torch.arange(n * width, **i).view(n, width).contiguous()
refs, pairs, result = torch.ones(blocks, **i), torch.empty(blocks // 2, 2, **i), torch.empty(2, **i)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    remp.remp_pages_compact(lens, tables, 16, refs, tables, refs, pairs, result)
result.fill_(-9)
graph.replay()
assert result.tolist() == [0, 0]
"""


def test_first_call_of_a_program_in_a_capture():
    # the library's pool is made in it
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
