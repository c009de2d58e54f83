"""Eviction from a cache of 16-bit values against plain sorting: whole numbers and copies, compared exactly."""
import math

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import kv_reference as ref
from tests.test_kv_gpu import Case

pytestmark = pytest.mark.gpu


def weights_of(kind, shape, rng):
    if kind == "heavy":
        return np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 3, shape).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, dtype=np.float32)
    x = rng.standard_normal(shape).astype(np.float32)  # everything that a float can be
    for value in (math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, 3e38, -3e38):
        x[rng.random(shape) < 0.06] = value
    return x


def check(lens, keep, heads, d, bs, first, recent, kind="heavy", dtype=torch.bfloat16, seed=0, in_place=False, token_major=False, kept_width=None, max_tokens=None,
          slack=3):
    rng = np.random.default_rng(seed)
    keep = np.full(len(lens), keep, dtype=np.int32) if np.isscalar(keep) else np.asarray(keep, dtype=np.int32)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case(lens, [0] * len(lens), heads, d, bs, dtype, seed=seed, token_major=token_major, layers=2, layer=1)
    longest = max(1, int(np.max(lens))) + slack
    host = weights_of(kind, (len(lens), heads, longest), rng)
    weights = torch.from_numpy(host).cuda()
    out = weights if in_place else torch.full_like(weights, 8.0)
    after = np.minimum(lens, keep)
    kept = torch.full((len(lens), heads, kept_width or max(1, int(after.max()))), 55, dtype=torch.int32, device="cuda")
    want = c.cache.data.clone()
    remp.remp_kv_evict(c.pool, c.dev_lens, c.dev_tables, torch.from_numpy(keep).cuda(), weights, out, kept, first=first, recent=recent, max_tokens=max_tokens,
                       error=word)
    got_kept, got_out = kept.cpu().numpy(), out.cpu().numpy()
    model = ref.Cache.__new__(ref.Cache)
    model.__dict__.update(c.cache.__dict__, data=want)
    for s, n in enumerate(lens):
        table = c.dev_tables[s].long()
        for h in range(heads):
            stay = ref.choose(host[s, h], int(n), int(keep[s]), first, recent)
            assert got_kept[s, h, :len(stay)].tolist() == stay, (s, h)
            assert (got_kept[s, h, len(stay):] == -1).all()
            assert np.array_equal(got_out[s, h, :len(stay)].view(np.uint32), host[s, h, stay].view(np.uint32))
            rest = host[s, h, len(stay):] if in_place else np.full(longest - len(stay), 8.0, dtype=np.float32)
            assert np.array_equal(got_out[s, h, len(stay):].view(np.uint32), rest.astype(np.float32).view(np.uint32))
            source, to = torch.tensor(stay, dtype=torch.long, device="cuda"), torch.arange(len(stay), device="cuda")
            for kv in (0, 1):
                x = model.slots(1, kv)
                x[table[to // bs], to % bs, h] = x[table[source // bs], source % bs, h]
    assert torch.equal(c.cache.data.view(torch.int16), want.view(torch.int16))
    assert int(word) == 0


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "any"])
@pytest.mark.parametrize("first,recent", [(0, 0), (4, 16), (1, 0), (0, 9), (1000, 3), (30, 1000)])
def test_choice_and_move(kind, first, recent):
    check([100, 1, 64, 65, 0, 40, 333, 41], 40, 2, 64, 16, first, recent, kind, in_place=kind == "any")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("token_major", [False, True])
def test_rows(d, dtype, token_major):
    check([257, 90, 511], [100, 89, 300], 3, d, 32, 4, 16, dtype=dtype, token_major=token_major, in_place=token_major)


@pytest.mark.parametrize("keep", [0, 1, 2, 99, 100, 101])
def test_budgets(keep):
    check([100, 100, 7], keep, 2, 128, 16, 1, 1)
    check([100, 100, 7], [keep, 50, 3], 1, 64, 48, 0, 0, kept_width=120)


@pytest.mark.parametrize("length,keep", [(4096, 4095), (4097, 1000), (5000, 17), (16384, 9000), (16385, 16000), (50001, 2048), (131072, 70000), (131073, 100)])
@pytest.mark.parametrize("kind", ["heavy", "ties"])
def test_long_sequences(length, keep, kind):
    check([length, 100], keep, 1, 64, 64, 4, 100, kind, slack=0)


def test_many_sequences():
    rng = np.random.default_rng(5)
    check(rng.integers(0, 300, 150).tolist(), rng.integers(0, 300, 150).tolist(), 2, 64, 16, 2, 8)


def test_kernel_is_chosen_by_max_tokens_and_gives_the_same():
    for most in (300, 5000, 20000, 200000):
        check([300, 123, 299], 100, 2, 64, 16, 4, 8, "ties", slack=200000, max_tokens=most)


def test_errors_leave_a_sequence_as_it_is():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([50, 60, 70, 80, 90], [0] * 5, 1, 64, 16, torch.bfloat16)
    c.lens[0], c.lens[3] = -1, 1000  # negative; beyond its row and the weights
    c.rebatch()
    weights = torch.rand(5, 1, 90, device="cuda")
    out, kept = torch.full_like(weights, 3.0), torch.full((5, 1, 30), 7, dtype=torch.int32, device="cuda")
    before = c.cache.data.clone()
    keep = torch.tensor([10, -2, 31, 10, 20], dtype=torch.int32, device="cuda")  # the third: more than `kept` holds
    remp.remp_kv_evict(c.pool, c.dev_lens, c.dev_tables, keep, weights, out, kept, error=word)
    assert int(word) == 2
    assert (kept[:4] == -1).all() and (out[:4] == 3).all() and (kept[4, 0, :20] >= 0).all()
    own = torch.from_numpy(c.tables[4, :6]).cuda().long()
    c.cache.data[:, :, own] = 0
    before[:, :, own] = 0
    assert torch.equal(c.cache.data, before)


def test_blocks_outside_the_pool_lose_their_rows_only():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([64], [0], 1, 64, 16, torch.bfloat16)
    c.cache.data[:] = torch.arange(c.cache.blocks * 16, device="cuda").view(1, 1, -1, 1, 16, 1) % 128
    old = c.tables[0].copy()
    c.tables[0, 0], c.tables[0, 3] = 10 ** 6, -7
    c.rebatch()
    weights = torch.arange(64, device="cuda").float().view(1, 1, 64).contiguous()
    kept = torch.empty(1, 1, 40, dtype=torch.int32, device="cuda")
    before = c.cache.data.clone()
    remp.remp_kv_evict(c.pool, c.dev_lens, c.dev_tables, torch.tensor([40], dtype=torch.int32, device="cuda"), weights, weights.clone(), kept, error=word)
    assert int(word) == 8 and kept[0, 0].tolist() == list(range(24, 64))
    for i in range(40):
        src, dst = i + 24, i
        got = c.cache.data[0, 0, old[dst // 16], 0, dst % 16]
        if src // 16 in (0, 3) or dst // 16 in (0, 3):
            assert torch.equal(got, before[0, 0, old[dst // 16], 0, dst % 16])
        else:
            assert torch.equal(got, before[0, 0, old[src // 16], 0, src % 16])


def test_captured():
    c = Case([200, 90], [0, 0], 2, 64, 16, torch.bfloat16)
    weights, kept = torch.rand(2, 2, 200, device="cuda"), torch.empty(2, 2, 64, dtype=torch.int32, device="cuda")
    out, keep = torch.zeros_like(weights), torch.tensor([64, 64], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        remp.remp_kv_evict(c.pool, c.dev_lens, c.dev_tables, keep, weights, out, kept, recent=8)
    for n in (200, 130):
        c.dev_lens[0] = n
        weights.copy_(torch.rand(2, 2, 200, device="cuda"))
        graph.replay()
        for h in range(2):
            assert kept[0, h].tolist() == ref.choose(weights[0, h].cpu().numpy(), n, 64, 0, 8)
