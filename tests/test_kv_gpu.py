"""The cache of 16-bit values on the GPU against plain formulas in 64 bits: append, attention, weights of positions.

Tolerances. Products of 16-bit numbers are exact in 32 bits; a matrix instruction cuts its sum of 16 of them at 2^-22 of its largest
partial sum, and a score is at most 16 of these: a score is off by at most 2^-18 of scale * sum |q||k| (`terms`), the power
of two by 2^-21 of itself and 2^-23 of the score. A probability goes to the matrix instructions with 16 bits at least, their sums over
a warp's tiles are cut at 2^-22 each, at most 256 tiles here: 2^-14. So |out - exact| <= half a step of the output +
(2 * (terms * 2^-18 + 2^-20) + 2^-14 + P) * sum p|v| / sum p, with P = 0 up to FEW rows of a sequence and KV head; above, where
probabilities are rounded to the output's type, P is half a step of it. lse: terms * 2^-18 + |lse| * 2^-22 + 2^-18.
Weights: (terms * 2^-18 + |lse| * 2^-21 + 2^-18) of what is added + 2^-22 of the sum. Append: norms and turns are a handful of
operations in 32 bits, each off by 2^-24 of the larger operand: half a step of the output + 2^-20 of the larger of the pair.
"""
import math

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu

FEW = 16
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Case:
    """A cache, a batch over it, and its tables on the host."""

    def __init__(self, lens, new, heads, d, bs, dtype, seed=0, token_major=False, layers=1, layer=0, spare=3, error=None, width=None):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.new = np.asarray(lens, dtype=np.int64), np.asarray(new, dtype=np.int64)
        need = -(-self.lens // bs)
        blocks = int(need.sum()) + spare
        self.tables = np.full((len(lens), width or max(1, int(need.max(initial=0)) + 1)), -1, dtype=np.int32)
        ids = rng.permutation(blocks)
        at = 0
        for s, n in enumerate(need):
            self.tables[s, :n] = ids[at:at + n]
            at += n
        self.cache = ref.Cache(layers, blocks, heads, d, bs, dtype, token_major, gen=self.gen)
        self.layer, self.dtype, self.d, self.heads, self.bs = layer, dtype, d, heads, bs
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.error = error
        self.pool = remp.make_kv_pool(self.cache.data, blocks, heads, d, bs, layer=layer, strides=self.cache.strides())
        self.rebatch()

    def rebatch(self):
        self.dev_tables = torch.from_numpy(self.tables).cuda()
        self.dev_lens = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.batch = remp.make_kvq_batch(self.dev_lens, self.dev_tables, torch.from_numpy(self.start).cuda(), int(self.start[-1]),
                                         int(self.new.max(initial=0)), self.error)

    def queries(self, heads, size=1.0):
        return (torch.randn(int(self.start[-1]), heads, self.d, generator=self.gen, device="cuda") * size).to(self.dtype)

    def exact(self, q, scale, window, first):
        """For each sequence: (slice of rows, out, lse, size, terms, weights)."""
        for s in range(len(self.lens)):
            mine = slice(int(self.start[s]), int(self.start[s + 1]))
            room = self.tables.shape[1] * self.bs
            length = min(max(int(self.lens[s]), 0), room)
            yield (mine,) + ref.attend(self.cache, self.layer, self.dev_tables[s], length, q[mine].double(), int(max(self.lens[s], 0) - self.new[s]), scale,
                                       window, first)


def check(c, q_heads, window=0, first=0, size=1.0, few=None, q=None, out=None, stream=None):
    q = c.queries(q_heads, size) if q is None else q
    scale = c.d ** -0.5
    out = torch.full_like(q, 7.0, memory_format=torch.contiguous_format) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    remp.remp_kv_attend(c.pool, c.batch, q, out, scale, remp.make_kv_workspace(), window=window, first=first, lse=lse, stream=stream)
    torch.cuda.synchronize()
    rows = int(c.new.max(initial=0)) * q_heads // c.heads
    extra = 0.0 if (rows <= FEW if few is None else few) else HALF_STEP[c.dtype]
    for mine, want, want_lse, weight, terms, _ in c.exact(q, scale, window, first):
        tol = HALF_STEP[c.dtype] * want.abs() + (2 * (terms * 2.0 ** -18 + 2.0 ** -20) + 2.0 ** -14 + extra) * weight + 2.0 ** -26
        err = (out[mine].double() - want).abs()
        assert (err <= tol).all(), (float((err / tol).max()), window, first)
        some = torch.isfinite(want_lse)
        assert torch.equal(torch.isfinite(lse[mine]), some) and (lse[mine][~some] == -math.inf).all()
        bound = terms * 2.0 ** -18 + want_lse[some].abs() * 2.0 ** -22 + 2.0 ** -18
        assert ((lse[mine][some].double() - want_lse[some]).abs() <= bound).all()
    return q, out, lse


# ---- attention ----

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 1), (8, 2), (3, 3), (32, 2), (64, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_single_tokens(d, hq, hk, dtype):
    lens = [1, 15, 16, 17, 31, 33, 100, 0, 257, 640]
    check(Case(lens, [min(1, n) for n in lens], hk, d, 16, dtype, seed=d + hq), hq)


@pytest.mark.parametrize("bs", [16, 32, 48, 128])
@pytest.mark.parametrize("token_major", [False, True])
def test_blocks_and_orders(bs, token_major):
    lens = [1, 47, 48, 49, 96, 200, 333]
    check(Case(lens, [1] * 7, 3, 128, bs, torch.bfloat16, token_major=token_major, layers=2, layer=1), 6)
    check(Case(lens, [1, 3, 1, 2, 5, 1, 4], 2, 64, bs, torch.float16, token_major=token_major), 4, window=60, first=5)


@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (7, 3), (16, 16), (17, 40), (100, 4), (1000, 4), (64, 1000), (2 ** 31 - 1, 2 ** 31 - 1), (0, 9)])
@pytest.mark.parametrize("queries", [1, 3, 16])
def test_windows_and_first_tokens(window, first, queries):
    lens = [queries, 17 + queries, 64, 65, 130, 500, 40]
    check(Case(lens, [queries] * 6 + [0], 2, 128, 16, torch.bfloat16, seed=window % 97), 4, window=window, first=first)


@pytest.mark.parametrize("queries,hq,hk", [(2, 8, 2), (2, 16, 2), (3, 7, 1), (9, 4, 4), (16, 2, 2), (17, 1, 1), (40, 4, 2), (5, 40, 8)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_several_queries(queries, hq, hk, d):
    lens = [queries, queries + 1, 100 + queries, 300, 41]
    check(Case(lens, [queries, 1, queries, queries // 2, 2], hk, d, 16, torch.bfloat16, seed=queries), hq)


def test_one_long_sequence_and_many_short_ones():
    check(Case([20011], [1], 2, 128, 16, torch.bfloat16), 16)
    check(Case([20011], [2], 1, 64, 32, torch.float16), 4, window=9000, first=100)
    rng = np.random.default_rng(1)
    lens = rng.integers(1, 64, 1300)
    check(Case(lens, [1] * 1300, 2, 128, 32, torch.bfloat16), 8)


def test_rows_before_the_first_position_and_lengths_beyond_the_table():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([2, 40, 0], [5, 1, 2], 2, 128, 16, torch.bfloat16, error=word)
    q, out, lse = check(c, 4)
    assert int(word) == 2 and (out[:3] == 0).all() and (lse[:3] == -math.inf).all()
    word.zero_()
    c = Case([70], [1], 2, 128, 16, torch.bfloat16, error=word, width=5)
    c.lens[0] = 1000
    c.rebatch()
    check(c, 4)
    assert int(word) == 2


def test_blocks_outside_the_pool_are_not_there():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([100, 64, 30], [1, 3, 1], 2, 128, 16, torch.float16, error=word)
    c.tables[0, 2], c.tables[1, 0], c.tables[2, 0], c.tables[2, 1] = 10 ** 6, -5, 2 ** 31 - 1, -1
    c.rebatch()
    _, out, _ = check(c, 4)
    assert int(word) == 8 and (out[4] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("queries", [1, 2])
def test_slots_that_nobody_sees_hold_anything(bad, queries):
    c = Case([100, 33], [queries] * 2, 2, 128, 16, torch.bfloat16)
    window, first = 20, 3
    for s, n in enumerate(c.lens):
        for pos in range(c.tables.shape[1] * 16):
            block = c.tables[s, pos // 16]
            if block >= 0 and (pos >= n or first <= pos <= n - queries - window):
                c.cache.slots(0, 0)[block, pos % 16] = bad
                c.cache.slots(0, 1)[block, pos % 16] = bad
    check(c, 8, window=window, first=first)


def test_very_large_and_very_low_scores():
    c = Case([200, 77], [1, 2], 2, 128, 16, torch.bfloat16)
    check(c, 8, size=60.0)
    c = Case([200, 77], [1, 2], 2, 128, 16, torch.float16)
    c.cache.data[:, 0] = -c.cache.data[:, 0].abs() * 30
    q = c.queries(8).abs() * 20
    check(c, 8, q=q)


def test_strides_of_rows():
    c = Case([50, 20, 7], [1, 2, 1], 2, 128, 16, torch.bfloat16)
    wide = torch.randn(4, 3, 8, 160, generator=c.gen, device="cuda").bfloat16()
    out = torch.full((4, 8, 160), 3.0, device="cuda", dtype=torch.bfloat16)
    check(c, 4, q=wide[:, 1, 2:6, 16:144], out=out[:, 1:5, 16:144])
    assert (out[:, 0] == 3).all() and (out[:, 5:] == 3).all() and (out[..., :16] == 3).all() and (out[..., 144:] == 3).all()
    check(c, 4, q=wide[:1, 0, :4, :128].expand(4, 4, 128))  # one row for every token


def test_results_do_not_depend_on_the_run_and_workspaces_are_left_ready():
    c = Case([3000, 10, 777], [1, 1, 1], 4, 128, 16, torch.bfloat16)
    q, w, outs = c.queries(32), remp.make_kv_workspace(), []
    for _ in range(3):
        out = torch.empty_like(q)
        remp.remp_kv_attend(c.pool, c.batch, q, out, 0.1, w)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_captured_and_on_another_stream():
    c = Case([300, 40], [1, 1], 2, 128, 16, torch.bfloat16)
    q, w = c.queries(8), remp.make_kv_workspace()
    out, lse, weights = torch.empty_like(q), torch.empty(2, 8, device="cuda"), torch.zeros(2, 2, 300, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            remp.remp_kv_attend(c.pool, c.batch, q, out, 0.1, w, lse=lse)
            remp.remp_kv_weigh(c.pool, c.batch, q, lse, weights, 0.1)
    for size in (1.0, 3.0):
        q.copy_(c.queries(8, size))
        graph.replay()
        torch.cuda.synchronize()
        again, wanted = torch.empty_like(q), weights.clone()
        remp.remp_kv_attend(c.pool, c.batch, q, again, 0.1, w)
        assert torch.equal(out, again)
        weights.zero_()
        remp.remp_kv_weigh(c.pool, c.batch, q, lse, weights, 0.1)
        if size == 1.0:
            assert torch.equal(weights, wanted)


# ---- weights of positions ----

def check_weights(c, q_heads, window=0, first=0, fresh=False, stride=None):
    q = c.queries(q_heads)
    scale, longest = c.d ** -0.5, int(max(c.lens.max(), 1))
    lse = torch.empty(q.shape[0], q_heads, device="cuda")
    remp.remp_kv_attend(c.pool, c.batch, q, torch.empty_like(q), scale, remp.make_kv_workspace(), window=window, first=first, lse=lse)
    stride = stride or longest + 3
    before = torch.rand(len(c.lens), c.heads, stride, device="cuda", generator=c.gen) * 2
    got = before.clone()
    remp.remp_kv_weigh(c.pool, c.batch, q, lse, got, scale, window=window, first=first, fresh=fresh)
    for s, (mine, _, _, _, terms, _) in enumerate(c.exact(q, scale, window, first)):
        n, new = min(int(c.lens[s]), stride), int(c.new[s])
        if new == 0 or n == 0:
            assert torch.equal(got[s], before[s])
            continue
        key = torch.arange(int(c.lens[s]), device="cuda")
        k, good = c.cache.rows(c.layer, 0, c.dev_tables[s], key)
        k = torch.where(good[:, None, None], k, 0.0)
        seen = ref.sees(c.lens[s] - new + torch.arange(new, device="cuda"), key, window, first) & good[None]
        group = q_heads // c.heads
        added, big = torch.zeros(c.heads, len(key), dtype=torch.float64, device="cuda"), 0.0
        for h in range(q_heads):
            norm = lse[mine, h].double()
            x = q[mine, h].double() @ k[:, h // group].T * scale - norm[:, None]
            added[h // group] += torch.where(seen & torch.isfinite(norm)[:, None], torch.exp(x), 0.0).sum(0)
            big = max([big] + norm[torch.isfinite(norm)].abs().tolist())
        old = torch.where((key[:n] >= c.lens[s] - new) | fresh, 0.0, before[s, :, :n].double())
        want = old + added[:, :n]
        tol = (terms * 2.0 ** -18 + big * 2.0 ** -21 + 2.0 ** -18) * added[:, :n] + 2.0 ** -22 * want + 1e-30
        err = (got[s, :, :n].double() - want).abs()
        assert (err <= tol).all(), float((err / tol).max())
        assert torch.equal(got[s, :, n:], before[s, :, n:])
    return got


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk,queries", [(1, 1, 1), (8, 1, 1), (32, 8, 1), (6, 2, 3), (8, 2, 33), (20, 4, 7)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weights(d, hq, hk, queries, dtype):
    lens = [queries, queries + 1, 100, 129, 64, 500]
    check_weights(Case(lens, [queries, 1, queries, 1, 0, queries], hk, d, 16, dtype, seed=queries), hq)


@pytest.mark.parametrize("window,first,fresh", [(1, 0, False), (20, 4, False), (20, 4, True), (1000, 40, True), (0, 0, True), (2 ** 31 - 1, 3, False)])
@pytest.mark.parametrize("token_major", [False, True])
def test_weights_windows(window, first, fresh, token_major):
    check_weights(Case([3, 150, 40, 97], [3, 2, 0, 20], 2, 128, 32, torch.bfloat16, token_major=token_major), 8, window, first, fresh)


def test_weights_bad_blocks_short_rows_and_rows_without_keys():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([100, 64], [1, 3], 2, 128, 16, torch.float16, error=word)
    c.tables[0, 2] = 10 ** 6
    c.rebatch()
    check_weights(c, 4)
    assert int(word) == 8
    word.zero_()
    check_weights(Case([100, 30], [1, 1], 2, 128, 16, torch.float16, error=word), 4, stride=50)
    assert int(word) == 2
    c = Case([2, 9], [4, 1], 1, 64, 16, torch.bfloat16)
    q, lse, got = c.queries(2), torch.full((5, 2), -math.inf, device="cuda"), torch.full((2, 1, 9), 5.0, device="cuda")
    remp.remp_kv_weigh(c.pool, c.batch, q, lse, got, 1.0)
    assert (got[0, :, :2] == 0).all() and (got[0, :, 2:] == 5).all() and (got[1, :, 8] == 0).all() and (got[1, :, :8] == 5).all()


def test_weights_of_one_token_sum_to_the_query_heads():
    c = Case([777, 50], [1, 1], 4, 128, 16, torch.bfloat16)
    q, lse = c.queries(32), torch.empty(2, 32, device="cuda")
    remp.remp_kv_attend(c.pool, c.batch, q, torch.empty_like(q), 0.1, remp.make_kv_workspace(), lse=lse)
    weights = torch.zeros(2, 4, 777, device="cuda")
    remp.remp_kv_weigh(c.pool, c.batch, q, lse, weights, 0.1)
    torch.testing.assert_close(weights.sum(-1), torch.full((2, 4), 8.0, device="cuda"), rtol=1e-4, atol=0)


# ---- append ----

def check_append(c, hq, norm, rotary, interleaved, positions=False, in_place=False):
    t, d = int(c.start[-1]), c.d
    x = (torch.randn(t, hq + 2 * c.heads, d, generator=c.gen, device="cuda") * 2).to(c.dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + c.heads], x[:, hq + c.heads:]
    wq, wk = (torch.rand(d, generator=c.gen, device="cuda") + 0.5 if norm else None for _ in range(2))
    pos = torch.cat([torch.arange(n - m, n) for n, m in zip(c.lens, c.new)]).cuda()
    seq = torch.cat([torch.full((int(m),), s) for s, m in enumerate(c.new)]).cuda()
    rows = int(c.lens.max()) + 4
    rope = torch.rand(rows, rotary, generator=c.gen, device="cuda") * 2 - 1 if rotary else None
    turn = torch.randint(0, rows, (t,), generator=c.gen, device="cuda").int() if positions else pos
    before = c.cache.data.clone()
    source = x.clone()
    q_out = q if in_place else torch.empty(t, hq, d, dtype=c.dtype, device="cuda")
    remp.remp_kv_append(c.pool, c.batch, q if hq else None, k, v, q_out if hq else None, q_norm=wq, k_norm=wk, eps=1e-5, rope=rope, interleaved=interleaved,
                        positions=turn if positions else None)

    def formula(y, w):
        y = y.double()
        if w is not None:
            y = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.double()
        size = y.abs()
        if rope is not None:
            r = rotary // 2
            cos, sin = rope[turn.long(), None, :r].double(), rope[turn.long(), None, r:].double()
            at = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, r), slice(r, rotary))
            a, b = y[..., at[0]].clone(), y[..., at[1]].clone()
            y, size = y.clone(), size.clone()
            y[..., at[0]], y[..., at[1]] = a * cos - b * sin, b * cos + a * sin
            size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
        return y, size

    sq, sk, sv = source[:, :hq], source[:, hq:hq + c.heads], source[:, hq + c.heads:]
    block = c.dev_tables[seq, pos // c.bs].long()
    got_k, got_v = c.cache.slots(c.layer, 0)[block, pos % c.bs], c.cache.slots(c.layer, 1)[block, pos % c.bs]
    assert torch.equal(got_v, sv)
    for got, (want, size) in ((q_out, formula(sq, wq)), (got_k, formula(sk, wk))):
        assert ((got.double() - want).abs() <= HALF_STEP[c.dtype] * want.abs() + 2.0 ** -20 * size + 2.0 ** -25).all()
    if not norm and not rotary:
        assert torch.equal(got_k, sk)
    # everything else is as it was
    for kv in (0, 1):
        c.cache.slots(c.layer, kv)[block, pos % c.bs] = 0
    mine = ref.Cache.__new__(ref.Cache)
    mine.__dict__.update(c.cache.__dict__, data=before)
    for kv in (0, 1):
        mine.slots(c.layer, kv)[block, pos % c.bs] = 0
    assert torch.equal(c.cache.data, before)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 1), (3, 3), (64, 8), (0, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_append(d, hq, hk, dtype):
    check_append(Case([1, 16, 17, 40, 0, 33, 5], [1, 1, 17, 3, 0, 1, 5], hk, d, 16, dtype, seed=d + hq), hq, True, d, False)


@pytest.mark.parametrize("rotary,interleaved,norm", [(16, False, False), (32, True, True), (48, False, True), (64, True, False), (0, False, True), (0, False, False)])
@pytest.mark.parametrize("token_major", [False, True])
def test_append_transforms(rotary, interleaved, norm, token_major):
    check_append(Case([70, 3, 64], [70, 2, 1], 2, 64, 32, torch.bfloat16, token_major=token_major), 4, norm, rotary, interleaved)
    check_append(Case([70, 3, 64], [4, 3, 33], 2, 128, 48, torch.float16, layers=3, layer=1, token_major=token_major), 4, norm, rotary, interleaved,
                 positions=True, in_place=True)


def test_append_many_tokens():
    check_append(Case([2500, 1900, 1], [2500, 1700, 1], 3, 128, 16, torch.bfloat16), 5, True, 128, False)


def test_append_invalid_tokens_write_nothing():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case([20, 3, 33], [2, 5, 1], 1, 64, 16, torch.bfloat16, error=word)
    c.tables[0, 1] = 99
    c.rebatch()
    x = torch.randn(8, 4, 64, device="cuda").bfloat16()
    q_out = torch.full((8, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16)
    before = c.cache.data.clone()
    remp.remp_kv_append(c.pool, c.batch, x[:, :2], x[:, 2:3], x[:, 3:], q_out)
    assert int(word) == 10
    assert torch.equal(q_out[:2], x[:2, :2]) and (q_out[2:4] == 9).all() and torch.equal(q_out[4:], x[4:, :2])
    block = c.tables[1, 0]
    changed = (c.cache.data != before).any(-1).nonzero().tolist()
    assert {(b, t) for _, _, b, _, t in changed} <= {(block, 0), (block, 1), (block, 2), (c.tables[2, 2], 0)}
