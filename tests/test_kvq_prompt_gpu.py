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


# ---- the range of the numbers ----

def _sized(blocks, heads, d, bs, rng, k_size, v_size):
    """A pool whose tokens have K and V of the given sizes (numbers, or arrays [blocks][bs] for each slot)."""
    p = base.ref.Pool(1, blocks, heads, d, bs)
    for kv, size in enumerate((k_size, v_size)):
        size = np.broadcast_to(np.asarray(size, dtype=np.float32), (blocks, bs)).reshape(blocks, 1, bs // 16, 16, 1)
        c, s, m = base.ref.quantise(rng.standard_normal((blocks, heads, bs // 16, 16, d)).astype(np.float32) * size)
        c = c[..., base.ref.place_of(d, kv == 1)]
        b = (c[..., 0::2] | c[..., 1::2] << 4).reshape(blocks, heads, bs // 16, -1)
        p.bytes[0, kv] = np.concatenate([b, np.stack([s, m], -1).reshape(blocks, heads, bs // 16, -1).view(np.uint8)], -1)
    return p


def _check_range(out, lse, q, pool, lens, new, tables, scale):
    """As base._check, with nothing that does not shrink with the values: half an ulp of the output, what rounding
    probabilities and values to 11 bits does to sums of p * (largest of V's row), and what rounding keys does to scores."""
    at = 0
    for s in range(len(lens)):
        n, length = int(new[s]), int(lens[s])
        k, v = (pool.rows(0, kv, tables[s], length) for kv in (0, 1))
        want, want_lse, _, size, move = base.ref.attend(q[at:at + n].double().cpu().numpy(), k, v, length - n, scale, 0)
        tol = base.ULP[out.dtype] / 2 * np.abs(want) + ((2.0 ** -10 + 2 * move) * size)[..., None]
        err = np.abs(out[at:at + n].double().cpu().numpy() - want)
        assert (err <= tol).all(), (s, (err / tol).max())
        assert (np.abs(lse[at:at + n].double().cpu().numpy() - want_lse) <= 2e-5 * np.maximum(1, np.abs(want_lse)) + move).all()
        at += n


def _range_case(d, hq, hk, lens, new, k_size, v_size, q_size, score=1.0, seed=0, per_token=None):
    rng = np.random.default_rng(seed)
    blocks = int((-(-np.asarray(lens) // 16)).sum())
    lens, new, tables, start, batch = base._batch(lens, new, 16, blocks, rng)
    if per_token:
        k_size, v_size = (x * 10.0 ** rng.uniform(*per_token[i], (blocks, 16)) for i, x in enumerate((k_size, v_size)))
    pool = _sized(blocks, hk, d, 16, rng, k_size, v_size)
    buf, dev = base._dev_pool(pool)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn(int(start[-1]), hq, d, device="cuda", generator=gen) * q_size).bfloat16()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    scale = score * d ** -0.5
    remp.remp_kvq_attend(dev, batch, q, out, scale, remp.make_kvq_workspace(), lse=lse)
    _check_range(out, lse, q, pool, lens, new, tables, scale)


# prompts of more than 32 rows: one matrix, two matrices, keys in parts
PROMPTS = [(64, 2, 1, [70, 150], [70, 33]), (128, 4, 1, [200, 40], [80, 20]), (256, 1, 1, [60, 130], [60, 40])]


@pytest.mark.parametrize("size", [1e-3, 1e-5, 1e-7, 1e-12, 1e-25, 1e7, 1e20])
@pytest.mark.parametrize("d,hq,hk,lens,new", PROMPTS)
def test_prompt_values_of_any_size(d, hq, hk, lens, new, size):
    _range_case(d, hq, hk, lens, new, 1.0, size, 1.0, seed=d)


@pytest.mark.parametrize("size", [1e-3, 1e-5, 1e-7, 1e-12, 1e7, 1e12])
@pytest.mark.parametrize("d,hq,hk,lens,new", PROMPTS)
def test_prompt_keys_of_any_size(d, hq, hk, lens, new, size):
    _range_case(d, hq, hk, lens, new, size, 1.0, 1 / size, seed=d + 1)


@pytest.mark.parametrize("d,hq,hk,lens,new", PROMPTS)
def test_prompt_tokens_of_different_sizes(d, hq, hk, lens, new):
    # a row that sees only small values is as exact as one that sees large ones
    _range_case(d, hq, hk, lens, new, 1.0, 1.0, 1.0, seed=d + 2, per_token=((-3, 0.5), (-9, 6)))
    _range_case(d, hq, hk, lens, new, 1.0, 1.0, 1.0, seed=d + 3, per_token=((-3, -1), (-5, -2)))  # around where the kernel changes its way
    _range_case(d, hq, hk, lens, new, 1.0, 1.0, 1.0, seed=d + 5, per_token=((0, 0), (1, 4)))
    _range_case(d, hq, hk, lens, new, 1e-2, 1.0, 100.0, seed=d + 4, per_token=((-1.5, 0.5), (3, 6)))


# ---- many blocks of keys in a thread block ----

# (head_dim, query heads, KV heads, sequences, tokens, query tokens, window): of 148 units and more, so that the first 148 walk all
# their keys and the others share theirs; a block of keys is 128 of them (64 with 256 dims); up to 128 rows, and above
LONG = [(128, 16, 8, 20, 800, 20, 0), (128, 32, 16, 10, 600, 70, 0), (64, 16, 8, 20, 900, 20, 0), (64, 10, 10, 15, 700, 150, 0), (256, 8, 8, 20, 500, 40, 0),
        (128, 16, 8, 20, 800, 20, 300), (64, 10, 10, 15, 700, 150, 170), (256, 8, 8, 20, 500, 40, 150), (128, 4, 4, 37, 700, 40, 0)]


@pytest.mark.parametrize("dtype,half_ulp", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("d,hq,hk,seqs,length,queries,window", LONG)
def test_prompt_over_many_blocks_of_keys(d, hq, hk, seqs, length, queries, window, rising, dtype, half_ulp):
    # Keys are whole numbers from -7 to 8 with both ends in each group: step 1 and minimum -7, exact in half, so nothing in the
    # tolerance grows with the scores (2^-13 is for their sums in 32 bits, 2^-20 of the sizes of some 30 that they add up).
    # rising: eight dims make the scores of each sixteenth of the sequence 9 (base 2) higher than those of the one before, so that
    # references move between blocks of keys and within them.
    rng = np.random.default_rng(d + queries)
    lens = rng.integers(length * 3 // 4, length + 1, seqs)
    lens[0] = length
    blocks = int((-(-lens // 16)).sum())
    lens, new, tables, start, batch = base._batch(lens, np.full(seqs, queries), 16, blocks, rng)
    k = rng.integers(-7, 9, (blocks, hk, 16, d))
    k[..., 0::64], k[..., 1::64] = -7, 8
    q = rng.standard_normal((int(start[-1]), hq, d))
    if rising:
        q[..., 2:10] = 9 / (8 * d ** -0.5 * np.log2(np.e))
        for s in range(seqs):
            level = np.arange(-(-lens[s] // 16) * 16) * 16 // lens[s] - 7
            k[tables[s, :len(level) // 16], :, :, 2:10] = np.minimum(level, 8).reshape(-1, 1, 16, 1)
    else:
        q *= 0.5
    pool = base.ref.Pool(1, blocks, hk, d, 16)
    for kv, x in enumerate((k, rng.standard_normal(k.shape))):
        c, step, low = base.ref.quantise(x.astype(np.float32))
        assert kv or ((step == 0x3f80) & (low == 0xc0e0)).all()
        c = c[..., base.ref.place_of(d, kv == 1)]
        codes = (c[..., 0::2] | c[..., 1::2] << 4).reshape(blocks, hk, 1, -1)
        pool.bytes[0, kv] = np.concatenate([codes, np.stack([step, low], -1).reshape(blocks, hk, 1, -1).view(np.uint8)], -1)
    buf, dev = base._dev_pool(pool)
    q = torch.from_numpy(q).to(dtype).cuda()
    out, again, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = remp.make_kvq_workspace()
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, ws, window=window, lse=lse)
    remp.remp_kvq_attend(dev, batch, q, again, d ** -0.5, ws, window=window)
    assert torch.equal(out, again)
    for s in (0, 1, seqs // 2, seqs - 1):
        rows = slice(s * queries, (s + 1) * queries)
        kk, vv = (pool.rows(0, kv, tables[s], int(lens[s])) for kv in (0, 1))
        want, want_lse, _, size, _ = base.ref.attend(q[rows].double().cpu().numpy(), kk, vv, int(lens[s]) - queries, d ** -0.5, window)
        err = np.abs(out[rows].double().cpu().numpy() - want)
        tol = half_ulp * np.abs(want) + (2.0 ** -10 + 2.0 ** -13) * size[..., None]
        assert (err <= tol).all(), (s, (err / tol).max())
        assert (np.abs(lse[rows].double().cpu().numpy() - want_lse) <= 2e-5 * np.maximum(1, np.abs(want_lse))).all()
