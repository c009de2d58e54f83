"""The 4-bit cache on the GPU against plain numpy: bytes written, values read back, attention in 64 bits.

Tolerances. The bytes are compared exactly: the reference does the same float32 operations one by one. Values read back
are one float32 multiply-add, rounded once to 16 bits. Attention: p*step is rounded to half (at most 2^-11 of it, and the
codes it meets are at most the row's spread), scores carry the float32 sums of the matrix instructions (a few 2^-20), the
output is rounded once to its type: |error| <= half an ulp of the output + 2^-10 * sum of p * spread of V's row.
lse: 2e-5, from float32 sums of scores up to a few tens.
With more than 32 rows of a sequence and KV head (PROMPT_ROWS), keys, values and probabilities are rounded to half: a value
and a probability by 2^-11 of themselves, a score by at most `move` = scale * sum |q||k| * 2^-11, a probability's share by
twice that: |error| <= half an ulp + (2^-10 + 2 move) * sum of p * largest of V's row; lse: 2e-5 + move.
"""
import math

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import kvq_reference as ref

pytestmark = pytest.mark.gpu

PROMPT_ROWS = 32
ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _batch(lens, new, bs, blocks, rng, max_blocks=None, error=None):
    lens, new = np.asarray(lens, dtype=np.int32), np.asarray(new, dtype=np.int32)
    need = -(-np.maximum(lens, 0) // bs)
    width = max_blocks or max(1, int(need.max(initial=0)) + 1)
    assert need.sum() <= blocks
    ids = rng.permutation(blocks)
    tables = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for s in range(len(lens)):
        tables[s, :need[s]] = ids[at:at + need[s]]
        at += need[s]
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return lens, new, tables, start, _dev_batch(lens, tables, start, new, error)


def _dev_batch(lens, tables, start, new, error=None):
    return remp.make_kvq_batch(*(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (lens, tables, start)), int(start[-1]),
                               int(new.max(initial=0)), error)


def _dev_pool(p, layer=0):
    buf = torch.from_numpy(p.bytes.reshape(-1)).cuda()
    return buf, remp.make_kvq_pool(buf, p.blocks, p.heads, p.d, p.bs, layer=layer)


def _rope(rows, dim, rng):
    a = rng.uniform(0, 2 * np.pi, size=(rows, dim // 2))
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def _append_case(d, hq, hk, bs, dtype, norm, rotary, interleaved, lens, new, seed, layers=1, layer=0, positions=False):
    rng = np.random.default_rng(seed)
    blocks = int((-(-np.asarray(lens) // bs)).sum()) + 3
    lens, new, tables, start, batch = _batch(lens, new, bs, blocks, rng)
    t = int(start[-1])
    pool = ref.Pool(layers, blocks, hk, d, bs)
    x = torch.from_numpy(rng.standard_normal((t, hq + 2 * hk, d)).astype(np.float32) * (1 + 4 * (rng.random((hq + 2 * hk, d)) < 0.05))).to(dtype).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    wq, wk = (rng.uniform(0.5, 1.5, d).astype(np.float32) if norm else None for _ in range(2))
    rope = _rope(int(lens.max()) + 4, rotary, rng) if rotary else None
    pos = np.concatenate([np.arange(n - c, n) for n, c in zip(lens, new)]).astype(np.int64)
    turn = rng.integers(0, rope.shape[0], t).astype(np.int32) if positions else pos
    buf, dev = _dev_pool(pool, layer)
    dv = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    q_out = torch.empty(t, hq, d, dtype=dtype, device="cuda")
    remp.remp_kvq_append(dev, batch, q, k, v, q_out, q_norm=dv(wq), k_norm=dv(wk), eps=1e-5, rope=dv(rope), interleaved=interleaved,
                         positions=dv(turn) if positions else None)
    k_out, v_out = (torch.empty(t, hk, d, dtype=dtype, device="cuda") for _ in range(2))
    remp.remp_kvq_read(dev, batch, k_out, v_out)
    # the plain statement
    qf, kf, vf = (a.float().cpu().numpy() for a in (q, k, v))
    qf = ref.turn_rows(ref.norm_rows(qf, wq, 1e-5), rope, turn, interleaved)
    kf = ref.turn_rows(ref.norm_rows(kf, wk, 1e-5), rope, turn, interleaved)
    i = 0
    want_k, want_v = np.empty((t, hk, d)), np.empty((t, hk, d))
    for s in range(len(lens)):
        for _ in range(new[s]):
            b = tables[s, pos[i] // bs]
            pool.write(layer, 0, b, pos[i], kf[i])
            pool.write(layer, 1, b, pos[i], vf[i])
            want_k[i], want_v[i] = pool.read(layer, 0, b, pos[i]), pool.read(layer, 1, b, pos[i])
            i += 1
    assert torch.equal(q_out.cpu(), torch.from_numpy(qf).to(dtype))
    assert np.array_equal(buf.cpu().numpy(), pool.bytes.reshape(-1))
    for got, want in ((k_out, want_k), (v_out, want_v)):
        # float32(c*s) + m, then one rounding: within one ulp of the exact value rounded
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= ULP[dtype] * np.abs(want) + 2.0 ** -24 * np.abs(want).max()).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 1), (8, 2), (3, 3), (64, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_append_writes_the_bytes_of_the_plain_statement(d, hq, hk, dtype):
    lens, new = [1, 16, 17, 40, 0, 33, 5], [1, 1, 17, 3, 0, 1, 5]
    _append_case(d, hq, hk, 16, dtype, True, d, False, lens, new, d + hq)


@pytest.mark.parametrize("rotary,interleaved,norm", [(16, False, False), (32, True, True), (48, False, True), (64, True, False), (0, False, True), (0, False, False)])
def test_append_rotations_and_norms(rotary, interleaved, norm):
    _append_case(64, 4, 2, 32, torch.bfloat16, norm, rotary, interleaved, [70, 3, 64], [70, 2, 1], 7)
    _append_case(128, 4, 2, 48, torch.float16, norm, rotary, interleaved, [70, 3, 64], [4, 3, 33], 8)


def test_append_layer_of_a_pool_and_given_positions():
    _append_case(128, 6, 2, 16, torch.bfloat16, True, 128, False, [20, 21], [3, 21], 9, layers=3, layer=1, positions=True)


def test_append_one_sequence_of_many_and_many_of_one():
    rng = np.random.default_rng(3)
    new = rng.integers(0, 2, 1500)
    new[0] = 1
    lens = new + rng.integers(0, 40, 1500) * (new > 0)
    _append_case(64, 1, 1, 16, torch.bfloat16, False, 64, False, lens, new, 4)


def test_append_in_place_and_keys_only():
    rng = np.random.default_rng(1)
    d, hk, bs = 128, 2, 16
    lens, new, tables, start, batch = _batch([18, 2], [2, 2], bs, 6, rng)
    x = torch.randn(4, 3 * hk, d, device="cuda").bfloat16()
    rope = torch.from_numpy(_rope(20, d, rng)).cuda()
    p1, p2, p3 = (ref.Pool(1, 6, hk, d, bs) for _ in range(3))
    (b1, d1), (b2, d2), (b3, d3) = (_dev_pool(p) for p in (p1, p2, p3))
    apart = torch.empty(4, hk, d, dtype=x.dtype, device="cuda")
    remp.remp_kvq_append(d1, batch, x[:, :hk], x[:, hk:2 * hk], x[:, 2 * hk:], apart, rope=rope)
    remp.remp_kvq_append(d3, batch, None, x[:, hk:2 * hk], x[:, 2 * hk:], None, rope=rope)
    y = x.clone()
    remp.remp_kvq_append(d2, batch, y[:, :hk], y[:, hk:2 * hk], y[:, 2 * hk:], y[:, :hk], rope=rope)
    assert torch.equal(b1, b2) and torch.equal(b1, b3) and torch.equal(y[:, :hk], apart) and torch.equal(y[:, hk:], x[:, hk:])


def test_append_special_values():
    rng = np.random.default_rng(2)
    d, bs = 128, 16
    lens, new, tables, start, batch = _batch([8], [8], bs, 2, rng)
    v = torch.randn(8, 1, d, device="cuda").half()
    v[0, 0, 3] = math.nan
    v[1, 0, 70] = math.inf
    v[2, 0, 70] = -math.inf
    v[3] = 100.3           # constant rows: the step takes up the minimum's rounding
    v[4] = 0
    v[5, 0, ::2], v[5, 0, 1::2] = 65504, -65504
    v[6] = v[6] * 1e-5
    pool = ref.Pool(1, 2, 1, d, bs)
    buf, dev = _dev_pool(pool)
    remp.remp_kvq_append(dev, batch, None, v, v, None)
    x = v.float().cpu().numpy()
    for i in range(8):
        for kv in (0, 1):
            pool.write(0, kv, tables[0, 0], i, x[i])
    assert np.array_equal(buf.cpu().numpy(), pool.bytes.reshape(-1))
    out = torch.zeros_like(v)
    remp.remp_kvq_read(dev, batch, None, out)
    got = out[:, 0].float().cpu().numpy()
    assert np.isnan(got[0, :64]).all() and np.isfinite(got[0, 64:]).all()
    assert np.isnan(got[1, 64:]).all() and np.isnan(got[2, 64:]).all() and np.isfinite(got[1, :64]).all()
    assert np.abs(got[3] - 100.3).max() < 0.1 and (got[4] == 0).all()
    assert np.abs(got[5] - x[5, 0]).max() <= 65504 * 2.0 ** -8


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-3, 1.0, 1e30])
def test_append_codes_on_the_edge(size):
    # values of few bits: many quotients lie exactly between two codes, and steps of every size
    rng = np.random.default_rng(11)
    d, bs, n = 128, 16, 64
    lens, new, tables, start, batch = _batch([n], [n], bs, 4, rng)
    x = (rng.integers(-15, 16, (n, 2, d)) * 0.5 * size).astype(np.float32)
    x[::3] *= rng.choice([1.0, 0.75, 3.0], (len(x[::3]), 1, 1)).astype(np.float32)
    v = torch.from_numpy(x).bfloat16().cuda()
    pool = ref.Pool(1, 4, 1, d, bs)
    buf, dev = _dev_pool(pool)
    remp.remp_kvq_append(dev, batch, None, v[:, :1], v[:, 1:], None)
    f = v.float().cpu().numpy()
    for i in range(n):
        for kv in (0, 1):
            pool.write(0, kv, tables[0, i // bs], i, f[i, kv:kv + 1])
    assert np.array_equal(buf.cpu().numpy(), pool.bytes.reshape(-1))


def test_append_and_read_skip_what_is_not_there():
    rng = np.random.default_rng(5)
    d, bs, hk = 64, 16, 2
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, new = np.array([3, 1, 17, 40], dtype=np.int32), np.array([2, 2, 2, 1], dtype=np.int32)
    tables = np.array([[0, 1], [1, 2], [3, 99], [4, 5]], dtype=np.int32)  # seq 1: position -1; seq 2: its second block; seq 3: beyond the row
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    batch = _dev_batch(lens, tables, start, new, error)
    pool = ref.Pool(1, 6, hk, d, bs)
    buf, dev = _dev_pool(pool)
    x = torch.randn(7, 3 * hk, d, device="cuda").bfloat16()
    q_out = torch.full((7, hk, d), 7.0, dtype=x.dtype, device="cuda")
    remp.remp_kvq_append(dev, batch, x[:, :hk], x[:, hk:2 * hk], x[:, 2 * hk:], q_out)
    assert int(error) == 2 | 8
    f = x.float().cpu().numpy()
    for i, (b, p) in {0: (0, 1), 1: (0, 2), 3: (1, 0), 4: (3, 15)}.items():
        for kv in (0, 1):
            pool.write(0, kv, b, p, f[i, (kv + 1) * hk:(kv + 2) * hk])
    assert np.array_equal(buf.cpu().numpy(), pool.bytes.reshape(-1))
    skipped = (q_out.float() == 7).all(-1).all(-1).cpu().numpy()
    assert skipped.tolist() == [False, False, True, False, False, False, True]  # a bad block loses K and V only
    out = torch.full((7, hk, d), 7.0, dtype=x.dtype, device="cuda")
    error.zero_()
    remp.remp_kvq_read(dev, batch, out, None)
    assert (out.float() == 7).all(-1).all(-1).cpu().numpy().tolist() == [False, False, True, False, False, True, True]
    assert int(error) == 2 | 8


# ---- attention ----

def _filled(blocks, heads, d, bs, rng, layers=1):
    """A pool whose every slot holds a quantised row."""
    p = ref.Pool(layers, blocks, heads, d, bs)
    n = 16
    for l in range(layers):
        for kv in (0, 1):
            x = rng.standard_normal((blocks, heads, bs // 16, n, d)).astype(np.float32)
            if kv == 0:
                x = x * rng.uniform(0.3, 2, d).astype(np.float32) + rng.standard_normal(d).astype(np.float32)
            c, s, m = ref.quantise(x)
            c = c[..., ref.place_of(d, kv == 1)]
            b = (c[..., 0::2] | c[..., 1::2] << 4).reshape(blocks, heads, bs // 16, -1)
            par = np.stack([s, m], -1).reshape(blocks, heads, bs // 16, -1).view(np.uint8)
            p.bytes[l, kv] = np.concatenate([b, par], -1)
    return p


def _check(out, lse, q, pool, layer, lens, new, tables, scale, window, dtype):
    at = 0
    for s in range(len(lens)):
        n, length = int(new[s]), max(0, int(lens[s]))
        length = min(length, tables.shape[1] * pool.bs)
        k, v = (pool.rows(layer, kv, tables[s], length) for kv in (0, 1))
        want, want_lse, weight, size, move = ref.attend(q[at:at + n].double().cpu().numpy(), k, v, int(lens[s]) - n, scale, window)
        got = out[at:at + n].double().cpu().numpy()
        prompt = int(new.max()) * q.shape[1] // pool.heads > PROMPT_ROWS
        rounding = (2.0 ** -10 + 2 * move) * size if prompt else 2.0 ** -10 * weight
        tol = ULP[dtype] / 2 * np.abs(want) + rounding[..., None] + 2.0 ** -24
        assert (np.abs(got - want) <= tol).all(), (s, n, length, np.abs(got - want).max())
        if lse is not None:
            g = lse[at:at + n].double().cpu().numpy()
            assert np.array_equal(np.isinf(g), np.isinf(want_lse))
            f = np.isfinite(want_lse)
            assert (np.abs(g[f] - want_lse[f]) <= 2e-5 * np.maximum(1, np.abs(want_lse[f])) + (move[f] if prompt else 0)).all()
        at += n


def _attend_case(d, hq, hk, bs, dtype, lens, new, window=0, seed=0, layers=1, layer=0, q_scale=1.0, spoil=True, ws=None):
    rng = np.random.default_rng(seed)
    blocks = int((-(-np.maximum(lens, 0) // bs)).sum()) + 2
    lens, new, tables, start, batch = _batch(lens, new, bs, blocks, rng)
    pool = _filled(blocks, hk, d, bs, rng, layers)
    if spoil:  # slots behind a sequence's end: steps and minima of NaN and infinity
        for s in range(len(lens)):
            if lens[s] > 0 and lens[s] % bs:
                b = tables[s, lens[s] // bs]
                for p in range(lens[s] % bs, bs):
                    o = 8 * d + p % 16 * d // 16
                    pool.bytes[:, :, b, :, p // 16, o:o + d // 16] = np.array([0xC0, 0x7F, 0x80, 0x7F] * (d // 64), dtype=np.uint8)
    buf, dev = _dev_pool(pool, layer)
    t = int(start[-1])
    wide = torch.randn(t, hq + 3, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * q_scale
    q = wide.to(dtype)[:, 1:1 + hq]
    out = torch.full((t, 2 * hq, d), 9.0, dtype=dtype, device="cuda")
    lse = torch.full((t, hq), 9.0, device="cuda")
    scale = d ** -0.5 / q_scale
    ws = remp.make_kvq_workspace() if ws is None else ws
    remp.remp_kvq_attend(dev, batch, q, out[:, ::2], scale, ws, window=window, lse=lse)
    assert (out[:, 1::2].float() == 9).all()
    _check(out[:, ::2], lse, q, pool, layer, lens, new, tables, scale, window, dtype)
    first = out.clone()
    remp.remp_kvq_attend(dev, batch, q, out[:, ::2], scale, ws, window=window)
    assert torch.equal(first, out)  # the same bits again
    return ws


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (8, 1), (5, 1), (10, 2), (16, 1), (24, 2)])
def test_attend_one_token(d, hq, hk):
    lens = [1, 2, 15, 16, 17, 31, 33, 0, 64, 100, 129, 300]
    new = [1] * 12
    _attend_case(d, hq, hk, 16, torch.bfloat16, lens, new, seed=d + hq)


@pytest.mark.parametrize("bs", [16, 32, 48, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_block_sizes_and_types(bs, dtype):
    _attend_case(128, 8, 2, bs, dtype, [5, 47, 48, 49, 255, 256, 257, 500], [1] * 8, seed=bs)
    _attend_case(64, 2, 2, bs, dtype, [5, 47, 48, 49, 255, 256, 257, 500], [1, 2, 0, 3, 1, 7, 1, 2], seed=bs)


@pytest.mark.parametrize("hq,hk,new", [(4, 4, [5, 1, 0, 3, 9]), (8, 1, [2, 3, 1, 4, 6]), (6, 2, [3, 8, 20, 1, 2])])
def test_attend_several_tokens(hq, hk, new):
    for d in (64, 128, 256):
        _attend_case(d, hq, hk, 16, torch.bfloat16, [5, 40, 33, 18, 200], new, seed=3)


@pytest.mark.parametrize("window", [1, 2, 16, 17, 100])
def test_attend_window(window):
    _attend_case(128, 8, 2, 16, torch.bfloat16, [1, 16, 17, 150, 99, 400], [1] * 6, window=window, seed=window)
    _attend_case(64, 4, 1, 32, torch.float16, [7, 30, 60, 150], [7, 3, 12, 30], window=window, seed=window)


def test_attend_rows_that_see_nothing():
    # more query tokens than cached ones: the first rows stand before the sequence
    ws = _attend_case(128, 4, 1, 16, torch.bfloat16, [0, 1, 3, 20], [3, 4, 5, 2], seed=1)
    _attend_case(128, 4, 1, 16, torch.bfloat16, [0, 0, 0], [1, 1, 1], seed=2, ws=ws)
    _attend_case(64, 4, 1, 16, torch.bfloat16, [0, 5], [0, 1], seed=2, ws=ws)


def test_attend_long_and_uneven_one_workspace():
    ws = None
    for seed, (lens, hq, hk) in enumerate([([4000], 8, 1), ([3000, 1, 1, 2000, 7], 8, 2), ([1] * 700, 2, 1), ([2500], 1, 1), ([20] * 40 + [1500], 4, 4)]):
        ws = _attend_case(128, hq, hk, 16, torch.bfloat16, lens, [1] * len(lens), seed=seed, ws=ws)
    _attend_case(64, 16, 1, 16, torch.float16, [2000, 900], [3, 2], seed=9, ws=ws)


@pytest.mark.parametrize("q_scale", [1e-6, 1e-3, 1e4])
def test_attend_query_sizes(q_scale):
    _attend_case(128, 8, 2, 16, torch.bfloat16, [100, 33], [1, 1], q_scale=q_scale, seed=4)


def test_attend_layer_of_a_pool():
    _attend_case(128, 8, 2, 16, torch.bfloat16, [100, 33], [1, 1], layers=3, layer=2, seed=4)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hk,lens,new", [
    (8, 1, [40], [40]), (8, 1, [16], [16]), (5, 1, [150, 30, 200], [37, 30, 1]), (2, 2, [130, 128, 129, 127], [130, 64, 65, 127]),
    (16, 2, [300, 0, 17, 5], [20, 0, 17, 9]), (1, 1, [700], [260]), (7, 1, [64, 65], [19, 65])])
def test_attend_prompts(d, hq, hk, lens, new):
    _attend_case(d, hq, hk, 16, torch.bfloat16, lens, new, seed=d + hq)


@pytest.mark.parametrize("window", [1, 15, 64, 200])
def test_attend_prompts_window_blocks_and_half(window):
    _attend_case(128, 4, 1, 32, torch.float16, [150, 90, 333], [150, 33, 40], window=window, seed=window)
    _attend_case(64, 4, 2, 48, torch.bfloat16, [150, 90, 33], [15, 90, 40], window=window, seed=window, layers=2, layer=1)


def test_attend_prompts_whole_gpu_and_few_units_one_workspace():
    # more thread blocks than the GPU holds, then one unit whose keys are split, then single tokens, all on one workspace
    ws = _attend_case(128, 32, 32, 16, torch.bfloat16, [40] * 12, [40] * 12, seed=1)
    _attend_case(128, 8, 1, 16, torch.bfloat16, [1500], [5], seed=2, ws=ws)
    _attend_case(256, 8, 1, 16, torch.bfloat16, [900], [5], seed=2, ws=ws)
    _attend_case(128, 8, 1, 16, torch.bfloat16, [1500], [1], seed=2, ws=ws)
    _attend_case(64, 8, 2, 16, torch.bfloat16, [800, 10], [30, 10], seed=3, ws=ws)


@pytest.mark.parametrize("q_scale", [1e-6, 1e4])
def test_attend_prompts_query_sizes(q_scale):
    _attend_case(128, 8, 2, 16, torch.bfloat16, [100, 33], [30, 10], q_scale=q_scale, seed=4)


@pytest.mark.parametrize("n", [30, 50])
def test_attend_prompts_sharp_scores(n):
    # scores that grow along the keys: references move again and again, in the first 32 keys of a block and behind
    rng = np.random.default_rng(0)
    d, bs, length = 64, 16, 400
    lens, new, tables, start, batch = _batch([length], [n], bs, 25, rng)
    pool = ref.Pool(1, 25, 1, d, bs)
    base = rng.standard_normal(d)
    q = torch.from_numpy(np.tile(base, (n, 1, 1)) + 0.1 * rng.standard_normal((n, 1, d))).bfloat16().cuda()
    for p in range(length):
        pool.write(0, 0, tables[0, p // bs], p, (base * (p / 16)).astype(np.float32)[None])
        pool.write(0, 1, tables[0, p // bs], p, rng.standard_normal((1, d)).astype(np.float32))
    buf, dev = _dev_pool(pool)
    out, lse = torch.empty_like(q), torch.empty(n, 1, device="cuda")
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace(), lse=lse)
    _check(out, lse, q, pool, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)


def test_attend_prompts_bad_blocks():
    rng = np.random.default_rng(6)
    d, bs, hk, n = 128, 16, 1, 24
    pool = _filled(6, hk, d, bs, rng)
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, new = np.array([90, 70], dtype=np.int32), np.array([n, n], dtype=np.int32)
    tables = np.array([[0, 77, 2, 1, 4, 5], [-1, 1, 2, 3, 1 << 30, 0]], dtype=np.int32)
    start = np.array([0, n, 2 * n], dtype=np.int32)
    batch = _dev_batch(lens, tables, start, new, error)
    buf, dev = _dev_pool(pool)
    q = torch.randn(2 * n, 4, d, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(2 * n, 4, device="cuda")
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace(), lse=lse)
    _check(out, lse, q, pool, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)
    assert int(error) == 8


def test_attend_sharp_scores():
    # one key far above the others, at the end: every tile raises the reference
    rng = np.random.default_rng(0)
    d, bs, length = 64, 16, 320
    lens, new, tables, start, batch = _batch([length], [1], bs, 20, rng)
    pool = ref.Pool(1, 20, 1, d, bs)
    q = torch.randn(1, 1, d, device="cuda").bfloat16()
    qf = q.float().cpu().numpy()[0, 0]
    for p in range(length):
        pool.write(0, 0, tables[0, p // bs], p, (qf * (p / 16)).astype(np.float32)[None])
        pool.write(0, 1, tables[0, p // bs], p, rng.standard_normal((1, d)).astype(np.float32))
    buf, dev = _dev_pool(pool)
    out, lse = torch.empty_like(q), torch.empty(1, 1, device="cuda")
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace(), lse=lse)
    _check(out, lse, q, pool, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)


def test_attend_nan_stays_in_its_sequence():
    rng = np.random.default_rng(0)
    d, bs = 128, 16
    lens, new, tables, start, batch = _batch([40, 50], [1, 1], bs, 8, rng)
    pool = _filled(8, 1, d, bs, rng)
    pool.write(0, 1, tables[0, 1], 20, np.full((1, d), np.nan, dtype=np.float32))
    buf, dev = _dev_pool(pool)
    q = torch.randn(2, 4, d, device="cuda").bfloat16()
    q[1, 2] = math.nan
    out = torch.empty_like(q)
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace())
    bad = torch.isnan(out).all(-1).cpu().numpy()
    assert bad.tolist() == [[True] * 4, [False, False, True, False]]


def test_attend_bad_blocks_and_lengths():
    rng = np.random.default_rng(6)
    d, bs, hk = 128, 16, 1
    pool = _filled(6, hk, d, bs, rng)
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, new = np.array([40, 90, -3], dtype=np.int32), np.array([1, 1, 1], dtype=np.int32)
    tables = np.array([[0, 77, 2], [3, 4, 5], [1, 1, 1]], dtype=np.int32)
    start = np.arange(4, dtype=np.int32)
    batch = _dev_batch(lens, tables, start, new, error)
    buf, dev = _dev_pool(pool)
    q = torch.randn(3, 4, d, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(3, 4, device="cuda")
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace(), lse=lse)
    _check(out, lse, q, pool, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)
    assert int(error) == 2 | 8
    assert (out[2] == 0).all() and torch.isinf(lse[2]).all()


def test_attend_offsets_beyond_32_bits():
    rng = np.random.default_rng(8)
    d, bs, hk, blocks = 128, 16, 2, 4
    pool = _filled(blocks, hk, d, bs, rng)
    step = 1_700_000_000 // 16 * 16
    one = pool.bytes[0, 0, 0].size
    buf = torch.zeros(2 * one + blocks * step, dtype=torch.uint8, device="cuda")
    for b in range(blocks):
        for kv in (0, 1):
            buf[b * step + kv * one:b * step + (kv + 1) * one] = torch.from_numpy(pool.bytes[0, kv, b].reshape(-1)).cuda()
    dev = remp.make_kvq_pool(buf, blocks, hk, d, bs, strides={"layer": 2 * one, "kv": one, "block": step})
    lens, new, tables, start, batch = _batch([63], [1], bs, blocks, rng)
    q = torch.randn(1, 8, d, device="cuda").bfloat16()
    out = torch.empty_like(q)
    remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, remp.make_kvq_workspace())
    _check(out, None, q, pool, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)
    x = torch.randn(1, hk, d, device="cuda").bfloat16()
    remp.remp_kvq_append(dev, batch, None, x, x, None)
    back = torch.empty_like(x)
    remp.remp_kvq_read(dev, batch, None, back)
    assert (back - x).abs().max() < 0.4


def test_streams_and_graph():
    rng = np.random.default_rng(9)
    d, bs, hk = 128, 16, 2
    pool = _filled(30, hk, d, bs, rng)
    lens, new, tables, start, batch = _batch([100, 200], [1, 1], bs, 30, rng)
    buf, dev = _dev_pool(pool)
    x = torch.randn(2, 12, d, device="cuda").bfloat16()
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    out, again = torch.empty(2, 8, d, dtype=x.dtype, device="cuda"), torch.empty(2, 8, d, dtype=x.dtype, device="cuda")
    ws, other_ws = remp.make_kvq_workspace(), remp.make_kvq_workspace()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        remp.remp_kvq_append(dev, batch, None, k, v, None)
        remp.remp_kvq_attend(dev, batch, q, out, d ** -0.5, ws)
    side.synchronize()
    p2 = ref.Pool(1, 30, hk, d, bs)
    p2.bytes[:] = buf.cpu().numpy().reshape(p2.bytes.shape)
    _check(out, None, q, p2, 0, lens, new, tables, d ** -0.5, 0, torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        remp.remp_kvq_append(dev, batch, None, k, v, None)
        remp.remp_kvq_attend(dev, batch, q, again, d ** -0.5, other_ws)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again)
