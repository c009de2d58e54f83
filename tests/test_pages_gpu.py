"""Page management on the GPU against plain loops: whole numbers and bytes, compared exactly."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200.synth import Shape, Topo
from tests import kvq_reference as ref

pytestmark = pytest.mark.gpu


def _d(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _state(n, extra, max_len, bs, spare, seed, share=True):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, max_len + 1, n).astype(np.int32)
    need = -(-lens // bs)
    blocks = int(need.sum()) + spare
    width = max(1, int(need.max())) + 1
    ids = rng.permutation(blocks)
    tables = np.full((n + extra, width), -1, dtype=np.int32)
    at = 0
    for s in range(n):
        tables[s, :need[s]] = ids[at:at + need[s]]
        at += need[s]
    if share:
        for a in range(0, n - 1, 3):
            both = int(min(lens[a], lens[a + 1])) // bs
            tables[a + 1, :both] = tables[a, :both]
    lens = np.concatenate([lens, np.zeros(extra, dtype=np.int32)]).astype(np.int32)
    return rng, lens, tables, ref.refs_of(lens, tables, bs, blocks), blocks


# sizes on both sides of the one-launch rule
SIZES = [(1, 1, 5, 16, 3), (3, 4, 40, 16, 6), (20, 50, 300, 16, 55), (64, 300, 900, 16, 300), (40, 1300, 64, 32, 1400), (700, 40, 400, 16, 9000)]


@pytest.mark.parametrize("n,kids,max_len,bs,spare", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_fork(n, kids, max_len, bs, spare, in_place):
    rng, lens, tables, refs, blocks = _state(n, kids, max_len, bs, spare, n + kids)
    parents = rng.integers(0, n, kids).astype(np.int32)
    children = (n + rng.permutation(kids)).astype(np.int32)
    want = ref.fork(lens, tables, bs, parents, children, refs)
    dl, dt, dr = _d(lens), _d(tables), _d(refs)
    out = dr if in_place else torch.full_like(dr, -9)
    pairs, result = torch.full((kids, 2), -9, dtype=torch.int32, device="cuda"), torch.full((2,), -9, dtype=torch.int32, device="cuda")
    remp.remp_pages_fork(dl, dt, bs, _d(parents), _d(children), dr, out, pairs, result)
    got = [x.cpu().numpy() for x in (dl, dt, out, pairs)]
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    assert result.tolist() == want[4]
    assert np.array_equal(got[2], ref.refs_of(got[0], got[1], bs, blocks))


@pytest.mark.parametrize("kids", [6, 1200])
def test_fork_without_room_or_with_bad_parents_changes_nothing(kids):
    rng, lens, tables, refs, blocks = _state(9, kids, 50, 16, 2, 1, share=False)
    lens[0] = 33
    for parents, bits in ((np.zeros(kids, dtype=np.int32), 1), (np.full(kids, 9 + kids, dtype=np.int32), 2)):
        need = -(-lens // 16)
        row = tables.copy()
        dl, dt, dr = _d(lens), _d(row), _d(refs)
        out, pairs, result = torch.empty_like(dr), torch.zeros(kids, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        remp.remp_pages_fork(dl, dt, 16, _d(parents), _d(np.arange(9, 9 + kids).astype(np.int32)), dr, out, pairs, result)
        assert result.tolist() == [0, bits] and need.size
        assert np.array_equal(dl.cpu().numpy(), lens) and np.array_equal(dt.cpu().numpy(), row)
        assert torch.equal(out, dr) and (pairs == -1).all()


@pytest.mark.parametrize("n,kids,max_len,bs,spare", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_free_and_compact(n, kids, max_len, bs, spare, in_place):
    rng, lens, tables, refs, blocks = _state(n, 2, max_len, bs, spare, n)
    done = (rng.random(n + 2) < 0.4).astype(np.int32)
    w_lens, w_tables, w_refs, w_res = ref.free(lens, tables, bs, done, refs)
    dl, dt, dr = _d(lens), _d(tables), _d(refs)
    ol, ot, orf = (dl, dt, dr) if in_place else tuple(torch.full_like(x, -9) for x in (dl, dt, dr))
    result = torch.full((2,), -9, dtype=torch.int32, device="cuda")
    remp.remp_pages_free(dl, dt, bs, _d(done), dr, ol, ot, orf, result)
    assert result.tolist() == w_res
    for g, w in ((ol, w_lens), (ot, w_tables), (orf, w_refs)):
        assert np.array_equal(g.cpu().numpy(), w)
    m = blocks // 2 + 3
    c_tables, c_refs, c_pairs, c_res = ref.compact(w_lens, w_tables, bs, w_refs, m)
    pairs = torch.full((m, 2), -9, dtype=torch.int32, device="cuda")
    ot2, or2 = (ot, orf) if in_place else (torch.full_like(ot, -9), torch.full_like(orf, -9))
    remp.remp_pages_compact(ol, ot, bs, orf, ot2, or2, pairs, result)
    assert result.tolist() == c_res
    for g, w in ((ot2, c_tables), (or2, c_refs), (pairs, c_pairs)):
        assert np.array_equal(g.cpu().numpy(), w)
    # nothing moves a second time
    remp.remp_pages_compact(ol, ot2, bs, or2, ot2, or2, pairs, result)
    assert result.tolist() == [0, 0] and np.array_equal(ot2.cpu().numpy(), c_tables) and (pairs == -1).all()


def test_free_and_compact_report_bad_entries():
    lens, tables = np.array([20, 20, 99], dtype=np.int32), np.array([[0, 7], [1, 2], [3, 3]], dtype=np.int32)
    refs = np.array([1, 1, 0, 1], dtype=np.int32)  # block 2's count is wrong, block 7 outside, sequence 2 too long for its row
    dl, dt, dr = _d(lens), _d(tables), _d(refs)
    result = torch.zeros(2, dtype=torch.int32, device="cuda")
    remp.remp_pages_free(dl, dt, 16, _d(np.array([1, 0, 0], dtype=np.int32)), dr, dl.clone(), torch.empty_like(dt), torch.empty_like(dr), result)
    assert result.tolist() == [1, 8]
    remp.remp_pages_free(dl, dt, 16, _d(np.array([0, 1, 1], dtype=np.int32)), dr, dl.clone(), torch.empty_like(dt), torch.empty_like(dr), result)
    assert result.tolist() == [1, 8 | 2]
    pairs, out = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.empty_like(dt)
    remp.remp_pages_compact(dl, dt, 16, dr, out, torch.empty_like(dr), pairs, result)
    assert result.tolist() == [1, 8 | 2] and pairs.tolist() == [[3, 2], [-1, -1]]
    assert out.tolist() == tables.tolist()


def _copy_case(T, m, nb, strides, seed, n, max_pairs):
    rng = np.random.default_rng(seed)
    bufs, shards = [], []
    for r in range(T.tp * T.pp):
        lo, hi, h0, h1 = remp.remp_rank_ownership(T, m, r)
        size = strides["bytes"] if strides else remp.remp_shard_bytes(T, m, r, nb)
        bufs.append(torch.from_numpy(rng.integers(0, 256, size, dtype=np.uint8)).cuda())
    shards = remp.make_shards(bufs, [nb] * len(bufs), [strides["st"]] * len(bufs) if strides else None)
    ids = rng.permutation(nb)
    pairs = np.full((max_pairs, 2), -1, dtype=np.int32)
    pairs[:n] = ids[:2 * n].reshape(n, 2)
    pairs[n:] = [0, 1]  # behind the count: not read
    before = [b.cpu().numpy() for b in bufs]
    remp.remp_pages_copy(T, m, shards, _d(pairs), _d(np.array([n, 0], dtype=np.int32)))
    hs = m.block_size * m.head_dim * m.elem_bytes
    row = m.head_dim * m.elem_bytes
    for r, b in enumerate(bufs):
        lo, hi, h0, h1 = remp.remp_rank_ownership(T, m, r)
        st = dict(strides["st"]) if strides else {}
        sb = st.get("block", (h1 - h0) * hs)
        sk = st.get("kv", nb * sb)
        sl = st.get("layer", 2 * sk)
        sh, stk = st.get("head", hs), st.get("token", row)
        want = before[r].copy()
        for l in range(hi - lo):
            for kv in range(2):
                for s, d in pairs[:n]:
                    for h in range(h1 - h0):
                        for t in range(m.block_size):
                            o = l * sl + kv * sk + h * sh + t * stk
                            want[o + d * sb:o + d * sb + row] = before[r][o + s * sb:o + s * sb + row]
        assert np.array_equal(b.cpu().numpy(), want), r


@pytest.mark.parametrize("T", [Topo(1, 1), Topo(2, 2), Topo(8, 1)])
@pytest.mark.parametrize("m", [Shape(3, 4, 64, 16, 2), Shape(2, 4, 72, 16, 1), Shape(2, 4, 9, 16, 1), Shape(2, 4, 128, 64, 2)])
def test_copy_dense(T, m):
    for n in (0, 1, 5):
        _copy_case(T, m, 11, None, n, n, 7)


def test_copy_strided():
    m = Shape(2, 3, 16, 16, 2)
    hs, row = 16 * 32, 32
    token_major = {"st": {"head": row, "token": 3 * row, "block": 3 * hs}, "bytes": 2 * 2 * 9 * 3 * hs}
    padded_heads = {"st": {"head": hs + 64, "block": 3 * hs + 256}, "bytes": 2 * 2 * 9 * (3 * hs + 256)}
    padded_tokens = {"st": {"head": row, "token": 3 * row + 16, "block": 16 * (3 * row + 16)}, "bytes": 2 * 2 * 9 * 16 * (3 * row + 16)}
    for st in (token_major, padded_heads, padded_tokens):
        _copy_case(Topo(1, 1), m, 9, st, 1, 4, 4)


def test_copy_skips_ids_outside_the_pool():
    m, T = Shape(1, 1, 16, 16, 1), Topo(1, 1)
    buf = torch.arange(2 * 3 * 256, dtype=torch.int32, device="cuda").to(torch.uint8)
    before = buf.clone()
    pairs = _d(np.array([[0, 3], [-1, 1], [7, 2]], dtype=np.int32))
    remp.remp_pages_copy(T, m, remp.make_shards([buf], [3]), pairs, _d(np.array([99], dtype=np.int32)))
    assert torch.equal(buf, before)


def test_many_ranks_in_one_call():
    m, T = Shape(60, 1, 16, 16, 1), Topo(1, 60)
    _copy_case(T, m, 4, None, 0, 2, 2)
