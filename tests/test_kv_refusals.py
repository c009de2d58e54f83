"""What the calls on a cache of 16-bit values, and the verification of drafts, refuse before anything is enqueued: host checks only,
so no GPU is needed."""
import pytest

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200 import _lib
from paper_2606_18741_b200._lib import RempBlockTables, RempKvqBatch, RempKvqPool, RempKvqRows, RempKvqTransform, RempShard

PTR = 1 << 20  # stands for device memory; never dereferenced
ARG, SHAPE, OK = remp.REMP_ERR_INVALID_ARG, remp.REMP_ERR_SHAPE, remp.REMP_OK


def _pool(**kw):
    sh = RempShard(kw.pop("base", PTR), kw.pop("blocks", 8), *[kw.pop(k, 0) for k in ("s_layer", "s_kv", "s_block", "s_head", "s_token")])
    return RempKvqPool(sh, kw.pop("layer", 0), kw.pop("kv_heads", 2), kw.pop("head_dim", 128), kw.pop("block_size", 16))


def _batch(tokens=4, queries=2, seqs=2, width=4, lens=PTR, tables=PTR, start=PTR):
    return RempKvqBatch(RempBlockTables(seqs, width, lens, tables), start, tokens, queries, None)


def _rows(data=PTR, token=1024, head=128):
    return RempKvqRows(data, token, head)


def _append(pool=None, batch=None, q=None, k=None, v=None, q_out=None, q_heads=0, dtype=1, tr=None):
    return _lib.load().remp_kv_append(pool or _pool(), batch or _batch(), q, k or _rows(), v or _rows(), q_out, q_heads, dtype, tr, None)


def _attend(pool=None, batch=None, q=None, out=None, heads=4, dtype=1, scale=1.0, window=0, first=0, ws=PTR):
    return _lib.load().remp_kv_attend(pool or _pool(), batch or _batch(), q or _rows(), out or _rows(), heads, dtype, scale, window, first, None, ws, None)


def _weigh(pool=None, batch=None, q=None, heads=4, dtype=1, scale=1.0, window=0, first=0, lse=PTR, weights=PTR, stride=64):
    return _lib.load().remp_kv_weigh(pool or _pool(), batch or _batch(), q or _rows(), heads, dtype, scale, window, first, lse, weights, stride, 0, None)


def _evict(pool=None, seqs=2, width=4, lens=PTR, tables=PTR, keep=PTR, first=0, recent=0, weights=PTR, out=PTR, stride=64, kept=PTR, kept_stride=32, most=64,
           null_tables=False):
    return _lib.load().remp_kv_evict(pool or _pool(), None if null_tables else RempBlockTables(seqs, width, lens, tables), keep, first, recent, weights, out, stride, kept,
                                     kept_stride, most, None, None)


def _verify(n=2, m=3, vocab=100, start=PTR, drafts=PTR, target=PTR, st=100, draft=PTR, sd=100, dtype=3, accept=PTR, pick=PTR, tokens=PTR, accepted=PTR):
    return _lib.load().remp_draft_verify(n, m, vocab, start, drafts, target, st, draft, sd, dtype, accept, pick, tokens, accepted, None, None)


CALLS = (_append, _attend, _weigh)


@pytest.mark.parametrize("kw,status", [
    ({"head_dim": 96}, SHAPE), ({"head_dim": 0}, SHAPE), ({"block_size": 8}, SHAPE), ({"block_size": 24}, SHAPE), ({"block_size": 0}, SHAPE),
    ({"kv_heads": 0}, SHAPE), ({"layer": -1}, ARG), ({"base": None}, ARG), ({"base": PTR + 8}, SHAPE), ({"blocks": -1}, ARG),
    ({"s_head": 128}, SHAPE), ({"s_head": 1024}, SHAPE), ({"s_block": 16}, SHAPE), ({"s_token": 272 + 8}, SHAPE), ({"s_token": 272}, SHAPE), ({"s_kv": 24}, SHAPE),
    ({"s_head": 256, "s_token": 256}, SHAPE)])
def test_pools(kw, status):
    for call in CALLS + (_evict,):
        assert call(pool=_pool(**kw)) == status
    assert remp.remp_last_error()


@pytest.mark.parametrize("kw", [{"tokens": -1}, {"queries": -1}, {"seqs": -1}, {"width": -1}, {"lens": None}, {"tables": None}, {"start": None}])
def test_batches(kw):
    for call in CALLS:
        assert call(batch=_batch(**kw)) == ARG


def test_numbers_close_to_2_to_the_31():
    for call in CALLS:
        assert call(batch=_batch(seqs=2 ** 31 - 1)) == SHAPE and call(batch=_batch(tokens=2 ** 31 - 1)) == SHAPE
    assert _attend(heads=2 ** 31 - 2) == SHAPE and _weigh(heads=2 ** 31 - 2) == SHAPE
    assert _evict(seqs=2 ** 31 - 1) == SHAPE
    assert _verify(n=2 ** 31 - 1) == SHAPE and _verify(m=2 ** 31 - 1) == SHAPE and _verify(vocab=2 ** 31 - 1) == SHAPE


def test_append_rows_and_transform():
    assert _append(k=_rows(PTR + 2)) == SHAPE
    assert _append(v=_rows(token=1020)) == SHAPE
    assert _append(v=_rows(head=64)) == SHAPE
    assert _append(dtype=3) == ARG
    assert _append(q_heads=2) == ARG and _append(q=_rows(), q_heads=2) == ARG and _append(q=_rows(), q_out=_rows()) == ARG
    assert _append(q=_rows(), q_out=_rows(head=0), q_heads=2) == SHAPE
    assert _append(tr=RempKvqTransform(None, None, PTR, None, 1e-6, 10, 24, 0)) == SHAPE
    assert _append(tr=RempKvqTransform(PTR + 4, None, None, None, 1e-6, 0, 0, 0)) == SHAPE
    assert _append(tr=RempKvqTransform(PTR, None, None, None, -1.0, 0, 0, 0)) == ARG
    assert _append(batch=_batch(tokens=0)) == OK


def test_attend_and_weigh_arguments():
    for call in (_attend, _weigh):
        assert call(heads=3) == SHAPE and call(heads=0) == SHAPE
        assert call(dtype=0) == ARG and call(dtype=3) == ARG and call(window=-1) == ARG and call(first=-1) == ARG
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            assert call(scale=scale) == ARG
        assert call(q=_rows(PTR + 8)) == SHAPE
        assert call(batch=_batch(tokens=0)) == OK
    assert _attend(ws=None) == ARG and _attend(ws=PTR + 16) == ARG and _attend(out=_rows(None)) == ARG and _attend(out=_rows(head=0)) == SHAPE
    assert _attend(batch=_batch(queries=0)) == ARG
    assert _weigh(lse=None) == ARG and _weigh(weights=None) == ARG and _weigh(stride=-1) == ARG
    assert _lib.load().remp_kv_workspace_bytes() > 0


def test_evict_arguments():
    assert _evict(null_tables=True) == ARG
    for bad in ({"seqs": -1}, {"width": -1}, {"lens": None}, {"tables": None}, {"keep": None}, {"first": -1}, {"recent": -1}, {"weights": None}, {"out": None},
                {"stride": -1}, {"kept": None}, {"kept_stride": -1}, {"most": -1}):
        assert _evict(**bad) == ARG, bad
    assert _evict(most=65) == SHAPE and _evict(most=2 ** 18 + 1, stride=2 ** 20) == SHAPE
    assert _evict(seqs=0) == OK


def test_verify_arguments():
    for bad in ({"n": -1}, {"m": -1}, {"vocab": 0}, {"dtype": 0}, {"dtype": 4}, {"start": None}, {"drafts": None}, {"target": None}, {"accept": None}, {"pick": None},
                {"tokens": None}, {"accepted": None}):
        assert _verify(**bad) == ARG, bad
    assert _verify(st=99) == SHAPE and _verify(sd=99) == SHAPE and _verify(target=PTR + 2) == SHAPE and _verify(draft=PTR + 1, dtype=1) == SHAPE
    assert _verify(n=0) == OK
