"""What the serving calls refuse, before anything is enqueued: host checks only, so no GPU is needed."""
import ctypes as C

import numpy as np
import pytest

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200 import _lib
from paper_2606_18741_b200._lib import (RempBlockTables, RempKvqBatch, RempKvqPool, RempKvqRows, RempKvqTransform, RempModelShape,
                                        RempShard, RempTopo)

PTR = 1 << 20  # stands for device memory; never dereferenced


def _pool(**kw):
    sh = RempShard(kw.pop("base", PTR), kw.pop("blocks", 8), *[kw.pop(k, 0) for k in ("s_layer", "s_kv", "s_block", "s_head", "s_token")])
    return RempKvqPool(sh, kw.pop("layer", 0), kw.pop("kv_heads", 2), kw.pop("head_dim", 128), kw.pop("block_size", 16))


def _batch(tokens=4, queries=2, seqs=2, width=4, lens=PTR, tables=PTR, start=PTR):
    return RempKvqBatch(RempBlockTables(seqs, width, lens, tables), start, tokens, queries, None)


def _rows(data=PTR, token=1024, head=128):
    return RempKvqRows(data, token, head)


def _append(pool=None, batch=None, q=None, k=None, v=None, q_out=None, q_heads=0, dtype=1, tr=None):
    return _lib.load().remp_kvq_append(pool or _pool(), batch or _batch(), q, k or _rows(), v or _rows(), q_out, q_heads, dtype, tr, None)


def _attend(pool=None, batch=None, q=None, out=None, heads=4, dtype=1, scale=1.0, window=0, ws=PTR):
    return _lib.load().remp_kvq_attend(pool or _pool(), batch or _batch(), q or _rows(), out or _rows(), heads, dtype, scale, window, None, ws, None)


ARG, SHAPE = remp.REMP_ERR_INVALID_ARG, remp.REMP_ERR_SHAPE


@pytest.mark.parametrize("kw,status", [
    ({"head_dim": 96}, SHAPE), ({"head_dim": 0}, SHAPE), ({"block_size": 8}, SHAPE), ({"block_size": 24}, SHAPE), ({"block_size": 0}, SHAPE),
    ({"kv_heads": 0}, SHAPE), ({"layer": -1}, ARG), ({"base": None}, ARG), ({"base": PTR + 8}, SHAPE), ({"blocks": -1}, ARG),
    ({"s_head": 128}, SHAPE), ({"s_block": 16}, SHAPE), ({"s_token": 128}, SHAPE), ({"s_kv": 24}, SHAPE)])
def test_pools(kw, status):
    assert _append(pool=_pool(**kw)) == status
    assert _attend(pool=_pool(**kw)) == status
    assert _lib.load().remp_kvq_read(_pool(**kw), _batch(), _rows(), None, 1, None) == status
    assert remp.remp_last_error()


@pytest.mark.parametrize("kw", [{"tokens": -1}, {"queries": -1}, {"seqs": -1}, {"width": -1}, {"lens": None}, {"tables": None}, {"start": None}])
def test_batches(kw):
    assert _append(batch=_batch(**kw)) == ARG
    assert _attend(batch=_batch(**kw)) == ARG


def test_append_rows_and_transform():
    assert _append(k=_rows(PTR + 2)) == SHAPE
    assert _append(v=_rows(token=1020)) == SHAPE
    assert _append(v=_rows(head=64)) == SHAPE
    assert _append(dtype=3) == ARG
    assert _append(q_heads=2) == ARG and _append(q=_rows(), q_heads=2) == ARG and _append(q=_rows(), q_out=_rows()) == ARG
    assert _append(tr=RempKvqTransform(None, None, PTR, None, 1e-6, 10, 24, 0)) == SHAPE
    assert _append(tr=RempKvqTransform(None, None, PTR, None, 1e-6, 10, 144, 0)) == SHAPE
    assert _append(tr=RempKvqTransform(PTR + 4, None, None, None, 1e-6, 0, 0, 0)) == SHAPE
    assert _append(tr=RempKvqTransform(PTR, None, None, None, -1.0, 0, 0, 0)) == ARG
    assert _append(tr=RempKvqTransform(PTR, None, None, None, float("nan"), 0, 0, 0)) == ARG
    assert _append(batch=_batch(tokens=0)) == remp.REMP_OK


def test_attend_arguments():
    assert _attend(heads=3) == SHAPE and _attend(heads=0) == SHAPE
    assert _attend(dtype=0) == ARG and _attend(window=-1) == ARG and _attend(ws=None) == ARG and _attend(ws=PTR + 16) == ARG
    assert _attend(batch=_batch(queries=0)) == ARG
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _attend(scale=scale) == ARG
    assert _attend(q=_rows(PTR + 8)) == SHAPE and _attend(out=_rows(None)) == ARG
    assert _attend(batch=_batch(tokens=0)) == remp.REMP_OK
    assert _lib.load().remp_kvq_workspace_bytes() > 0


def test_token_bytes():
    assert [remp.remp_kvq_token_bytes(d) for d in (64, 128, 256)] == [36, 72, 144]
    with pytest.raises(remp.RempError):
        remp.remp_kvq_token_bytes(80)


def test_pages_arguments():
    L = _lib.load()
    ok = dict(lens=PTR, tabs=PTR, n=3, width=4, bs=16, a=PTR, b=PTR, m=2, refs=PTR, out=PTR, nb=9, pairs=PTR, result=PTR)

    def fork(**kw):
        x = {**ok, **kw}
        return L.remp_pages_fork(x["lens"], x["tabs"], x["n"], x["width"], x["bs"], x["a"], x["b"], x["m"], x["refs"], x["out"], x["nb"], x["pairs"], x["result"], None)

    def free(**kw):
        x = {**ok, **kw}
        return L.remp_pages_free(x["lens"], x["tabs"], x["n"], x["width"], x["bs"], x["a"], x["refs"], x["nb"], x["b"], x["pairs"], x["out"], x["result"], None)

    def compact(**kw):
        x = {"m": 4, **kw}
        x = {**ok, **x}
        return L.remp_pages_compact(x["lens"], x["tabs"], x["n"], x["width"], x["bs"], x["refs"], x["nb"], x["b"], x["out"], x["pairs"], x["m"], x["result"], None)

    for f in (fork, free, compact):
        for bad in ({"lens": None}, {"tabs": None}, {"n": -1}, {"width": -1}, {"nb": -1}, {"refs": None}, {"out": None}, {"result": None}):
            assert f(**bad) == ARG, (f, bad)
        assert f(bs=0) == SHAPE
    assert fork(a=None) == ARG and fork(b=None) == ARG and fork(pairs=None) == ARG and fork(m=-1) == ARG and fork(pairs=PTR + 4) == SHAPE
    assert free(a=None) == ARG and free(b=None) == ARG and free(pairs=None) == ARG
    assert compact(m=3) == ARG and compact(pairs=None) == ARG and compact(b=None) == ARG and compact(pairs=PTR + 4) == SHAPE

    shape, topo = RempModelShape(2, 2, 64, 16, 2), RempTopo(1, 1, None)

    def copy(topo=topo, shape=shape, shard=RempShard(PTR, 4, 0, 0, 0, 0, 0), pairs=PTR, count=PTR, m=2):
        arr = (RempShard * 4)(*[shard] * 4)
        return L.remp_pages_copy(C.byref(topo), C.byref(shape), arr, pairs, count, m, None)

    assert copy(pairs=None) == ARG and copy(count=None) == ARG and copy(m=-1) == ARG and copy(pairs=PTR + 4) == SHAPE
    assert copy(topo=RempTopo(3, 1, None)) == remp.REMP_ERR_INVALID_TOPOLOGY
    assert copy(shape=RempModelShape(2, 2, 64, 16, 3)) == SHAPE
    assert copy(shard=RempShard(None, 4, 0, 0, 0, 0, 0)) == ARG
    assert copy(shard=RempShard(PTR, 4, 0, 0, 0, 512, 0)) == SHAPE  # heads inside one another
    assert copy(m=0) == remp.REMP_OK and copy(shard=RempShard(None, 0, 0, 0, 0, 0, 0)) == remp.REMP_OK


def test_places_are_permutations():
    from tests import kvq_reference as ref
    for d in (64, 128, 256):
        for is_v in (False, True):
            assert sorted(ref.place_of(d, is_v)) == list(range(d))


def test_quantiser_of_the_reference():
    """The tests' quantiser: within half a step of every value (and the rounding of the step)."""
    from tests import kvq_reference as ref
    x = (np.random.default_rng(0).standard_normal((50, 128)) * 3).astype(np.float32)
    c, s, m = ref.quantise(x)
    sf, mf = np.repeat(ref.bf16_value(s), 64, -1), np.repeat(ref.bf16_value(m), 64, -1)
    assert (np.abs(c * sf + mf - x) <= 0.5 * sf * (1 + 2 ** -6) + 2 ** -8 * np.abs(mf)).all()


def test_numbers_close_to_2_to_the_31():
    assert _attend(batch=_batch(tokens=2 ** 31 - 1)) == SHAPE and _append(batch=_batch(seqs=2 ** 31 - 1)) == SHAPE
    L = _lib.load()
    assert L.remp_pages_compact(PTR, PTR, 3, 4, 16, PTR, 9, PTR, PTR, PTR, 2 ** 31 - 1, PTR, None) == SHAPE


def test_outputs_whose_rows_overlap():
    # inputs may repeat a head or a token, outputs may not
    assert _attend(out=_rows(head=0)) == SHAPE and _attend(out=_rows(token=0)) == SHAPE and _attend(out=_rows(token=64)) == SHAPE
    assert _append(q=_rows(), q_out=_rows(head=0), q_heads=2) == SHAPE and _append(q=_rows(), q_out=_rows(token=0), q_heads=2) == SHAPE
    assert _lib.load().remp_kvq_read(_pool(), _batch(), _rows(token=0), None, 1, None) == SHAPE
    assert _append(v=_rows(token=0), k=_rows(head=0), batch=_batch(tokens=0)) == remp.REMP_OK
