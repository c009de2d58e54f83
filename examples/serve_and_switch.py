"""Serving from a 4-bit paged cache, and a topology switch in the middle of it.

Prompts are written and attended, forked into samples, decoded for a few steps; finished samples give their pages back, the
cache is compacted and re-sharded from TP1PP1 to TP2PP2, and decoding goes on in the new layout. Random weights stand
in for a model: what is shown is the order of the calls. Run on a GPU: python examples/serve_and_switch.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_18741_b200 as remp  # noqa: E402
from paper_2606_18741_b200.synth import Shape, Topo  # noqa: E402

LAYERS, Q_HEADS, KV_HEADS, DIM, BLOCK, WIDTH = 4, 8, 2, 128, 16, 16
PROMPTS, SAMPLES, STEPS = (37, 90, 64), 3, 5


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Ranks:
    """The pools of every rank of a topology, and the calls of one model step on them."""

    def __init__(self, topo, blocks):
        self.topo, self.blocks = topo, blocks
        # a head slice is opaque bytes to the migration: token rows of remp_kvq_token_bytes, one byte an element
        self.shape = Shape(LAYERS, KV_HEADS, remp.remp_kvq_token_bytes(DIM), BLOCK, 1)
        n = topo.tp * topo.pp
        self.pools = [torch.zeros(remp.remp_shard_bytes(topo, self.shape, r, blocks), dtype=torch.uint8, device="cuda") for r in range(n)]
        self.owned = [remp.remp_rank_ownership(topo, self.shape, r) for r in range(n)]
        self.workspace = remp.make_kvq_workspace()
        self.norm = torch.ones(DIM, device="cuda")
        at = torch.arange(4096, device="cuda", dtype=torch.float64)[:, None]
        angle = at * 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda", dtype=torch.float64) / DIM)
        self.rope = torch.cat((angle.cos(), angle.sin()), 1).float()

    def shards(self):
        return remp.make_shards(self.pools, [self.blocks] * len(self.pools))

    def step(self, batch, qkv):
        """qkv [layers][tokens][heads][dim] -> attention outputs, same query shape: append, then attend, layer by layer."""
        out = torch.empty(LAYERS, qkv.shape[1], Q_HEADS, DIM, dtype=qkv.dtype, device="cuda")
        group = Q_HEADS // KV_HEADS
        for pool, (l0, l1, h0, h1) in zip(self.pools, self.owned):
            for layer in range(l0, l1):
                cache = remp.make_kvq_pool(pool, self.blocks, h1 - h0, DIM, BLOCK, layer=layer - l0)
                q = qkv[layer, :, h0 * group:h1 * group]
                k = qkv[layer, :, Q_HEADS + h0:Q_HEADS + h1]
                v = qkv[layer, :, Q_HEADS + KV_HEADS + h0:Q_HEADS + KV_HEADS + h1]
                turned = torch.empty_like(q, memory_format=torch.contiguous_format)
                remp.remp_kvq_append(cache, batch, q, k, v, turned, q_norm=self.norm, k_norm=self.norm, rope=self.rope)
                remp.remp_kvq_attend(cache, batch, turned, out[layer, :, h0 * group:h1 * group], DIM ** -0.5, self.workspace)
        return out


def batch_of(lens, tables, new):
    start = torch.cat((ints(0), torch.cumsum(new, 0).int()))
    return remp.make_kvq_batch(lens, tables, start, int(new.sum()), int(new.max()))


def pages_for(lens, tables, refs, new):
    """Blocks for `new` more tokens of each sequence, lowest free ids first (what a server's scheduler does on the host)."""
    host, table, free = lens.tolist(), tables.cpu(), [i for i, r in enumerate(refs.tolist()) if r == 0]
    for s, n in enumerate(new.tolist()):
        for j in range(-(-host[s] // BLOCK), -(-(host[s] + n) // BLOCK)):
            table[s, j] = free.pop(0)
            refs[int(table[s, j])] += 1
    tables.copy_(table)
    lens += new


def main():
    gen = torch.Generator(device="cuda").manual_seed(0)
    draw = lambda tokens: torch.randn(LAYERS, tokens, Q_HEADS + 2 * KV_HEADS, DIM, generator=gen, device="cuda").bfloat16()  # noqa: E731
    prompts, seqs = len(PROMPTS), len(PROMPTS) * (1 + SAMPLES)
    lens, tables = torch.zeros(seqs, dtype=torch.int32, device="cuda"), torch.full((seqs, WIDTH), -1, dtype=torch.int32, device="cuda")
    blocks = 96
    refs, result = torch.zeros(blocks, dtype=torch.int32, device="cuda"), ints(0, 0)
    ranks = Ranks(Topo(1, 1), blocks)

    # prompts: every row of the batch is a prompt's token
    new = ints(*PROMPTS, *[0] * (seqs - prompts))
    pages_for(lens, tables, refs, new)
    ranks.step(batch_of(lens, tables, new), draw(sum(PROMPTS)))

    # samples share their prompt's pages, all but a last one that both would write
    parents = torch.arange(prompts, device="cuda").repeat_interleave(SAMPLES).int()
    children = torch.arange(prompts, seqs, device="cuda").int()
    pairs = torch.empty(len(children), 2, dtype=torch.int32, device="cuda")
    remp.remp_pages_fork(lens, tables, BLOCK, parents, children, refs, refs, pairs, result)
    remp.remp_pages_copy(ranks.topo, ranks.shape, ranks.shards(), pairs, result)
    assert int(result[1]) == 0

    # single tokens
    one = torch.ones(seqs, dtype=torch.int32, device="cuda")
    for _ in range(STEPS):
        pages_for(lens, tables, refs, one)
        ranks.step(batch_of(lens, tables, one), draw(seqs))

    # every second sequence is done: its pages become free, and the cache compact
    done = (torch.arange(seqs, device="cuda") % 2).int()
    remp.remp_pages_free(lens, tables, BLOCK, done, refs, lens, tables, refs, result)
    remp.remp_pages_compact(lens, tables, BLOCK, refs, tables, refs, moves := torch.empty(blocks // 2, 2, dtype=torch.int32, device="cuda"), result)
    remp.remp_pages_copy(ranks.topo, ranks.shape, ranks.shards(), moves, result)
    used = int((refs > 0).sum())
    assert int(result[1]) == 0 and int(tables.max()) < used

    # the switch: shared pages stay shared, the new pools hold what is used and room for what comes
    after = Ranks(Topo(2, 2), used + 24)
    moved = torch.empty_like(tables)
    plan = remp.remp_plan_create(ranks.topo, after.topo, ranks.shape, lens, tables)
    total = remp.remp_alloc_dst_blocks_shared(plan, [after.blocks] * 4, 0, blocks, moved)
    remp.remp_migrate_kv(plan, ranks.shards(), after.shards())
    assert remp.remp_plan_status(plan) == remp.REMP_OK and total == used
    remp.remp_plan_destroy(plan)

    # the same queries against both layouts give the same outputs (up to the order in which parts of a sequence are added)
    live = (done == 0).int()
    refs_after = torch.zeros(after.blocks, dtype=torch.int32, device="cuda")
    entries = moved[torch.arange(WIDTH, device="cuda")[None] < ((lens + BLOCK - 1) // BLOCK)[:, None]].long()
    refs_after += torch.bincount(entries, minlength=after.blocks).int()
    lens_after = lens.clone()
    qkv = draw(int(live.sum()))
    pages_for(lens, tables, refs, live)
    pages_for(lens_after, moved, refs_after, live)
    before_switch = ranks.step(batch_of(lens, tables, live), qkv)
    after_switch = after.step(batch_of(lens_after, moved, live), qkv)
    torch.testing.assert_close(before_switch, after_switch, rtol=2.0 ** -7, atol=1e-3)
    print(f"served {seqs} sequences, switched TP1PP1 -> TP2PP2 with {used} pages of {sum(p.numel() for p in ranks.pools) // blocks} bytes: same outputs")


if __name__ == "__main__":
    main()
