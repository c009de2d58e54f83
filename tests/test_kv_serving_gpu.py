"""The calls on a cache of 16-bit values as a server makes them: prompts, their weights, eviction, a topology switch, drafts and their
verification, the next token. What the cache holds is followed row by row and compared exactly; attention over it goes by the
formula in 64 bits (tolerances: test_kv_gpu)."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from paper_2606_18741_b200.synth import Shape, Topo
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu

HEADS, GROUP, DIM, BLOCK, WIDTH, KEEP, FIRST, RECENT, DRAFTS, VOCAB = 2, 4, 128, 16, 12, 48, 2, 8, 3, 500
LENS = [70, 150, 33]


class Rank:
    def __init__(self, topo, rank, blocks):
        self.shape, self.blocks = Shape(1, HEADS, DIM, BLOCK, 2), blocks
        self.pool = torch.zeros(remp.remp_shard_bytes(topo, self.shape, rank, blocks), dtype=torch.uint8, device="cuda")
        _, _, self.h0, self.h1 = remp.remp_rank_ownership(topo, self.shape, rank)
        self.cache = remp.make_kv_pool(self.pool, blocks, self.h1 - self.h0, DIM, BLOCK)
        self.model = ref.Cache.__new__(ref.Cache)
        self.model.__dict__.update(blocks=blocks, heads=self.h1 - self.h0, d=DIM, bs=BLOCK, token_major=False,
                                   data=self.pool.view(torch.bfloat16).view(1, 2, blocks, self.h1 - self.h0, BLOCK, DIM))

    def rows(self, tables, s, n):
        """[K, V][position][head][dim] of a sequence, as the cache holds them."""
        at = torch.arange(n, device="cuda")
        return torch.stack([self.model.rows(0, kv, tables[s], at)[0] for kv in (0, 1)])

    def step(self, batch, lens, new, tables, qkv, positions, rope, norm, workspace, weights, fresh):
        """Append, attend, weigh; the attention checked. qkv [tokens][heads of q, k, v][dim]."""
        q = qkv[:, self.h0 * GROUP:self.h1 * GROUP]
        k, v = (qkv[:, HEADS * (GROUP + i) + self.h0:HEADS * (GROUP + i) + self.h1] for i in (0, 1))
        turned = torch.empty_like(q, memory_format=torch.contiguous_format)
        remp.remp_kv_append(self.cache, batch, q, k, v, turned, q_norm=norm, k_norm=norm, rope=rope, positions=positions)
        out, lse = torch.empty_like(turned), torch.empty(turned.shape[:2], device="cuda")
        remp.remp_kv_attend(self.cache, batch, turned, out, DIM ** -0.5, workspace, window=100, first=FIRST, lse=lse)
        mine = weights[:, self.h0:self.h1].contiguous()
        remp.remp_kv_weigh(self.cache, batch, turned, lse, mine, DIM ** -0.5, window=100, first=FIRST, fresh=fresh)
        at = 0
        for s, (n, m) in enumerate(zip(lens, new)):
            want, want_lse, size, terms, added = ref.attend(self.model, 0, tables[s], n, turned[at:at + m].double(), n - m, DIM ** -0.5, 100, FIRST)
            tol = 2.0 ** -8 * want.abs() + (2 * (terms * 2.0 ** -18 + 2.0 ** -20) + 2.0 ** -14 + 2.0 ** -8) * size + 2.0 ** -26
            assert ((out[at:at + m].double() - want).abs() <= tol).all()
            assert ((lse[at:at + m].double() - want_lse).abs() <= terms * 2.0 ** -18 + want_lse.abs() * 2.0 ** -22 + 2.0 ** -18).all()
            old = torch.zeros_like(added) if fresh else weights[s, self.h0:self.h1, :n].double()
            old[:, n - m:] = 0
            # lse is off by what its bound says, a weight by as much of itself
            bound = (2 * terms * 2.0 ** -18 + want_lse.abs().max() * 2.0 ** -20 + 2.0 ** -17) * added + 2.0 ** -22 * (old + added) + 1e-30
            assert ((mine[s, :, :n].double() - old - added).abs() <= bound).all()
            at += m
        weights[:, self.h0:self.h1] = mine


def batch_of(lens, new, tables):
    start = torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device="cuda")
    return remp.make_kvq_batch(torch.tensor(lens, dtype=torch.int32, device="cuda"), tables, start, int(sum(new)), max(new))


def test_prompts_eviction_switch_drafts_and_on():
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda n: torch.randn(n, HEADS * (GROUP + 2), DIM, generator=gen, device="cuda").bfloat16()  # noqa: E731
    rng, n, workspace = np.random.default_rng(3), len(LENS), remp.make_kv_workspace()
    norm = torch.rand(DIM, generator=gen, device="cuda") + 0.5
    angle = torch.arange(512, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda") / DIM)
    rope = torch.cat((angle.cos(), angle.sin()), 1).contiguous()
    before, blocks = Rank(Topo(1, 1), 0, 40), 40
    tables = torch.from_numpy(rng.permutation(blocks)[:n * WIDTH].reshape(n, WIDTH).astype(np.int32)).cuda()

    # prompts, and how much each of their tokens is looked at
    weights = torch.full((n, HEADS, WIDTH * BLOCK), 7.0, device="cuda")
    before.step(batch_of(LENS, LENS, tables), LENS, LENS, tables, draw(sum(LENS)), None, rope, norm, workspace, weights, True)

    # eviction: rows that stay, in their order
    rows = [before.rows(tables, s, LENS[s]) for s in range(n)]
    host = weights.cpu().numpy()
    kept = torch.empty(n, HEADS, KEEP, dtype=torch.int32, device="cuda")
    remp.remp_kv_evict(before.cache, torch.tensor(LENS, dtype=torch.int32, device="cuda"), tables, torch.full((n,), KEEP, dtype=torch.int32, device="cuda"),
                       weights, weights, kept, first=FIRST, recent=RECENT)
    lens = [min(x, KEEP) for x in LENS]
    for s in range(n):
        stay = [ref.choose(host[s, h], LENS[s], KEEP, FIRST, RECENT) for h in range(HEADS)]
        assert [kept[s, h, :lens[s]].tolist() for h in range(HEADS)] == stay
        assert all(np.array_equal(weights[s, h, :lens[s]].cpu().numpy(), host[s, h, stay[h]]) for h in range(HEADS))
        rows[s] = torch.stack([rows[s][:, stay[h], h] for h in range(HEADS)], 2)
        assert torch.equal(before.rows(tables, s, lens[s]), rows[s])

    # the switch to two ranks
    topo, used = Topo(2, 1), sum(-(-x // BLOCK) for x in lens)
    after = [Rank(topo, r, used + 6) for r in range(2)]
    dev_lens, moved = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.empty_like(tables)
    plan = remp.remp_plan_create(Topo(1, 1), topo, before.shape, dev_lens, tables)
    assert remp.remp_alloc_dst_blocks(plan, [r.blocks for r in after], 0, moved) == used
    remp.remp_migrate_kv(plan, remp.make_shards([before.pool], [blocks]), remp.make_shards([r.pool for r in after], [r.blocks for r in after]))
    assert remp.remp_plan_status(plan) == remp.REMP_OK
    remp.remp_plan_destroy(plan)
    for s in range(n):  # a block for what comes
        moved[s, -(-lens[s] // BLOCK):] = -1
        moved[s, -(-lens[s] // BLOCK)] = used + s
        for r in after:
            assert torch.equal(r.rows(moved, s, lens[s]), rows[s][:, :, r.h0:r.h1])

    # a token and drafts behind it; positions are those of the text, not of the cache
    text, new = list(LENS), [1 + DRAFTS] * n
    for _ in range(2):
        lens, text = [x + y for x, y in zip(lens, new)], [x + y for x, y in zip(text, new)]
        positions = torch.cat([torch.arange(t - m, t, device="cuda") for t, m in zip(text, new)]).int()
        qkv, batch = draw(sum(new)), batch_of(lens, new, moved)
        for r in after:
            r.step(batch, lens, new, moved, qkv, positions, rope, norm, workspace, weights, False)

        drafts = rng.integers(0, VOCAB, n * DRAFTS).astype(np.int32)
        target, draft = (rng.dirichlet(np.full(VOCAB, 0.1), m).astype(np.float32) for m in (n * (DRAFTS + 1), n * DRAFTS))
        for i in range(n * DRAFTS):  # likely ones
            target[i + i // DRAFTS, drafts[i]] = draft[i, drafts[i]] = 0.5
        accept, pick = rng.random(n * DRAFTS).astype(np.float32), rng.random(n).astype(np.float32)
        start = np.arange(n + 1, dtype=np.int32) * DRAFTS
        dev = [torch.from_numpy(x).cuda() for x in (start, drafts, target, draft, accept, pick)]
        tokens, accepted = torch.empty(n * (DRAFTS + 1), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        remp.remp_draft_verify(*dev, tokens, accepted)
        want_tokens, want_accepted, _ = ref.verify(start, drafts, *(x.astype(np.float64) for x in (target, draft, accept, pick)))
        assert accepted.tolist() == want_accepted.tolist() and tokens.tolist() == want_tokens.tolist()

        # drafts that were refused leave: the next tokens are written over their rows
        back = [DRAFTS - int(x) for x in accepted]
        lens, text = [x - y for x, y in zip(lens, back)], [x - y for x, y in zip(text, back)]
        for s in range(n):
            weights[s, :, lens[s]:] = 7.0
