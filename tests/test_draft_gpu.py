"""Verification of drafts against a plain statement in 64 bits: whole numbers, compared exactly (random numbers are inputs; sums
of a few hundred thousand numbers of 24 bits in 64 bits do not come near an edge by chance)."""
import math

import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu


def distributions(rows, vocab, dtype, gen, sharp=2.5):
    return torch.softmax(torch.randn(rows, vocab, generator=gen, device="cuda") * sharp, -1).to(dtype)


def call(start, drafts, target, draft, accept, pick, error=None):
    n, m = len(start) - 1, len(drafts)
    tokens, accepted = torch.full((m + n,), 77, dtype=torch.int32, device="cuda"), torch.full((n,), 77, dtype=torch.int32, device="cuda")
    dev = lambda x, t: torch.as_tensor(np.ascontiguousarray(x)).to(t).cuda()  # noqa: E731
    remp.remp_draft_verify(dev(start, torch.int32), dev(drafts, torch.int32), target, draft, dev(accept, torch.float32), dev(pick, torch.float32), tokens, accepted,
                           error=error)
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def check(counts, vocab, dtype=torch.float32, given=True, seed=0, near=0.5, view=None):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    m, n = int(start[-1]), len(counts)
    target = distributions(m + n, vocab, dtype, gen)
    draft = None
    row = np.concatenate([np.arange(a, b) + s for s, (a, b) in enumerate(zip(start[:-1], start[1:]))]).astype(int) if m else np.zeros(0, int)
    chance = (target[torch.from_numpy(row).cuda()].float() * (1 - near) + near * distributions(m, vocab, torch.float32, gen)) if m else torch.zeros(0, vocab, device="cuda")
    if given:
        draft = chance.to(dtype)
    drafts = np.array([rng.choice(vocab, p=(p := chance[i].double().cpu().numpy()) / p.sum()) for i in range(m)], dtype=np.int32)
    accept, pick = rng.random(m).astype(np.float32), rng.random(n).astype(np.float32)
    if view is not None:
        target, draft = view(target), view(draft) if draft is not None else None
    tokens, accepted = call(start, drafts, target, draft, accept, pick)
    d64 = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
    want, many, word = ref.verify(start, drafts, d64(target), d64(draft), accept.astype(np.float64), pick.astype(np.float64))
    assert word == 0
    assert accepted.tolist() == many.tolist() and tokens.tolist() == want.tolist()
    return accepted


@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 1000, 4097, 8192, 8193, 32001, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("given", [True, False])
def test_vocabularies(vocab, dtype, given):
    check([3, 0, 1, 5, 2], vocab, dtype, given, seed=vocab)


@pytest.mark.parametrize("counts", [[0], [1], [40], [31, 32, 33, 70], [0] * 9, [2] * 200, list(range(20))])
def test_counts(counts):
    check(counts, 503, seed=len(counts), near=0.05)
    check(counts, 9001, seed=len(counts), near=0.02)


def test_some_are_accepted_and_some_are_not():
    accepted = check([4] * 300, 300, near=0.5)
    assert 0 < (accepted == 4).sum() < 300 and 0 < (accepted == 0).sum() < 300


def test_strides():
    for dtype in (torch.float32, torch.bfloat16):
        def wide(x):
            y = torch.zeros(x.shape[0], 10007, dtype=x.dtype, device="cuda")
            y[:, 3:9004] = x
            return y[:, 3:9004]
        check([2, 1, 3], 9001, dtype, view=wide)


def test_equal_probabilities_fall_on_the_lower_side():
    """Powers of two: every sum is exact, and a mark that a sum meets exactly is not passed."""
    vocab = 16384
    target = torch.full((9, vocab), 2.0 ** -14, device="cuda")
    pick = np.array([0.0, 2.0 ** -14, 0.5, 1 - 2.0 ** -14, 1 - 2.0 ** -24, 0.25, 2.0 ** -15, 3 * 2.0 ** -14, 0.75], dtype=np.float32)
    tokens, accepted = call(np.zeros(10, dtype=np.int32), [], target, None, [], pick)
    assert accepted.tolist() == [0] * 9
    assert tokens.tolist() == [0, 1, 8192, 16383, 16383, 4096, 0, 3, 12288]


def test_acceptance_is_strict_and_exact():
    vocab = 64
    p, q = torch.zeros(2, vocab, device="cuda"), torch.zeros(1, vocab, device="cuda")
    p[:, 5], p[:, 6], q[0, 5], q[0, 7] = 0.25, 0.75, 0.5, 0.5
    for u, want in ((0.5, 0), (float(np.nextafter(np.float32(0.5), np.float32(0))), 1)):
        tokens, accepted = call([0, 1], [5], p, q, [u], [0.0])
        assert accepted.tolist() == [want] and tokens.tolist() == ([6, -1] if want == 0 else [5, 5])


def test_the_same_distribution_and_nothing_left():
    """p <= q everywhere: the draft is refused by a random number at its edge, and the token comes from p."""
    vocab = 100
    p = torch.zeros(2, vocab, device="cuda")
    p[:, 3], p[:, 90] = 0.5, 0.5
    q = p[:1] * 2
    tokens, accepted = call([0, 1], [3], p, q, [0.75], [0.6])
    assert accepted.tolist() == [0] and tokens.tolist() == [90, -1]


def test_nan_negative_and_no_probability():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    vocab = 9000
    p = torch.zeros(3, vocab, device="cuda")
    p[0, 10], p[0, 20], p[0, 30], p[0, 8999] = math.nan, -5.0, 1.0, 1.0
    p[2] = math.nan
    p[1, 77] = 1e-30
    tokens, accepted = call([0, 0, 0, 0], [], p, None, [], [0.5, 0.999, 0.3], error=word)
    assert tokens.tolist() == [8999, 77, -1] and int(word) == 4
    q = torch.full((1, vocab), math.nan, device="cuda")  # counts as 0: accepted, and all of p is left
    tokens, accepted = call([0, 1], [30], torch.cat((p[:1], p[:1])), q, [0.9], [0.0])
    assert accepted.tolist() == [1] and tokens.tolist() == [30, 30]


def test_drafts_outside_the_vocabulary():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = torch.full((4, 8), 0.125, device="cuda")
    for given in (None, torch.full((2, 8), 0.0625, device="cuda")):
        for bad in (-1, 8, 2 ** 31 - 1):
            word.zero_()
            tokens, accepted = call([0, 2, 2], [3, bad], p, given, [0.1, 0.1], [0.0, 0.99], error=word)
            assert accepted.tolist() == [1, 0] and tokens.tolist() == [3, 0, -1, 7] and int(word) == 2


def test_starts_outside_the_drafts_stay_inside_the_arrays():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = torch.full((4, 8), 0.125, device="cuda")
    tokens, accepted = call([-3, 5, 1], [3, 4], p, None, [0.1, 0.1], [0.0, 0.99], error=word)
    assert int(word) == 2


def test_captured_and_replayed():
    gen = torch.Generator(device="cuda").manual_seed(1)
    start, drafts = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda"), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    target, draft = distributions(5, 10000, torch.float32, gen), distributions(3, 10000, torch.float32, gen)
    accept, pick = torch.rand(3, device="cuda"), torch.rand(2, device="cuda")
    tokens, accepted = torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        remp.remp_draft_verify(start, drafts, target, draft, accept, pick, tokens, accepted)
    for seed in range(4):
        gen.manual_seed(seed)
        accept.copy_(torch.rand(3, generator=gen, device="cuda"))
        pick.copy_(torch.rand(2, generator=gen, device="cuda"))
        drafts.copy_(torch.argmax(target[[0, 1, 3]], -1).int())
        graph.replay()
        want, many, _ = ref.verify(start.cpu().numpy(), drafts.cpu().numpy(), target.double().cpu().numpy(), draft.double().cpu().numpy(),
                                   accept.double().cpu().numpy(), pick.double().cpu().numpy())
        assert tokens.tolist() == want.tolist() and accepted.tolist() == many.tolist()
