"""Verification of drafts writes its tokens and counts and nothing beside them, also where draft_start leads outside the drafts."""
import numpy as np
import pytest
import torch

import paper_2606_18741_b200 as remp

pytestmark = pytest.mark.gpu

GUARD = 64


def guarded(n):
    whole = torch.full((n + 2 * GUARD,), 77, dtype=torch.int32, device="cuda")
    return whole, whole[GUARD:GUARD + n]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("vocab", [8, 16384])
@pytest.mark.parametrize("start,drafts,tokens,accepted,bits", [
    # cut to two drafts of the first sequence and none of the second
    ([-3, 5, 1], [3, 4], [3, 4, 0, -2], [2, 0], 2),
    ([0, 1, 2 ** 31 - 1], [3, 4], [3, 0, 4, -2], [1, 1], 2),
    ([-2 ** 31, 0, 2], [3, 4], [0, 3, 4, -2], [0, 2], 2),
    ([0, 2, 2], [3, 4], [3, 4, 0, -2], [2, 0], 0)])
def test_nothing_beside_the_outputs(given, vocab, start, drafts, tokens, accepted, bits):
    """-2: the last of the vocabulary's tokens, by a random number near 1; 0: the first, by 0."""
    m, n = len(drafts), len(accepted)
    dev = lambda x, t: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    target = torch.full((m + n, vocab), 1.0 / vocab, device="cuda")
    draft = torch.full((m, vocab), 1.0 / vocab, device="cuda") if given else None
    all_tokens, got = guarded(m + n)
    all_accepted, many = guarded(n)
    remp.remp_draft_verify(dev(start, torch.int32), dev(drafts, torch.int32), target, draft, dev([0.5 / vocab] * m, torch.float32),
                           dev([0.0, 1 - 0.5 / vocab], torch.float32), got, many, error=word)
    assert got.tolist() == [vocab - 1 if x == -2 else x for x in tokens] and many.tolist() == accepted and int(word) == bits
    for whole, size in ((all_tokens, m + n), (all_accepted, n)):
        assert (whole[:GUARD] == 77).all() and (whole[GUARD + size:] == 77).all()


def test_random_starts():
    rng = np.random.default_rng(0)
    for seed in range(20):
        m, n = int(rng.integers(1, 40)), int(rng.integers(1, 20))
        start = torch.tensor(rng.integers(-10, m + 10, n + 1).astype(np.int32), device="cuda")
        drafts = torch.tensor(rng.integers(-5, 505, m).astype(np.int32), device="cuda")
        all_tokens, got = guarded(m + n)
        all_accepted, many = guarded(n)
        p = torch.softmax(torch.randn(m + n, 500, device="cuda"), -1)
        remp.remp_draft_verify(start, drafts, p, p[:m].contiguous(), torch.rand(m, device="cuda"), torch.rand(n, device="cuda"), got, many)
        for whole, size in ((all_tokens, m + n), (all_accepted, n)):
            assert (whole[:GUARD] == 77).all() and (whole[GUARD + size:] == 77).all()
        assert (many >= 0).all() and (many <= m).all() and (got < 500).logical_or(got == 77).all()
