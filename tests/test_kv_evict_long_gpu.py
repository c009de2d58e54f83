"""Eviction where clusters of thread blocks choose and move, against plain statements (kv_reference)."""
import numpy as np
import pytest

from tests.test_kv_evict_gpu import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("longest", [1021, 1022, 4093, 4094, 16381, 16382, 32765, 32766, 131070])
@pytest.mark.parametrize("kind", ["heavy", "ties", "any"])
def test_each_choice(longest, kind):
    """On both sides of where another kernel chooses (three slots more than the longest sequence)."""
    check([longest, longest // 3, 5], [longest // 2, 7, 2], 1, 64, 16, 4, 16, kind)


@pytest.mark.parametrize("seqs,heads", [(1, 1), (20, 2), (40, 2), (80, 2), (150, 2)])
def test_each_move(seqs, heads):
    """Clusters of 8, 4, 2 thread blocks and single ones, chunks that end inside and behind the rows that stay."""
    rng = np.random.default_rng(seqs)
    lens = rng.integers(1, 700, seqs)
    check(lens.tolist(), rng.integers(0, 500, seqs).astype(np.int32), heads, 128, 16, 2, 9, seed=seqs)


@pytest.mark.parametrize("values", [(0.0, 1.0, 1e-30), (3e38, 3e38, 3e38), (np.inf, 3.4e38, 1.0), (-np.inf, np.inf, np.nan), (1.0, np.nextafter(np.float32(1), np.float32(2)), 1.0)])
def test_ranges_at_the_ends_of_what_a_weight_can_be(values, monkeypatch):
    from tests import test_kv_evict_gpu as base
    monkeypatch.setattr(base, "weights_of", lambda kind, shape, rng: rng.choice(np.array(values, dtype=np.float32), shape))
    check([900, 33, 2500], [400, 20, 1999], 2, 64, 16, 1, 3)
    check([5000, 20000], [1, 19990], 1, 64, 16, 0, 0)
