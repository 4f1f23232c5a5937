"""Attention over more groups and sequences than the plan holds in shared memory or has threads for, with rows
spread so unevenly that no row is where equal sequences would have it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import BF, HF, Batch  # noqa: E402


def test_thousands_of_groups():
    rng = np.random.RandomState(5)
    n = 2500
    groups = rng.randint(0, 3, n)
    S = int(groups.sum())
    own = rng.randint(0, 20, S)
    Batch(1, groups, rng.randint(0, 12, n), own, np.minimum(own, rng.randint(0, 3, S)), 2, 1, 32, 16, BF).check()


def test_two_thousand_and_forty_eight_groups():
    n = 2048
    Batch(2, [1] * n, [3] * n, [2] * n, [1] * n, 1, 1, 32, 16, HF).check()


@pytest.mark.parametrize("where", ["front", "back"])
def test_all_rows_in_one_sequence_of_many(where):
    rows = np.zeros(900, dtype=int)
    rows[0 if where == "front" else -1] = 300
    rows[450] = 1
    own = np.where(rows > 0, rows + 5, 7)
    Batch(3, [300, 0, 600], [40, 5, 0], own, rows, 4, 2, 64, 16, BF).check()


def test_ten_thousand_sequences_of_one_row():
    rng = np.random.RandomState(6)
    S = 10000
    Batch(4, [100] * 100, rng.randint(0, 30, 100), rng.randint(1, 4, S), [1] * S, 1, 1, 32, 16, BF).check()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_a_nan_in_a_split_unit_touches_only_the_rows_that_see_it(d):
    """The rows of a sequence with a value that is no number are computed again after the join of 40 pieces."""
    from paper_2603_02565_gb300 import PagedKV
    b = Batch(8, [4], [5003], [30, 21, 9, 40], [4, 4, 4, 4], 4, 2, d, 16, BF)
    want, lse = b.check()
    for what, bad in (("v", float("nan")), ("v", float("inf")), ("k", float("nan"))):
        kc, vc = b.kc.clone(), b.vc.clone()
        (vc if what == "v" else kc)[b.own[1][18 // 16], 0, 18 % 16] = bad  # row 18 of 21: the last three query rows see it
        out, l2 = PagedKV(kc, vc).attend(b.q, *b.args(), with_lse=True)
        same = torch.ones(16, 4, dtype=torch.bool, device="cuda")
        same[5:8, :2] = False  # sequence 1's rows see its rows 0 .. 17, .. 18, .. 19, .. 20; its key head 0 has query heads 0, 1
        # (the row before the bad one is in a recomputed sequence: another order of sums, the same numbers rounded)
        again = torch.zeros_like(same)
        again[4, :2] = True
        assert torch.equal(out[same & ~again], want[same & ~again])
        assert torch.allclose(out[again].float(), want[again].float(), rtol=2.0 ** -6, atol=2.0 ** -7)
        assert not torch.isfinite(out[~same]).any()
