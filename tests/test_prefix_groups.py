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
