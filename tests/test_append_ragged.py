"""fe_kv_append with as many rows as sequences, some of them without any: a row's number is then no sequence's."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_append import close, i32, rope_of  # noqa: E402


def rows_of(seed, S):
    """S rows over S sequences, about a third of them with one row, the others with none or several."""
    rng = np.random.RandomState(seed)
    return np.bincount(np.where(rng.rand(S) < 0.3, np.arange(S), rng.randint(0, S, S)), minlength=S)


@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("rows", [[1], [0, 2], [2, 0], [1, 0, 2], [0, 1, 2], [1, 1, 0, 2], [0, 0, 3], [0, 4, 0, 0], [1, 2, 0, 1],
                                  [1] * 5, rows_of(1, 64), rows_of(2, 1000)], ids=lambda r: str(len(r)) + "_" + str(r[0]) + str(r[-1]))
def test_as_many_rows_as_sequences(rows, pairs):
    from paper_2603_02565_gb300 import PagedKV
    rows = np.asarray(rows)
    S, hq, hkv, d, page = len(rows), 4, 2, 32, 16
    assert rows.sum() == S
    rng = np.random.RandomState(S)
    first, shift = rng.randint(0, 30, S), rng.randint(0, 50, S)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = -(-(first + rows) // page)
    table = np.full((S, max(1, n.max())), -1)
    free = rng.permutation(int(n.sum()) + 1)
    for s in range(S):
        table[s, :n[s]], free = free[:n[s]], free[n[s]:]
    x = torch.randn(S, hq + 2 * hkv, d, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    kc, vc = (torch.randn(int(n.sum()) + 1, hkv, page, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    rope, status = rope_of(int((first + rows + shift).max()) + 1, d), i32([0])
    want = O.append(k, v, q, start, first, table, rope, pairs, shift, kc, vc)
    out = PagedKV(kc, vc).append(k, v, i32(start), i32(first), i32(table), q=q, rope=rope, pairs=pairs, shift=i32(shift),
                                 status=status)
    assert status.item() == 0
    close(kc, want[0], want[3], torch.bfloat16)
    assert np.array_equal(O.f64(vc), want[1])
    close(out, want[2], want[4], torch.bfloat16)
