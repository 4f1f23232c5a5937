"""fe_nibble_attention: a query that holds an infinity makes its row NaN, whatever signs the keys have."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_nibble_attention import Batch4  # noqa: E402
from tests.test_prefix_attention import BF, HF  # noqa: E402

INF = float("inf")


def spoil(b, at, value, empty=()):
    """Rows `at` (token, head) get `value` at element 9, where all keys have a number of one sign."""
    b.kc[..., 9] = 5.0
    b.put(b.kc, b.vc)
    want, wl = (x.clone() for x in b.kv.attend(b.q, *b.args(), with_lse=True))
    alone = b.kv.attend(b.q, *b.args()).clone()
    q = b.q.clone()
    for t, h in at:
        q[t, h, 9] = value
        if t not in empty:
            want[t, h] = alone[t, h] = wl[t, h] = float("nan")
    out, lse = b.kv.attend(q, *b.args(), with_lse=True)
    for got, ref in ((out, want), (lse, wl), (b.kv.attend(q, *b.args()), alone)):
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(got.nan_to_num(), ref.nan_to_num())


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_one_key(d, dtype, value):
    spoil(Batch4(1, [1] * 4, [0] * 4, [1, 1, 40, 1], [1] * 4, 4, 2, d, 16, dtype, alone=True), [(0, 1), (2, 0), (3, 3)], value)
    spoil(Batch4(2, [2, 1], [1, 0], [0, 1, 2], [1] * 3, 3, 1, d, 16, dtype), [(0, 0), (2, 2)], value)


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_nine_to_sixteen_rows(d, dtype, value):
    spoil(Batch4(3, [1] * 3, [0] * 3, [1, 9, 50], [1] * 3, 12, 1, d, 16, dtype, alone=True), [(0, 0), (0, 11), (1, 8), (2, 3)], value)


@pytest.mark.parametrize("value", [INF, -INF])
def test_pieces_of_a_long_context(value):
    spoil(Batch4(4, [1], [0], [20000], [1], 2, 1, 64, 64, BF, alone=True), [(0, 1)], value)


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("prefix", [128, 300, 6000])
def test_many_rows(prefix, d, dtype, value):
    # keys that all rows see alone (own rows: none, one, several), units that are split
    b = Batch4(5, [100, 30], [prefix, 256], [i % 3 for i in range(130)], [1] * 130, 4, 2, d, 64, dtype)
    assert b.many()
    spoil(b, [(0, 0), (0, 3), (1, 2), (2, 1), (70, 0), (99, 3), (129, 1)], value)


@pytest.mark.parametrize("value", [INF, -INF])
def test_many_rows_without_groups(value):
    b = Batch4(6, [1] * 4, [0] * 4, [128, 129, 1, 400], [1, 2, 1, 1], 80, 2, 64, 32, BF, alone=True)
    assert b.many()
    spoil(b, [(0, 0), (1, 50), (2, 79), (3, 3), (4, 40)], value)


@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
def test_a_row_that_sees_nothing_stays_empty(value):
    b = Batch4(7, [2, 1], [0, 30], [0, 3, 2], [1, 4, 2], 4, 2, 64, 16, BF)
    spoil(b, [(0, 1), (1, 0), (2, 3)], value, empty=[0, 1])
