"""Attention with more query heads a key head than a tile of queries has rows."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import BF, HF, Batch  # noqa: E402


@pytest.mark.parametrize("hq,hkv,d,dtype", [(129, 1, 32, BF), (160, 1, 64, HF), (300, 2, 128, BF), (1024, 1, 32, HF), (2048, 2, 64, BF)])
def test_many_query_heads_a_key_head(hq, hkv, d, dtype):
    Batch(hq, [2, 1], [40, 0], [5, 21, 18], [1, 3, 2], hq, hkv, d, 16, dtype).check()
