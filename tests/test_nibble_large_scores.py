"""fe_nibble_attention where scores are as large as the interface allows: the largest takes all of a row's weight."""
import numpy as np
import pytest

from tests import nibble_oracle as N
from tests.generation_oracle import U, f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_nibble_attention import Batch4  # noqa: E402
from tests.test_prefix_attention import BF, HF  # noqa: E402


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("S,hq,hkv", [(2, 4, 2), (2, 12, 1), (30, 4, 2)])
def test_scores_up_to_the_limit(S, hq, hkv, dtype):
    """Where the largest score is ahead by twice the scores' error and the 40 powers of two that a weight counts down to, the
    result is its key's value, by the roundings of a weight or value, of a weight times its scale, and of the result."""
    b = Batch4(1, [S], [300], [1] * S, [1] * S, hq, hkv, 64, 32, dtype)
    kc, ks, vc, vs = b.np
    K, V = N.unpack(kc, ks), N.unpack(vc, vs)
    q = f64(b.q).reshape(S, hkv, hq // hkv, 64)
    at = [[(b.pre[0, c // 32], c % 32) for c in range(300)] + [(b.own[s, 0], 0)] for s in range(S)]
    keys = np.array([[K[p, :, i] for p, i in rows] for rows in at])  # [sequences, keys, heads, 64]
    values = np.array([[V[p, :, i] for p, i in rows] for rows in at])
    z = np.einsum("skhd,shrd->shrk", keys, q).reshape(S, hq, -1)
    scale = 2.0 ** 22 / np.abs(z).max()
    z = np.sort(z * scale, -1)
    top = np.einsum("skhd,shrd->shrk", keys, q).argmax(-1)  # [sequences, heads, query heads]
    want = np.take_along_axis(values.transpose(0, 2, 1, 3), top[..., None], 2).reshape(S, hq, 64)
    seen = 0
    for lse in (True, False):
        got = b.kv.attend(b.q, *b.args(), scale=scale, with_lse=lse)
        out = f64(got[0] if lse else got)
        assert np.isfinite(out).all()
        el = N.attend(b.q, K, V, b.start, b.lens, b.own, b.groups, b.prefix, b.pre, scale, ks, not lse and b.dense())[3]
        ahead = z[..., -1] - z[..., -2] > 2 * el + 40
        seen += ahead.sum()
        assert np.all(np.abs(out - want)[ahead] <= ((2.0 ** -10 + U[dtype]) * np.abs(want) + 2.0 ** -22)[ahead])
        if lse:
            assert np.all(np.abs(f64(got[1]) - z[..., -1])[ahead] <= el[ahead])
    assert seen > S * hq  # (most rows)
