"""fe_nibble_attention with more than 32 query rows a group: both forms of the products that many rows share, with log-sums
(the keys as they are) and without (bf16: keys rounded), each against its own bound."""
import numpy as np
import pytest

from tests import nibble_oracle as N
from tests.generation_oracle import f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_nibble_attention import Batch4  # noqa: E402
from tests.test_prefix_attention import BF, HF, i32  # noqa: E402


class Many(Batch4):
    rounded = False

    def dense(self):
        return self.rounded and super().dense()

    def both(self, scale=None, q=None, rows=None, **args):
        """Results with log-sums, and without, next to the definition."""
        assert self.many()
        q, rows = self.q if q is None else q, range(len(self.q)) if rows is None else rows
        out, lse = self.kv.attend(q, *self.args(**args), scale=scale, with_lse=True)
        alone = self.kv.attend(q, *self.args(**args), scale=scale)
        self.rounded = False
        self.compare(out, lse, rows, scale, q)
        self.rounded = True  # (of f16 both are the same)
        self.compare(alone, lse, rows, scale, q)
        return out, lse, alone


@pytest.mark.parametrize("d,hq,hkv,dtype", [(32, 40, 2, BF), (64, 24, 1, BF), (64, 24, 1, HF), (128, 17, 1, BF), (128, 64, 4, HF)])
@pytest.mark.parametrize("page", [16, 128])
def test_without_groups(d, hq, hkv, dtype, page):
    Many(1, [1] * 7, [0] * 7, [127, 128, 900, 131, 5, 1300, 0], [1, 1, 7, 4, 9, 2, 1], hq, hkv, d, page, dtype, alone=True).both()


@pytest.mark.parametrize("n", [127, 128, 129, 255, 257, 1000])
@pytest.mark.parametrize("d,dtype", [(32, BF), (64, BF), (128, BF), (128, HF)])
def test_prefixes_end_around_tiles(n, d, dtype):
    Many(2, [20, 0, 100, 30], [n, 400, n + 128, 0], [1 + i % 40 for i in range(150)], [1] * 150, 4, 2, d, 64, dtype).both()


@pytest.mark.parametrize("rows,K", [(16, 20), (1, 200), (40, 3), (130, 2)])
@pytest.mark.parametrize("d,hq,hkv", [(32, 2, 1), (64, 8, 1), (128, 4, 1)])
def test_several_units_of_rows(rows, K, d, hq, hkv):
    Many(3, [K], [700], [rows + 3 + i % 5 for i in range(K)], [rows] * K, hq, hkv, d, 32, BF).both()


@pytest.mark.parametrize("spread,scale", [(30.0, None), (0.01, None), (1.0, 0.0), (1.0, 3.0)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_peaked_and_flat_weights(spread, scale, dtype):
    Many(4, [20, 9], [700, 300], [1 + i % 9 for i in range(29)], [1] * 29, 8, 2, 128, 32, dtype, spread).both(scale)


def test_large_and_small_keys_and_values():
    b = Many(5, [30], [600], [3] * 30, [1] * 30, 4, 2, 64, 32, BF)
    for x, sizes in ((b.kc, (1e5, 1e-3)), (b.vc, (4e5, 1e-3))):
        x[::2] *= sizes[0] / 4
        x[1::2] *= sizes[1]
    b.put(b.kc, b.vc)
    b.both(scale=1e-6)


def test_more_row_tiles_than_a_block_counts_for_itself():
    Many(6, [2] * 520, [130 + i % 3 for i in range(520)], [1 + i % 5 for i in range(1040)], [1] * 1040, 32, 1, 32, 16, BF).both()


def test_split_units_and_stale_pages():
    Many(7, [40, 25], [5000, 700], [3] * 65, [1] * 65, 8, 2, 128, 64, BF).both()


@pytest.mark.parametrize("lse", [True, False])
def test_a_page_and_scales_that_are_wrong(lse):
    b = Many(8, [40, 25, 30], [900, 700, 256], [3] * 95, [1] * 95, 8, 2, 128, 64, BF)
    pre, status = b.pre.copy(), i32([0])
    pre[1, 3] = b.kc.shape[0] + 7
    b.kv.v_scales[int(b.pre[2, 2]), 1, 5, 1] = float("nan")
    got = b.kv.attend(b.q, *b.args(prefix_pages=pre), with_lse=lse, status=status)
    out = got[0] if lse else got
    assert status.item() == 1 and torch.isnan(out[40:65]).all()
    h = 4  # (the second key head's)
    assert torch.isnan(out[65:, h:, 32:64]).all()
    for part in (out[:40], out[65:, :h], out[65:, h:, :32], out[65:, h:, 64:]):
        assert torch.isfinite(part).all()
    if lse:
        assert torch.isnan(got[1][40:65]).all() and torch.isfinite(got[1][:40]).all() and torch.isfinite(got[1][65:]).all()
    kc, ks, vc, vs = b.np
    b.rounded = not lse
    clean = b.kv.attend(b.q, *b.args(), with_lse=True)[1]
    b.compare(out, clean, range(40))


@pytest.mark.parametrize("size,large", [(1e-3, 1e3), (1e-4, 1e4), (1e-5, 2e4), (1e-6, 3e4)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_small_keys_and_large_queries(size, large, dtype):
    """What rounding leaves over of a key's number is kept to half of 2^-24 times 8: scores are off by scale 2^-22 sum |q|."""
    b = Many(9, [30], [600], [3] * 30, [1] * 30, 4, 2, 64, 32, dtype)
    b.kc.mul_(size)
    b.put(b.kc, b.vc)
    q = (b.q.float() / b.q.float().abs().max() * large).to(dtype)
    out, lse = b.kv.attend(q, *b.args(), scale=1.0, with_lse=True)
    kc, ks, vc, vs = b.np
    _, want, _, el = N.attend(q, N.unpack(kc, ks), N.unpack(vc, vs), b.start, b.lens, b.own, b.groups, b.prefix, b.pre, 1.0, ks)
    assert np.all(np.abs(f64(lse) - want) <= el + 2.0 ** -22 * np.abs(f64(q)).sum(-1))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_log_sums_of_the_keys_as_they_are(d, dtype):
    """Queries along what rounding to f16 leaves over of equal keys: all errors of a product add up."""
    b = Many(10, [50], [256], [2] * 50, [1] * 50, 4, 2, d, 64, dtype)
    rng = np.random.RandomState(d)
    n = rng.choice([3, 5, 7], d) * rng.choice([-1, 1], d)
    n[::32] = 7
    b.kc[:] = torch.from_numpy(n * 0.2113).to(dtype).cuda()
    b.put(b.kc, b.vc)
    kc, ks, vc, vs = b.np
    ks[:] = 0.2113  # (all of f16's bits)
    b.kv.k_scales.fill_(float(ks[0, 0, 0, 0]))
    K = N.unpack(kc, ks)
    key = K[0, 0, 0]
    left = key / 8 - (key / 8).astype(np.float16).astype(float)
    q = torch.from_numpy(np.broadcast_to(np.sign(left) * 3, tuple(b.q.shape)).copy()).to(dtype).cuda()
    out, lse = b.kv.attend(q, *b.args(), scale=1.0, with_lse=True)
    _, want, _, el = N.attend(q, K, N.unpack(vc, vs), b.start, b.lens, b.own, b.groups, b.prefix, b.pre, 1.0, ks)
    assert 8 * 3 * np.abs(left).sum() > 2 * el.max()  # (rounded keys would be seen)
    assert np.all(np.abs(f64(lse) - want) <= el)
    b.rounded = False
    b.compare(out, lse, range(50), 1.0, q)
