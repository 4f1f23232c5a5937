"""fe_nibble_attention: many keys of small weights under a peak count, whatever the size of the values' scales."""
import numpy as np
import pytest

from tests import nibble_oracle as N
from tests.generation_oracle import TINY, U, f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_nibble_attention import Batch4  # noqa: E402
from tests.test_prefix_attention import BF, DEV, HF, i32  # noqa: E402

n = 131072  # keys


def tail(d, hq, dtype, scale, peak, what, below, S):
    """Key `peak` of a sequence has the whole weight but for 2^-below of it each of the others; the values, of this scale, are
    the others' or the peak's.  S sequences hold the same pages: many of them leave each to few warps, which meet the
    peak's weight or scale with the others'."""
    from paper_2603_02565_gb300 import PagedKV4
    k, v = np.zeros((2, d), np.float32), np.zeros((2, d), np.float32)  # of the others and of the peak
    k[0, 0] = -below * np.log(2.0)
    v[int(what == "peak")] = 7 * scale
    which = (np.arange(n) == peak).astype(int)
    held = [torch.from_numpy(x[which].reshape(n // 128, 1, 128, -1)).to(DEV) for y in (k, v) for x in N.pack(y)]
    q = torch.zeros(S, hq, d, dtype=dtype, device=DEV)
    q[..., 0] = 1
    pages = i32(np.arange(n // 128)[None]).repeat(S, 1)
    out, lse = PagedKV4(*held, dtype=dtype).attend(q, i32(np.arange(S + 1)), i32([n] * S), pages, scale=1.0, with_lse=True)
    w = np.exp(N.unpack(*N.pack(k))[0, 0])
    size = np.abs(N.unpack(*N.pack(v))).max()
    want = size * ((n - 1) * w if what == "others" else 1) / (1 + (n - 1) * w)
    return f64(out), f64(lse), want, size, w


@pytest.mark.parametrize("below", [14.0, 17.0, 18.5])
@pytest.mark.parametrize("peak", [0, 70000, n - 1])
@pytest.mark.parametrize("what,S", [("others", 1000), ("peak", 1000), ("others", 3)])
@pytest.mark.parametrize("d,hq,dtype,scale", [
    (64, 1, HF, 2.0 ** -14), (128, 12, HF, 1.3 * 2.0 ** -13), (32, 1, HF, 2.0 ** -10), (64, 12, HF, 1.0), (128, 1, HF, 2.0 ** 9),
    (128, 1, BF, 2.0 ** -24), (64, 1, BF, 1.37 * 2.0 ** -17), (32, 12, BF, 2.0 ** -15), (128, 12, BF, 2.0 ** -8), (64, 1, BF, 1.99 * 2.0 ** 7),
    (64, 12, BF, 2.0 ** 8), (128, 12, BF, 2.0 ** 12), (32, 1, BF, 2.0 ** 14), (128, 1, BF, 60000.0), (64, 12, BF, 65504.0)])
def test_a_long_flat_tail_under_a_peak(d, hq, dtype, scale, what, S, peak, below):
    """A weight, and again a weight times a scale, is rounded to 11 bits (2^-11 of it at most), or to 2^-28 of the largest one:
    numerators of the others are off by N (2^-10 w + 2 2^-28) |v|, that of the peak by 2^-10 |v|, the sum of
    weights by N (2^-11 w + 2^-28) + 2^-11.  Products of 16 keys are added up at a time, cut off at 2^-23 of the largest term (twice), and
    scores have an exponent's fp32."""
    out, lse, want, v, w = tail(d, hq, dtype, scale, peak, what, below, S)
    N1 = n - 1
    total = 1 + N1 * w
    top = N1 * (2.0 ** -10 * w + 2.0 ** -27) if what == "others" else 2.0 ** -10
    off = v * top / total + want * (N1 * (2.0 ** -11 * w + 2.0 ** -28) + 2.0 ** -11) / total
    steps = (n / 8 + 64) * 2.0 ** -23 + below * 2.0 ** -21
    assert np.all(np.abs(out - want) <= off + want * (steps + U[dtype]) + TINY[dtype]), np.abs(out / want - 1).max()
    assert np.all(np.abs(lse - np.log(total)) <= steps + 2.0 ** -22)


@pytest.mark.parametrize("peak", [0, 70000, n - 1])
@pytest.mark.parametrize("what", ["others", "peak"])
@pytest.mark.parametrize("d,dtype,scale", [(64, HF, 1.3 * 2.0 ** -11), (128, BF, 2.0 ** -14), (32, BF, 1.0), (128, HF, 2.0 ** 9), (64, BF, 65504.0)])
def test_a_long_flat_tail_of_many_rows(d, dtype, scale, what, peak, below=17.0):
    """Weights to 11 bits or 2^-32 of the largest, values to 11 bits or half of 2^-24 times 8; the sum is that of the weights as they
    are, one after another in fp32: 128 of a tile in chains of 32, tiles of a CTA's run."""
    out, lse, want, v, w = tail(d, 40, dtype, scale, peak, what, below, 200)
    N1 = n - 1
    total = 1 + N1 * w
    top = N1 * (2.0 ** -10 * w + 2.0 ** -32) if what == "others" else 2.0 ** -10
    steps = (n / 8 + 64) * 2.0 ** -23 + below * 2.0 ** -21
    bound = v * top / total + 2.0 ** -22 + want * (steps + U[dtype]) + TINY[dtype]
    assert np.all(np.abs(out - want) <= bound), np.abs(out / want - 1).max()
    assert np.all(np.abs(lse - np.log(total)) <= steps + 2.0 ** -22)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("hq", [2, 24])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_scales_over_their_whole_range_along_the_keys(d, hq, up):
    """From f16's smallest to its largest, in order, values of one size a key, all weights alike: each key's part in the sum counts
    as far as 2^-28 of the largest goes."""
    m = 1500
    b = Batch4(3, [1] * 2, [0] * 2, [m, 700], [1, 1], hq, 2, d, 16, BF, alone=True)
    for i, ln in enumerate(b.lens):
        for c in range(ln):
            b.vc[b.own[i, c // 16], :, c % 16] = 7 * 2.0 ** ((c if up else ln - 1 - c) * 39 / (ln - 1) - 24)
    b.kc.zero_()
    b.put(b.kc, b.vc)
    out = f64(b.kv.attend(b.q, *b.args()))
    kc, ks, vc, vs = b.np
    V = N.unpack(vc, vs)
    for i, ln in enumerate(b.lens):
        v = np.concatenate([V[p, :, : min(16, ln - 16 * j)] for j, p in enumerate(b.own[i]) if 16 * j < ln], 1)  # [heads, keys, d]
        want = np.repeat(v.mean(1), hq // 2, 0)
        # (weights are 1 / keys; a floor of 2^-28 of the largest weight times scale each, twice, and 2^-28 of the largest scale)
        bound = want * (2.0 ** -9 + U[BF] + (ln / 8 + 64) * 2.0 ** -23) + 3 * 2.0 ** -28 * v.max()
        assert np.all(np.abs(out[i] - want) <= bound)


@pytest.mark.parametrize("d,hq", [(32, 2), (64, 24), (128, 2)])
def test_scales_before_which_all_others_are_small(d, hq):
    # one key with a large scale in one group, at the context's end, at its beginning and in between
    b = Batch4(4, [1] * 3, [0] * 3, [300, 40, 1000], [1] * 3, hq, 2, d, 16, BF, alone=True)
    for i, c in ((0, 200), (1, 0), (2, 999)):
        b.vc[b.own[i, c // 16], :, c % 16, :8] *= 2.0 ** 10
    b.put(b.kc, b.vc)
    b.check()


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -12, 2.0 ** 10, 2.0 ** 15])
@pytest.mark.parametrize("d,hq", [(32, 2), (64, 24), (128, 2), (128, 24)])
def test_lifted_scales_with_gaps_and_no_numbers(d, hq, size):
    b = Batch4(5, [1] * 3, [0] * 3, [300, 40, 1000], [1] * 3, hq, 2, d, 16, BF, alone=True)
    b.vc *= size / 8
    for c in range(64):  # (tiles of zeros first)
        for i in (0, 2):
            b.vc[b.own[i, c // 16], :, c % 16] = 0
    b.put(b.kc, b.vc)
    _, lse = b.check()
    clean = b.kv.attend(b.q, *b.args()).clone()
    for i, c, bad in ((0, 250, float("nan")), (2, 10, float("-inf"))):
        b.kv.v_scales[int(b.own[i, c // 16]), 1, c % 16, 0] = bad
    out, same = b.kv.attend(b.q, *b.args(), with_lse=True)
    h = hq // 2
    assert torch.isnan(out[0::2, h:, :32]).all() and torch.equal(same, lse) and torch.equal(out[1], clean[1])
    assert torch.equal(out[:, :h], clean[:, :h]) and torch.equal(out[:, h:, 32:], clean[:, h:, 32:])


@pytest.mark.parametrize("dtype", [BF, HF])
def test_negative_scales(dtype):
    # (a cache of the caller's may hold them: they stand for negated numbers)
    b = Batch4(6, [1] * 2, [0] * 2, [100, 40], [1] * 2, 4, 2, 64, 16, dtype, alone=True)
    want = b.kv.attend(b.q, *b.args()).clone()
    b.kv.v_scales.neg_()
    assert torch.equal(b.kv.attend(b.q, *b.args()), -want)
