"""Attention weights far below their row's largest: many of them together count, in either type of pages."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import BF, HF, Batch, i32  # noqa: E402


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("peak", ["first", "middle", "last", "own"])
@pytest.mark.parametrize("groups", [1, 700])
@pytest.mark.parametrize("below", [20.0, 25.5, 28.0])
def test_a_long_flat_tail_under_a_peak(dtype, d, peak, groups, below):
    """One key holds the whole weight but for 2^-below each of 32768 others, whose values are 1 where its own are 0.
    All groups read the same pages; 700 of them leave each to a few CTAs, which meet the peak's scale with the tail's.

    Out is N 2^-below / (1 + N 2^-below).  A weight is rounded to the pages' type: relatively (u) as long as it is a
    normal number; f16's subnormal ones by up to 2^-25 on a scale whose largest is at least 2^7, so that all N
    are off by N 2^-32 of the peak's at most."""
    from paper_2603_02565_gb300 import PagedKV
    n = 32768
    b = Batch(1, [1], [n], [1], [1], 1, 1, d, 128, dtype)
    kc, vc = torch.zeros_like(b.kc), torch.ones_like(b.vc)
    kc[..., 0] = -below * np.log(2.0)
    page, at = {"first": (b.pre[0, 0], 0), "middle": (b.pre[0, 90], 77), "last": (b.pre[0, -1], 127), "own": (b.own[0, 0], 0)}[peak]
    kc[page, 0, at], vc[page, 0, at] = 0, 0
    q = torch.zeros(groups, 1, d, dtype=dtype, device="cuda")
    q[..., 0] = 1
    each, ones = i32(np.arange(groups + 1)), i32(np.ones(groups))
    out, lse = PagedKV(kc, vc).attend(q, each, ones, i32(np.repeat(b.own, groups, 0)), each, n * ones,
                                      i32(np.repeat(b.pre, groups, 0)), scale=1.0, with_lse=True)
    weight = np.exp(float(kc.to(torch.float64).min()))  # (the type's rounding of the keys is part of the input)
    want = n * weight / (1 + n * weight)
    u = O.U[dtype]
    off = (n * 2.0 ** -32 if dtype is HF else 0) + u * want
    # scores: one product, exact but for the exponent's fp32 (2^-22 times its size) and the sums' (as many terms)
    off = off + want * (below * 2.0 ** -21 + (n + 64) * 2.0 ** -24)
    assert np.all(np.abs(O.f64(out) - want) <= off + u * want + O.TINY[dtype])
    # (the oracle's bound of a sum of n + 1 terms, the largest of them 1)
    assert np.all(np.abs(O.f64(lse) - np.log1p(n * weight)) <= (n + 1 + 64) * 2.0 ** -22)
