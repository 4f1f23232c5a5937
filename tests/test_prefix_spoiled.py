"""Attention over very many rows that have to be computed again or are refused: more than a list of 65536 would hold."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_prefix_attention import BF, HF, Batch, i32  # noqa: E402

INDEX = 1


@pytest.mark.parametrize("S,hq,hkv", [(40, 8, 2), (1100, 64, 1), (1100, 64, 64)])
@pytest.mark.parametrize("prefix", [0, 40])
def test_refused_lengths_of_rows_without_keys(S, hq, hkv, prefix):
    """Lengths past the page tables leave no keys of their own; the last group's rows are as they should be (not to
    the bit: where units are split follows from all lengths)."""
    from paper_2603_02565_gb300 import PagedKV
    lens = [3] * (S + 3)
    b = Batch(1, [S, 3], [prefix, 5], lens, [1] * (S + 3), hq, hkv, 32, 16, BF)
    kv = PagedKV(b.kc, b.vc)
    want, want_lse, eo, el = O.attend(b.q[S:], b.kc, b.vc, np.arange(4), b.lens[S:], b.own[S:], [0, 3], [5], b.pre[1:], 32 ** -0.5)
    bound = (O.U[BF] + 2 * el[..., None]) * eo + O.U[BF] * np.abs(want) + 2.0 ** -24 * eo
    bad = np.array(lens)
    bad[:S] = b.own.shape[1] * 16 + 1
    for fill in (0.0, float("nan")):
        status, out = i32([0]), torch.full_like(b.q, fill)
        _, lse = kv.attend(b.q, *b.args(lengths=bad), with_lse=True, status=status, out=out)
        assert status.item() == INDEX
        assert torch.isnan(out[:S]).all() and torch.isnan(lse[:S]).all()
        assert np.all(np.abs(O.f64(out[S:]) - want) <= bound) and np.all(np.abs(O.f64(lse[S:]) - want_lse) <= el)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_rows_computed_again_beside_a_split_unit(dtype):
    """70400 rows x heads whose sequences hold a value that is no number, and a prefix of 20000 keys that many CTAs
    share: the rows of that prefix do not depend on what `out` held, nor on the other groups."""
    from paper_2603_02565_gb300 import PagedKV
    S, hq, hkv, d = 1100, 64, 1, 32
    lens = np.array([4] * S + [9, 2, 30])
    b = Batch(2, [S, 3], [0, 20000], lens, [1] * (S + 3), hq, hkv, d, 16, dtype)
    kv = PagedKV(b.kc, b.vc)
    want, want_lse = kv.attend(b.q, *b.args(), with_lse=True)
    pages = torch.tensor(b.own[:S, 0], dtype=torch.long, device="cuda")
    b.vc[pages, :, 2, 7] = float("inf")
    for fill in (0.0, float("nan"), float("-inf"), 3.0):
        for _ in range(3):
            out = torch.full_like(b.q, fill)
            _, lse = kv.attend(b.q, *b.args(), with_lse=True, out=out)
            assert torch.equal(out[S:], want[S:]) and torch.equal(lse[S:], want_lse[S:])
            assert torch.isinf(out[:S, :, 7]).all()
            rest = [i for i in range(d) if i != 7]
            # (computed again key by key: rounded once where the first way also rounds the weights)
            assert torch.allclose(out[:S, :, rest].float(), want[:S, :, rest].float(), rtol=2.0 ** -6, atol=2.0 ** -6)
