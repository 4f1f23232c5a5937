"""NaN among the logits of tokens that count: nothing that the loss says of such a row is a number, wherever in the row
they are and whoever reads them; the other rows are as they would be without."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_policy_loss import dev, make  # noqa: E402

PLACES = ["front", "back", "middle", "one", "all", "amid_inf", "last_of_inf"]


def spoil(row, where):
    V, nan = row.shape[0], float("nan")
    if where == "front":
        row[:V // 2] = nan
    elif where == "back":
        row[V // 2:] = nan
    elif where == "middle":
        row[V // 3:V // 3 + V // 5] = nan
    elif where == "one":
        row[V // 7] = nan
    elif where == "all":
        row[:] = nan
    else:
        row[:] = float("-inf")
        row[V // 2 if where == "amid_inf" else V - 1] = nan


@pytest.mark.parametrize("T,V", [(4, 200), (4, 5000), (4, 40000), (4, 150001), (320, 40000), (3, 32769)])
@pytest.mark.parametrize("where", PLACES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grad", [False, True])
def test_rows_with_nan(T, V, where, dtype, grad):
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, ref = make(V, 4, V, dtype)
    n = T // 4 + (T % 4 > 0)
    logits = logits.repeat(n, 1)[:T]
    y, adv, w, old, ref = (np.tile(a, n)[:T] for a in (y, adv, w, old, ref))
    a = (dev(y, torch.int32), dev(adv), dev(w))
    kw = dict(old_logp=dev(old), ref_logp=dev(ref), beta=0.1, with_grad=grad)
    clean = policy_loss(logits, *a, **kw)
    for t in (1, T - 1):
        spoil(logits[t], where)
    r = policy_loss(logits, *a, **kw)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[1, T - 1]] = True
    for name in ("logp", "lse", "terms", "coef"):
        got = getattr(r, name)
        assert torch.isnan(got[bad]).all(), name
        assert torch.equal(got[~bad], getattr(clean, name)[~bad]), name
    assert torch.isnan(r.loss)
    if grad:
        assert torch.isnan(r.grad[bad]).all() and torch.equal(r.grad[~bad], clean.grad[~bad])


@pytest.mark.parametrize("T,V", [(5, 64), (5, 40000), (400, 40000)])
@pytest.mark.parametrize("token", [-1, "V", 2 ** 31 - 1])
def test_an_invalid_token_leaves_no_number(T, V, token):
    """Its lse too: nothing of such a row is to be used."""
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, _ = make(V, 5, V, torch.bfloat16)
    n = T // 5
    logits = logits.repeat(n, 1)
    y, adv, w, old = (np.tile(a, n) for a in (y, adv, w, old))
    y[2] = V if token == "V" else token
    status = dev([0], torch.int32)
    r = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old), status=status)
    assert status.item() == 1
    for name in ("logp", "lse", "terms", "coef"):
        got = torch.isnan(getattr(r, name))
        assert got[2] and got.sum() == 1, name
    assert torch.isnan(r.loss) and torch.isnan(r.grad[2]).all() and torch.isnan(r.grad).any(1).sum() == 1
