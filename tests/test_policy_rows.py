"""fe_policy_loss at the sizes where the way a row is held changes, and sums of many tokens."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_policy_loss import check, dev, make  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("V", [1024, 1025, 2048, 2055, 4090, 8192, 8200, 12290, 16384, 16400, 24576, 24600, 32760, 32776])
@pytest.mark.parametrize("off", [0, 3])
@pytest.mark.parametrize("grad", [False, True])
def test_rows_around_every_size_limit(V, off, grad):
    from paper_2603_02565_gb300 import policy_loss
    clip, beta, temperature, scale = (0.2, 0.3), 0.05, 0.8, 8.0
    logits, y, adv, w, old, ref = make(V + off, 7, V + off, BF, row=V + 16, masked=0.3, temperature=temperature)
    logits, y = logits[:, off:], np.maximum(y - off, 0)  # rows that begin off a 16-byte boundary
    x = O.f64(logits) / temperature
    lp = x[np.arange(7), y] - (x.max(1) + np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)))
    old, ref = ((lp + d).astype(np.float32).astype(np.float64) for d in (-0.1, 0.2))
    want = O.policy(logits, y, adv, w, old, ref, clip, beta, temperature, scale)
    kw = dict(old_logp=dev(old), ref_logp=dev(ref), clip=clip, beta=beta, temperature=temperature, grad_scale=scale)
    got = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), with_grad=grad, **kw)
    check(got, want, BF, scale, temperature, adv, w, old, ref, beta)


@pytest.mark.parametrize("V", [1, 40, 9000])
def test_gradient_rows_of_tokens_without_weight(V):
    from paper_2603_02565_gb300 import policy_loss
    for dtype in (BF, F32):
        logits = torch.randn(6, V + 3, device="cuda").to(dtype)[:, 1:1 + V]
        store = torch.full((6, V + 5), 7.0, dtype=dtype, device="cuda")
        w = dev([0, 1, 0, 0, 1, 0])
        r = policy_loss(logits, dev([0] * 6, torch.int32), dev(np.ones(6)), w, grad=store[:, 2:2 + V])
        assert (store[:, :2] == 7).all() and (store[:, 2 + V:] == 7).all()
        assert (r.grad[w == 0] == 0).all() and (V == 1 or (r.grad[w != 0] != 0).any())


@pytest.mark.parametrize("T", [2047, 2048, 2049, 5000, 16389])
def test_sum_over_many_tokens(T):
    from paper_2603_02565_gb300 import policy_loss
    rng = np.random.RandomState(T)
    logits = torch.tensor(rng.randn(T, 24), dtype=F32, device="cuda")
    adv = (rng.randn(T) * 10.0 ** rng.uniform(-3, 3, T)).astype(np.float32)
    a = (logits, dev(rng.randint(0, 24, T), torch.int32), dev(adv), dev(rng.rand(T)))
    r, again = policy_loss(*a), policy_loss(*a)
    terms = O.f64(r.terms)
    # the terms are added in 64 bits and the sum is rounded once
    assert abs(O.f64(r.loss) - terms.sum()) <= 2.0 ** -24 * abs(terms.sum()) + T * 2.0 ** -52 * np.abs(terms).sum()
    assert torch.equal(r.loss, again.loss)
