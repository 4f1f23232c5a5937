"""fe_policy_loss and its backward entry on the GPU against float64: vocabulary sizes and alignments,
types, masked and invalid tokens, infinite logits; the gradient against its formula and against differences."""
import numpy as np
import pytest

from tests import generation_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32 = torch.float32


def dev(a, dtype=F32):
    return None if a is None else torch.tensor(np.asarray(a), dtype=dtype, device=DEV)


def make(seed, T, V, dtype, row=None, masked=0.0, temperature=1.0):
    rng = np.random.RandomState(seed)
    row = row or V
    store = torch.tensor(rng.randn(T, row) * 2, dtype=F32).to(dtype).to(DEV)
    logits = store[:, :V]
    y = rng.randint(0, V, T)
    logits[torch.arange(T), torch.tensor(y)] += 4
    x = O.f64(logits) / temperature
    lp = x[np.arange(T), y] - (x.max(1) + np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)))
    f = lambda a: np.asarray(a, dtype=np.float32).astype(np.float64)  # noqa: E731  (inputs are fp32)
    w = f(rng.rand(T) + 0.1)
    w[rng.rand(T) < masked] = 0
    # ratios from 0.5 to 2 on both sides of the clip range, none at its ends
    return logits, y, f(rng.randn(T)), w, f(lp - rng.choice([-0.6, -0.1, 0.0, 0.1, 0.6], T)), f(lp + rng.randn(T) * 0.3)


def check(got, want, dtype, grad_scale, temperature, adv, w, old, ref, beta):
    loss, terms, logp, lse, coef, grad, eps = want
    live = w != 0
    z = np.zeros(len(w))
    r = np.ones(len(w)) if old is None else np.exp(logp - old)
    slope = w * (np.abs(adv) * r + (0 if ref is None else beta * np.exp(ref - logp)))
    for name, value, bound in (("logp", logp, eps), ("lse", lse, eps), ("terms", terms, 2 * eps * slope + 2.0 ** -21 * np.abs(terms)),
                               ("coef", coef, 2 * eps * slope + 2.0 ** -21 * np.abs(coef))):
        g = O.f64(getattr(got, name))
        value = np.where(live, value, z)
        assert np.all(np.abs(g - value) <= bound), (name, np.max(np.abs(g - value) / bound))
    t = np.where(live, terms, z)
    assert abs(O.f64(got.loss) - t.sum()) <= (2 * eps * slope).sum() + 2.0 ** -21 * np.abs(t).sum()
    if got.grad is not None:
        check_grad(got.grad, want, dtype, grad_scale, temperature, w, slope)


def check_grad(g, want, dtype, grad_scale, temperature, w, slope):
    coef, grad, eps = want[4], want[5], want[6]
    live = (w != 0)[:, None]
    k = grad_scale / temperature
    hot_minus_p = np.abs(grad) / np.maximum(np.abs(k * coef)[:, None], 1e-300)
    bound = k * (2 * eps * slope)[:, None] * hot_minus_p + np.abs(k * coef)[:, None] * (2 * eps[:, None] + 2.0 ** -21) * hot_minus_p
    bound = bound + 2.0 ** -22 * np.abs(k * coef)[:, None] * (hot_minus_p < 1) * hot_minus_p + O.U[dtype] * np.abs(grad) + O.TINY[dtype]
    # where the one-hot and the softmax nearly cancel the error is that of the softmax
    bound = bound + np.abs(k * coef)[:, None] * np.where(np.sign(grad) == np.sign(coef)[:, None], 4 * eps[:, None], 0)
    got = O.f64(g)
    want_g = np.where(live, grad, 0)
    assert np.all(np.abs(got - want_g) <= bound * 1.001 + 1e-300), np.max(np.abs(got - want_g) / (bound + 1e-300))


SIZES = [(1, 1), (2, 2), (5, 7), (3, 33), (4, 1000), (9, 4097), (3, 32768), (2, 50021), (2, 131072), (1, 200003), (1, 300000)]


@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F32])
def test_matches_the_definition(T, V, dtype):
    from paper_2603_02565_gb300 import policy_loss
    clip, beta, temperature, scale = (0.2, 0.3), 0.05, 0.8, 64.0
    logits, y, adv, w, old, ref = make(T + V, T, V, dtype, masked=0.3, temperature=temperature)
    want = O.policy(logits, y, adv, w, old, ref, clip, beta, temperature, scale)
    a = (logits, dev(y, torch.int32), dev(adv), dev(w))
    kw = dict(old_logp=dev(old), ref_logp=dev(ref), clip=clip, beta=beta, temperature=temperature, grad_scale=scale)
    status = dev([0], torch.int32)
    got = policy_loss(*a, status=status, **kw)
    assert status.item() == 0
    check(got, want, dtype, scale, temperature, adv, w, old, ref, beta)
    alone = policy_loss(*a, with_grad=False, **kw)
    assert alone.grad is None
    check(alone, want, dtype, scale, temperature, adv, w, old, ref, beta)


@pytest.mark.parametrize("V,row", [(1000, 1001), (1003, 1024), (40000, 40007), (8, 9), (3, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
def test_rows_apart_and_misaligned(V, row, dtype):
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, ref = make(V, 6, V, dtype, row=row)
    want = O.policy(logits, y, adv, w, old, ref, (0.2, 0.2), 0.1, 1.0, 1.0)
    kw = dict(old_logp=dev(old), ref_logp=dev(ref), beta=0.1)
    a = (logits, dev(y, torch.int32), dev(adv), dev(w))
    got = policy_loss(*a, **kw)
    check(got, want, dtype, 1.0, 1.0, adv, w, old, ref, 0.1)
    # a gradient whose rows are aligned differently, and what lies between its rows
    store = torch.full((6, V + 5), 7.0, dtype=dtype, device=DEV)
    other = policy_loss(*a, grad=store[:, 2:2 + V], **kw)
    check(other, want, dtype, 1.0, 1.0, adv, w, old, ref, 0.1)
    assert (store[:, :2] == 7).all() and (store[:, 2 + V:] == 7).all()


def test_in_place_of_the_logits():
    from paper_2603_02565_gb300 import policy_loss
    for V in (777, 32768, 140001):
        logits, y, adv, w, old, ref = make(V, 4, V, torch.bfloat16, masked=0.2)
        a = (dev(y, torch.int32), dev(adv), dev(w))
        want = policy_loss(logits, *a, old_logp=dev(old))
        got = policy_loss(logits, *a, old_logp=dev(old), grad=logits)
        assert got.grad.data_ptr() == logits.data_ptr() and torch.equal(got.grad, want.grad)
        assert torch.equal(got.loss, want.loss)


def test_the_present_policy_without_kl_and_weights():
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, _, _ = make(1, 8, 500, F32)
    w = np.full(8, np.float32(1 / 8), np.float64)
    want = O.policy(logits, y, adv, w, None, None, (0.2, 0.2), 0.0, 1.0, 1.0)
    got = policy_loss(logits, dev(y, torch.int32), dev(adv))
    check(got, want, F32, 1.0, 1.0, adv, w, None, None, 0.0)


def test_gradient_against_differences():
    # central differences of the float64 loss at the kernel's logits, along random directions
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, ref = make(2, 6, 91, F32, masked=0.2, temperature=1.3)
    kw = dict(clip=(0.2, 0.2), beta=0.2, temperature=1.3)
    got = O.f64(policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old), ref_logp=dev(ref), **kw).grad)
    rng, x, h = np.random.RandomState(3), O.f64(logits), 1e-5
    loss = lambda z: O.policy(torch.tensor(z), y, adv, w, old, ref, kw["clip"], kw["beta"], kw["temperature"], 1.0)[0]  # noqa: E731
    for _ in range(10):
        u = rng.randn(*x.shape)
        slope = (loss(x + h * u) - loss(x - h * u)) / (2 * h)
        # third derivatives times h^2, 64-bit cancellation over h, and the kernel's fp32
        assert abs((got * u).sum() - slope) <= 1e-8 + 1e-5 * np.abs(got * u).sum()


@pytest.mark.parametrize("V", [600, 32768, 150001])
@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
def test_backward_from_saved_statistics(V, dtype):
    from paper_2603_02565_gb300 import policy_loss, policy_loss_backward
    logits, y, adv, w, old, ref = make(V, 5, V, dtype, masked=0.3)
    a, kw = (logits, dev(y, torch.int32)), dict(old_logp=dev(old), ref_logp=dev(ref), beta=0.1)
    r = policy_loss(*a, dev(adv), dev(w), with_grad=False, **kw)
    want = O.policy(logits, y, adv, w, old, ref, (0.2, 0.2), 0.1, 1.0, 2.5 * 8)
    g = policy_loss_backward(*a, r, dev(w), upstream=dev([2.5]), grad_scale=8.0)
    slope = w * (np.abs(adv) * np.exp(want[2] - old) + 0.1 * np.exp(ref - want[2]))
    check_grad(g, want, dtype, 20.0, 1.0, w, slope)


@pytest.mark.parametrize("V", [50, 40000])
def test_infinite_logits_and_masked_rows(V):
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, _ = make(5, 6, V, torch.bfloat16)
    clean = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old))
    # forbidden words; a whole row of them; a row with NaN, and one of +inf, both masked
    logits[0, 1:] = float("-inf")
    logits[0, 0] = 1.0
    y[0], w[3], w[4] = 0, 0, 0
    logits[2, :] = float("-inf")
    logits[3, 7] = float("nan")
    logits[4, :] = float("inf")
    r = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old))
    assert r.logp[0] == 0 and (r.grad[0] == 0).all()
    assert torch.isnan(r.logp[2]) and torch.isneginf(r.lse[2]) and torch.isnan(r.grad[2]).all() and torch.isnan(r.loss)
    assert (r.grad[3:5] == 0).all() and (r.terms[3:5] == 0).all() and (r.logp[3:5] == 0).all()
    assert torch.equal(r.grad[1], clean.grad[1]) and torch.equal(r.grad[5], clean.grad[5])


def test_the_chosen_word_has_probability_zero():
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, _ = make(6, 3, 100, F32)
    logits[1, y[1]] = float("-inf")
    r = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old))
    assert torch.isneginf(r.logp[1]) and r.terms[1] == (0 if adv[1] >= 0 else r.terms[1]) and not torch.isnan(r.loss)
    assert r.grad[1, y[1]] == 0 or adv[1] < 0


def test_invalid_tokens_are_nan_and_reported():
    from paper_2603_02565_gb300 import policy_loss, FeError, check_status
    logits, y, adv, w, old, _ = make(7, 5, 64, torch.float16)
    clean = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old))
    y[1], y[3] = 64, -1
    w[3] = 0  # (a masked token's index does not matter)
    status = dev([0], torch.int32)
    r = policy_loss(logits, dev(y, torch.int32), dev(adv), dev(w), old_logp=dev(old), status=status)
    with pytest.raises(FeError):
        check_status(status)
    assert torch.isnan(r.logp[1]) and torch.isnan(r.grad[1]).all() and torch.isnan(r.loss)
    for t in (0, 2, 4):
        assert torch.equal(r.grad[t], clean.grad[t]) and r.logp[t] == clean.logp[t]
    assert (r.grad[3] == 0).all()


def test_same_result_every_time_and_in_a_graph():
    from paper_2603_02565_gb300 import policy_loss
    logits, y, adv, w, old, ref = make(8, 300, 5000, torch.bfloat16)
    a, kw = (logits, dev(y, torch.int32), dev(adv), dev(w)), dict(old_logp=dev(old), ref_logp=dev(ref), beta=0.1)
    want = policy_loss(*a, **kw)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = policy_loss(*a, stream=side, **kw)
        side.synchronize()
        assert torch.equal(got.loss, want.loss) and torch.equal(got.grad, want.grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = policy_loss(*a, **kw)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held.loss, want.loss) and torch.equal(held.grad, want.grad)


def test_no_tokens():
    from paper_2603_02565_gb300 import policy_loss
    r = policy_loss(torch.empty(0, 10, device=DEV), dev([], torch.int32), dev([]))
    assert r.loss.item() == 0 and r.grad.shape == (0, 10)
