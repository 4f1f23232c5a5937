"""The gradient that policy_loss allocates begins as far off a 16-byte boundary as the logits do, row for row, so that it
leaves in whole pieces; and the kernels that hold rows in registers write rows that begin anywhere."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2603_02565_gb300 import generation as G  # noqa: E402
from tests import generation_oracle as O  # noqa: E402


def views(dtype, device):
    x = torch.zeros(5 * 40 + 8, dtype=dtype, device=device)
    yield x[:200].view(5, 40)
    for off in range(1, 8):
        yield x[off:off + 200].view(5, 40)          # contiguous, off a boundary
        yield x[:200].view(5, 40)[:, off:]          # rows apart
        yield x[:200].view(5, 40)[:1, off:off + 9]  # one row
        yield x[:200].view(5, 40)[:, off:off + 1]   # one word
        yield x[:200].view(5, 40)[:0, off:]         # no row


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_new_gradient_is_aligned_as_the_logits(dtype, device):
    for x in views(dtype, device):
        T, V = x.shape
        row = x.stride(0) if T > 1 else max(V, x.stride(0))
        g, at = G._grad(x, row, None, None)
        assert g.shape == x.shape and g.dtype is dtype and g.device == x.device and at == row
        assert T < 2 or g.stride(0) == row
        if T:
            assert g.stride(1) == 1 or V == 1
            assert g.data_ptr() % 16 == x.data_ptr() % 16
            assert g.untyped_storage().nbytes() >= (g.storage_offset() + (T - 1) * row + V) * x.element_size()
            g.fill_(1)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [7, 1024, 1025, 2048, 2055, 4090, 8192, 8200, 12290, 16384, 16400, 24576, 24600, 32760, 32776])
@pytest.mark.parametrize("off", [0, 1, 3, 5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_of_rows_off_a_boundary(V, off, dtype):
    """In place of the logits, in a buffer with the same offset, and allocated: the same bits, nothing around them."""
    from tests.test_policy_loss import check, dev, make
    clip, beta, temperature, scale = (0.2, 0.3), 0.05, 0.8, 8.0
    logits, y, adv, w, old, ref = make(V + off, 7, V + off, dtype, row=V + 16, masked=0.3, temperature=temperature)
    logits, y = logits[:, off:], np.maximum(y - off, 0)
    x = O.f64(logits) / temperature
    lp = x[np.arange(7), y] - (x.max(1) + np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)))
    old, ref = ((lp + d).astype(np.float32).astype(np.float64) for d in (-0.1, 0.2))
    want = O.policy(logits, y, adv, w, old, ref, clip, beta, temperature, scale)
    a = (logits, dev(y, torch.int32), dev(adv), dev(w))
    kw = dict(old_logp=dev(old), ref_logp=dev(ref), clip=clip, beta=beta, temperature=temperature, grad_scale=scale)
    got = G.policy_loss(*a, **kw)
    assert got.grad.data_ptr() % 16 == logits.data_ptr() % 16
    check(got, want, dtype, scale, temperature, adv, w, old, ref, beta)
    store = torch.full((7, V + 16), 7.0, dtype=dtype, device="cuda")
    same = G.policy_loss(*a, grad=store[:, off:off + V], **kw)
    assert torch.equal(same.grad, got.grad) and (store[:, :off] == 7).all() and (store[:, off + V:] == 7).all()
    r = G.policy_loss(*a, with_grad=False, **kw)
    assert torch.equal(r.logp, got.logp)
    back = G.policy_loss_backward(logits, a[1], r, a[3], temperature=temperature, grad_scale=scale)
    assert back.data_ptr() % 16 == logits.data_ptr() % 16
    G.policy_loss(*a, grad=logits, **kw)
    assert torch.equal(logits, got.grad)
