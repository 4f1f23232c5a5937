"""fe_verify_drafts where a token hangs on the last digits of the sums: random numbers next to the border between two tokens,
after rejections whose p - q does not fit 32 bits."""
from fractions import Fraction

import numpy as np
import pytest

from tests import nibble_oracle as N

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


def run(p, q, y, start, accept, sample, dtype):
    """(out, accepted) of the call and of the method, on the values that the type holds."""
    from paper_2603_02565_gb300 import verify_drafts
    p, q = (torch.tensor(x, dtype=torch.float32).to(dtype) for x in (p, q))
    y, start = (torch.tensor(x, dtype=torch.int32) for x in (y, start))
    accept, sample = (torch.tensor(x, dtype=torch.float32) for x in (accept, sample))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = verify_drafts(p.cuda(), y.cuda(), start.cuda(), accept.cuda(), sample.cuda(), draft_probs=q.cuda(), status=status)
    assert status.item() == 0
    return [x.cpu().numpy() for x in got], N.verify(p, q, y.numpy(), start.numpy(), accept.numpy(), sample.numpy())


def test_a_draw_next_to_a_border():
    # by the definition, 0; sums that lose 2^-25 of p - q give 1
    for p, q, u in (([0.5393387, 0.2069038, 0.0], [0.02098919, 0.0, 0.5], 0.7147151),
                    ([0.7104367, 0.2895633, 0.0], [0.082448214, 0.0, 0.5], 0.6844175)):
        (out, n), (want, wn) = run([p, p], [q, q], [2, 0], [0, 2], [0.9, 0.9], [u], F32)
        assert n.tolist() == wn.tolist() == [0] and out.tolist() == want.tolist() == [0, -1]


def remainders(rng, S, V, dtype):
    """Rows of p and q whose difference often has a tie at 2^-22 or 2^-23, and digits of q below the 24 of it; the last token
    is drafted and has p = 0, q = 0.5."""
    p, q = np.zeros((S, V), np.float32), np.zeros((S, V), np.float32)
    at = np.argsort(rng.rand(S, V - 1), axis=1)[:, : min(6, V - 1)]
    steps = {F32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11}[dtype]
    for c in range(at.shape[1]):
        top = rng.choice([1.0, 0.5, 0.25], S)
        x = np.floor(rng.uniform(0.5, 1, S) / steps) * steps * top
        p[np.arange(S), at[:, c]] = x
        small = 2.0 ** -rng.uniform(*((1.5, 30) if dtype is F32 else (17, 24)), S)
        q[np.arange(S), at[:, c]] = np.where(rng.rand(S) < 0.8, np.minimum(small, x), 0)
    q[:, -1] = 0.5
    return p, q


@pytest.mark.parametrize("dtype,V", [(F32, 3), (F32, 8), (F32, 301), (BF, 3), (BF, 16), (BF, 401), (HF, 16)])
def test_random_numbers_next_to_the_borders_between_tokens(dtype, V):
    S = 3000
    rng = np.random.RandomState(V)
    p, q = remainders(rng, S, V, dtype)
    held = [x.to(torch.float64).numpy() for x in (torch.from_numpy(p).to(dtype), torch.from_numpy(q).to(dtype))]
    w = np.maximum(held[0] - held[1], 0)
    sample = np.zeros(S, np.float32)
    for s in range(S):
        tokens = np.flatnonzero(w[s])
        k = rng.randint(0, max(1, len(tokens) - 1))
        part = sum((Fraction(w[s, i]) for i in tokens[: k + 1]), Fraction(0)) / sum(Fraction(w[s, i]) for i in tokens)
        u = np.float32(float(part))
        sample[s] = [u, np.nextafter(u, np.float32(0)), np.nextafter(u, np.float32(2))][s % 3]
    sample = np.clip(sample, 0, np.float32(1 - 2.0 ** -24))
    rows = lambda x: np.repeat(x, 2, axis=0)  # noqa: E731
    (out, n), (want, wn) = run(rows(p), rows(q), np.full(2 * S, V - 1), 2 * np.arange(S + 1), np.full(2 * S, 0.9), sample, dtype)
    assert not n.any() and np.array_equal(n, wn)
    assert np.array_equal(out, want), np.flatnonzero(out != want)[:5]


@pytest.mark.parametrize("dtype", [F32, BF])
def test_probabilities_of_one_and_next_to_it(dtype):
    # w next to 1, where the coarse part of a sum is at the end of its range
    S, V = 200, 5
    rng = np.random.RandomState(9)
    p, q = np.zeros((S, V), np.float32), np.zeros((S, V), np.float32)
    p[:, 0] = rng.choice([1.0, 1 - 2.0 ** -24, 1 - 2.0 ** -8, 0.5], S)
    p[:, 2] = rng.choice([1.0, 1 - 2.0 ** -24, 1 - 2.0 ** -8, 2.0 ** -30], S)
    q[:, 0], q[:, 2], q[:, -1] = 2.0 ** -rng.uniform(20, 60, S), 2.0 ** -rng.uniform(20, 60, S), 0.5
    sample = rng.choice(np.float32([0, 0.5, 0.5 - 2.0 ** -25, 1 - 2.0 ** -24]), S)
    rows = lambda x: np.repeat(x, 2, axis=0)  # noqa: E731
    (out, n), (want, wn) = run(rows(p), rows(q), np.full(2 * S, V - 1), 2 * np.arange(S + 1), np.full(2 * S, 0.9), sample, dtype)
    assert np.array_equal(n, wn) and np.array_equal(out, want)
