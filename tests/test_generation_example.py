"""The generator, the evaluator and the loss together, as examples/generate_and_learn.py runs them."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate_and_learn.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("generate_and_learn", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def generator(example, B=3, K=5, L=20, C=50, M=40, d=128):
    g = torch.Generator(device="cuda").manual_seed(3)
    context, pool = (torch.randn(B, n, d, generator=g, device="cuda").to(torch.bfloat16) * s for n, s in ((C, 1.0), (M, d ** -0.5)))
    return example.Generator(context, pool, K, L)


def dense(gen, tokens):
    """Hidden states of the candidates in float64 on the CPU: context and candidate rows in one causal sequence."""
    B, K, L, C = gen.B, gen.K, gen.L, gen.C
    S, h, kv, e = B * K, gen.heads, gen.kv_heads, gen.head_dim
    own = torch.cat([gen.begin.expand(S, 1, -1), gen.embed(tokens[:, :-1])], 1)
    x = torch.cat([gen.context.repeat_interleave(K, 0), own], 1).cpu().double()
    n = C + L
    rope = gen.rope[:n].cpu().double()
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]

    def turn(y):
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for w, mix in zip(gen.qkv, gen.mix):
        q, k, v = (x @ w.cpu().double()).view(S, n, -1, e).split([h, kv, kv], 2)
        q, k = turn(q).transpose(1, 2), turn(k).transpose(1, 2).repeat_interleave(h // kv, 1)
        v = v.transpose(1, 2).repeat_interleave(h // kv, 1)
        a = (q @ k.transpose(2, 3) * e ** -0.5 + torch.full((n, n), -torch.inf, dtype=torch.float64).triu(1)).softmax(-1)
        x = x + (a @ v).transpose(1, 2).reshape(S, n, -1) @ mix.cpu().double()
    return x[:, C:]


def test_cached_attention_is_the_dense_one(example):
    gen = generator(example)
    gen.read_context()
    tokens, logp = gen.write()
    hidden, logits = gen.read_candidates(tokens)
    example.check_status(gen.status)
    want = dense(gen, tokens)
    # two layers of about six roundings to bf16 (2^-9 of the value in the mean square's root, at most 2^-8): well under 2^-4
    assert (hidden.cpu().double() - want).norm() <= 2.0 ** -5 * want.norm()
    # and a token at a time writes what all rows at once read
    again = torch.log_softmax(logits.float(), -1).gather(2, tokens[..., None].long())[..., 0]
    assert (again - logp).abs().mean() <= 2.0 ** -5 * logits.float().masked_fill(logits.isinf(), 0).abs().amax()


def test_the_gradient_of_the_step_is_autograds(example):
    gen = generator(example)
    gen.read_context()
    tokens, logp = gen.write()
    hidden, logits = gen.read_candidates(tokens)
    adv = torch.randn(tokens.shape[0], device="cuda")
    x = logits.double().requires_grad_()
    lp = torch.log_softmax(x, -1).gather(2, tokens[..., None].long())[..., 0]
    r = (lp - logp.double()).exp()
    a = adv.double()[:, None]
    loss = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a).mean()
    loss.backward()
    before = gen.out.clone()
    got = gen.learn(tokens, logp, adv, 1.0)
    n = logp.numel()
    # fp32 sums of n terms of size 1, and a gradient rounded once to bf16
    assert abs(got.loss.item() - loss.item()) <= 2.0 ** -18
    g = got.grad.view_as(x).double() / n
    assert (g - x.grad).norm() <= 2.0 ** -8 * x.grad.norm()
    assert abs((gen.out - before).norm().item() - 1) <= 1e-3


def test_scores_rise(example):
    means = example.run(requests=4, candidates=32, length=6, steps=25, tell=lambda s: None)
    assert sum(means[-5:]) > sum(means[:5])
