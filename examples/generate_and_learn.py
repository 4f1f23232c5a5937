"""A candidate generator beside the evaluator: it writes each request's K candidate sequences, the
evaluator scores them, and the generator learns from the scores.

    python examples/generate_and_learn.py [--requests 16] [--candidates 50] [--length 6] [--steps 30]

The generator is a small attention model over the request: its context rows are the prefix that the K
candidates share, each candidate token is a row of the request's pool (taken once at most), and a token's logits are
its hidden state's products with the pool's rows.  One round:

1. read the contexts (PagedKV.append and .attend, all rows of a request at once);
2. write K candidates per request, a token of all of them at a time (append and attend, one row per sequence);
3. Evaluator.evaluate scores the candidates; a request's advantages are its scores, standardised;
4. read the written candidates again in one pass (many rows per sequence) for their logits, take policy_loss
   with its gradient, and step the output projection down it.

Weights and requests are random: this shows the path, not a trained model.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2603_02565_gb300 import Evaluator, PagedKV, check_status, policy_loss, rotary_table  # noqa: E402
from paper_2603_02565_gb300 import workloads as wl  # noqa: E402

PAGE = 16


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


class Generator:
    """Attention layers without anything between them; `out` is what learns."""

    def __init__(self, context, pool, K, L, heads=8, kv_heads=4, head_dim=32, n_layers=2, seed=0):
        self.context, self.pool, self.K, self.L = context, pool, K, L
        self.B, self.C, d = context.shape
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.rng = g
        self.begin = rand(1, d) * d ** 0.5
        self.qkv = [rand(d, (heads + 2 * kv_heads) * head_dim) for _ in range(n_layers)]
        self.mix = [rand(heads * head_dim, d) for _ in range(n_layers)]
        self.out = torch.eye(d, device="cuda")
        # pages: a request's context first, then one run of pages for each of its candidates
        B, C = self.B, self.C
        pre, own = -(-C // PAGE), -(-L // PAGE)
        self.prefix_pages = torch.arange(B * pre, dtype=torch.int32, device="cuda").view(B, pre)
        self.pages = B * pre + torch.arange(B * K * own, dtype=torch.int32, device="cuda").view(B * K, own)
        self.cache = [PagedKV.empty(B * (pre + K * own), PAGE, kv_heads, head_dim) for _ in range(n_layers)]
        self.rope = rotary_table(C + L, head_dim)
        self.status = i32([0])
        self.prefix, self.none = i32([C] * B), i32([0] * B)
        self.groups = K * torch.arange(B + 1, dtype=torch.int32, device="cuda")
        self.each = torch.arange(B + 1, dtype=torch.int32, device="cuda")  # groups of one sequence

    def layers(self, x, row_start, first, lengths, pages, shift, groups, prefix, prefix_pages):
        """Hidden states [rows, d] of rows that follow the first[s] rows each sequence holds."""
        h, kv, e = self.heads, self.kv_heads, self.head_dim
        for cache, w, mix in zip(self.cache, self.qkv, self.mix):
            q, k, v = (x @ w).view(-1, h + 2 * kv, e).split([h, kv, kv], 1)  # (strided: nothing is copied)
            q = cache.append(k, v, row_start, first, pages, q=q, rope=self.rope, shift=shift, status=self.status)
            o = cache.attend(q, row_start, lengths, pages, groups, prefix, prefix_pages, status=self.status)
            x = x + o.view(-1, h * e) @ mix
        return x

    def read_context(self):
        rows = self.C * torch.arange(self.B + 1, dtype=torch.int32, device="cuda")
        # (a request's context is its own sequence here, under a prefix of no rows)
        self.layers(self.context.reshape(-1, self.context.shape[2]), rows, self.none, self.prefix, self.prefix_pages, None,
                    self.each, self.none, self.prefix_pages)

    def rows(self, x, n, first):
        """Hidden states of n rows of each candidate, [B K, n, d] to the same."""
        S = self.B * self.K
        ints = lambda v: torch.full((S,), v, dtype=torch.int32, device="cuda")  # noqa: E731
        return self.layers(x.reshape(S * n, -1), n * torch.arange(S + 1, dtype=torch.int32, device="cuda"), ints(first),
                           ints(first + n), self.pages, ints(self.C), self.groups, self.prefix, self.prefix_pages).view(S, n, -1)

    def logits(self, hidden, taken):
        """[B K, n, M] in bf16 of hidden [B K, n, d]; -inf where taken."""
        x = (hidden @ self.out.to(torch.bfloat16)).view(self.B, -1, hidden.shape[2])
        y = (x @ self.pool.transpose(1, 2)).view(*hidden.shape[:2], -1)
        return y.masked_fill_(taken, -torch.inf)

    def embed(self, tokens):
        """Pool rows [B K, n, d] of tokens [B K, n]."""
        B, d = self.B, self.pool.shape[2]
        at = tokens.reshape(B, -1, 1).expand(-1, -1, d).long()
        return self.pool.gather(1, at).view(*tokens.shape, d)

    def write(self):
        """(tokens [B K, L] int32, their log probabilities)."""
        S, M = self.B * self.K, self.pool.shape[1]
        x = self.begin.expand(S, 1, -1)
        taken = torch.zeros(S, 1, M, dtype=torch.bool, device="cuda")
        tokens, logp = [], []
        for j in range(self.L):
            p = torch.log_softmax(self.logits(self.rows(x, 1, j), taken)[:, 0].float(), -1)
            y = torch.multinomial(p.exp(), 1, generator=self.rng)
            tokens.append(y)
            logp.append(p.gather(1, y))
            taken.scatter_(2, y[:, None], True)
            x = self.embed(y)
        return torch.cat(tokens, 1).to(torch.int32), torch.cat(logp, 1)

    def read_candidates(self, tokens):
        """(hidden [B K, L, d], logits [B K, L, M]) of written candidates, in one pass."""
        S, L = tokens.shape
        x = torch.cat([self.begin.expand(S, 1, -1), self.embed(tokens[:, :-1])], 1)
        hidden = self.rows(x, L, 0)
        hot = torch.zeros(S, L, self.pool.shape[1], dtype=torch.int32, device="cuda").scatter_(2, tokens[..., None].long(), 1)
        return hidden, self.logits(hidden, hot.cumsum(1) - hot > 0)

    def learn(self, tokens, old_logp, advantages, rate):
        """One step of `out`; the loss."""
        hidden, logits = self.read_candidates(tokens)
        S, L, M = logits.shape
        r = policy_loss(logits.view(S * L, M), tokens.reshape(-1), advantages.repeat_interleave(L), old_logp=old_logp.reshape(-1),
                        grad_scale=float(S * L), status=self.status)  # (gradients per token, in bf16's range)
        g = r.grad.view(self.B, -1, M) @ self.pool
        d_out = hidden.view(S * L, -1).float().T @ g.view(S * L, -1).float() / (S * L)
        self.out -= rate * d_out / d_out.norm()
        return r


def run(requests=16, candidates=50, length=6, steps=30, rate=0.5, seed=0, tell=print):
    w = wl.make_workload("serving", B=requests, K=candidates, L=length)
    context, pool = (torch.from_numpy(x).to("cuda", torch.bfloat16) for x in (w.context, w.pool))
    evaluator = Evaluator(w.cfg, w.weights)
    generator = Generator(context, pool, candidates, length, seed=seed)
    generator.read_context()
    means = []
    for step in range(steps):
        tokens, logp = generator.write()
        scores, best = evaluator.evaluate(context, pool, tokens.view(requests, candidates, length))
        spread, mean = torch.std_mean(scores, 1, keepdim=True)
        loss = generator.learn(tokens, logp, ((scores - mean) / (spread + 1e-6)).view(-1), rate)
        check_status(generator.status)
        means.append(scores.mean().item())
        tell(f"step {step}: mean score {means[-1]:.4f}, best {scores.amax(1).mean().item():.4f}, loss {loss.loss.item():+.4f}")
    evaluator.close()
    return means


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, n in (("requests", 16), ("candidates", 50), ("length", 6), ("steps", 30)):
        p.add_argument("--" + name, type=int, default=n)
    p.add_argument("--rate", type=float, default=0.5)
    run(**vars(p.parse_args()))
