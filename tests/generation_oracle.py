"""The candidate generator's operators in float64 numpy, row by row from their definitions, with a bound
on what a kernel's own arithmetic may be off: fp32 sums and products, one rounding to the output's type."""
import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # unit roundoff
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}  # half a subnormal step


def f64(t):
    return t.detach().double().cpu().numpy()


def append(k, v, q, row_start, first, pages, rope, pairs, shift, kc, vc):
    """(kc, vc, q_out) after the call and the bound of kc's and q_out's error, as float64 arrays."""
    k, v, kc, vc = f64(k), f64(v), f64(kc), f64(vc)
    ek, q = np.zeros(kc.shape), None if q is None else f64(q)
    eq = None if q is None else np.zeros(q.shape)
    R = kc.shape[2]

    def turn(x, p):
        if rope is None:
            return x.copy(), np.zeros(x.shape)
        c, s = f64(rope)[p, :, 0], f64(rope)[p, :, 1]
        r = 2 * len(c)
        a, b = (slice(0, r // 2), slice(r // 2, r)) if pairs == "half" else (slice(0, r, 2), slice(1, r, 2))
        y, e = x.copy(), np.zeros(x.shape)
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
        e[:, a] = e[:, b] = 3 * 2.0 ** -24 * (np.abs(x[:, a]) + np.abs(x[:, b]))
        return y, e

    for i in range(len(first)):
        for j, t in enumerate(range(row_start[i], row_start[i + 1])):
            c = first[i] + j
            p = c + (shift[i] if shift is not None else 0)
            page, at = pages[i][c // R], c % R
            kc[page, :, at], ek[page, :, at] = turn(k[t], p)
            vc[page, :, at] = v[t]
            if q is not None:
                q[t], eq[t] = turn(q[t], p)
    return kc, vc, q, ek, eq


def attend(q, kc, vc, row_start, lens, pages, group_start, prefix, prefix_pages, scale):
    """(out, lse, bound of out's error without its own rounding, bound of lse's error)."""
    q, kc, vc = f64(q), f64(kc), f64(vc)
    T, hq, d = q.shape
    hr, R = hq // kc.shape[1], kc.shape[2]
    out, lse = np.zeros(q.shape), np.full((T, hq), -np.inf)
    eo, el = np.zeros(q.shape), np.zeros((T, hq))
    for g in range(len(prefix)):
        pre = [(prefix_pages[g][c // R], c % R) for c in range(prefix[g])]
        for s in range(group_start[g], group_start[g + 1]):
            n = row_start[s + 1] - row_start[s]
            for j in range(n):
                seen = max(0, min(lens[s], lens[s] - n + j + 1))
                at = pre + [(pages[s][c // R], c % R) for c in range(seen)]
                if not at:
                    continue
                pg, pl = np.array(at).T
                for h in range(hq):
                    kk, vv, x = kc[pg, h // hr, pl], vc[pg, h // hr, pl], q[row_start[s] + j, h]
                    z = scale * (kk @ x)
                    es = (d + 8) * 2.0 ** -22 * scale * (np.abs(kk) @ np.abs(x)).max() + 2.0 ** -21 * np.abs(z).max()
                    m = z.max()
                    e = np.exp(z - m)
                    lse[row_start[s] + j, h] = m + np.log(e.sum())
                    p = e / e.sum()
                    out[row_start[s] + j, h] = p @ vv
                    # scores off by es, exponent and sums, rounded weights (u, added by the caller)
                    eo[row_start[s] + j, h] = p @ np.abs(vv)
                    el[row_start[s] + j, h] = es + (len(at) + 64) * 2.0 ** -22 + 2.0 ** -22 * abs(m)
    return out, lse, eo, el


def policy(logits, y, adv, w, old, ref, clip, beta, temperature, scale):
    """(loss, terms, logp, lse, coef, grad) and a bound of logp's error per token."""
    x = f64(logits) / temperature
    T, V = x.shape
    m = x.max(1, keepdims=True)
    lse = (m + np.log(np.exp(x - m).sum(1, keepdims=True)))[:, 0]
    logp = x[np.arange(T), y] - lse
    r = np.ones(T) if old is None else np.exp(logp - old)
    c = np.clip(r, 1 - clip[0], 1 + clip[1])
    use = r * adv <= c * adv
    terms, coef = np.where(use, -r * adv, -c * adv), np.where(use, -r * adv, 0.0)
    if ref is not None:
        d = ref - logp
        terms, coef = terms + beta * (np.exp(d) - d - 1), coef + beta * (1 - np.exp(d))
    terms, coef = w * terms, w * coef
    hot = np.zeros((T, V))
    hot[np.arange(T), y] = 1
    p = np.exp(x - lse[:, None])
    grad = scale / temperature * coef[:, None] * (hot - p)
    fin = np.where(np.isfinite(x), x, m)
    span = (m - fin.min(1, keepdims=True))[:, 0]
    eps = 2.0 ** -22 * (1 + span + np.abs(logp) + np.abs(lse)) + (V / 256 + 32) * 2.0 ** -23
    return terms.sum(), terms, logp, lse, coef, grad, eps
