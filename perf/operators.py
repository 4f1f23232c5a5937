"""What is measured of the candidate generator's operators.

The generator writes the candidate sequences that the evaluator scores, and
learns from the scores.  Three operators, each called as a user's program
calls it:

  append  `PagedKV.append`: new keys and values of ragged sequences go into a
          paged cache, rotated by position on the way, queries too;
  attend  `PagedKV.attend`: the sequences of a group share a prefix (the
          request's context) and attend to it and to their own rows;
  loss    `policy_loss`: clipped policy loss with a KL term on the candidates'
          tokens, its statistics and its gradient to the logits.

A case holds the ranges of the sequences' lengths; the lengths themselves
follow from the case, the contents and the pages' places in memory from the
seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
#: the policy loss's clip range below and above one, the KL term's weight, and the loss scale of 16-bit training
CLIP, BETA, SCALE = (0.2, 0.28), 0.04, 1024.0
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------- cases


def _append(name=None, **kw):
    c = dict(op="append", S=1, lo=1, hi=1, held_lo=0, held_hi=0, hq=8, hkv=8, d=64, page=16, rot=64, pairs="half",
             dtype="bf16")
    c.update(kw)
    return c if name is None else dict(c, name=name)


def _attend(name=None, **kw):
    c = dict(op="attend", G=1, K=1, prefix_lo=0, prefix_hi=0, own_lo=1, own_hi=1, rows_lo=1, rows_hi=1, hq=8, hkv=8,
             d=64, page=16, dtype="bf16", lse=False)
    c.update(kw)
    return c if name is None else dict(c, name=name)


def _loss(name=None, **kw):
    c = dict(op="loss", T=1, V=32768, dtype="bf16", grad=True, ref=True, masked=0.0, temperature=1.0)
    c.update(kw)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one token of each of four candidates enters the cache: only latency counts
        _append("append_few", S=4, held_lo=3, held_hi=40),
        # one token of each candidate of 64 requests, partly rotated rows, grouped heads
        _append("append_step", S=1024, held_lo=0, held_hi=63, hq=32, hkv=8, d=128, page=64, rot=64, pairs="interleaved",
                dtype="f16"),
        # the contexts of 37 requests, short to long, as they arrive
        _append("append_prompts", S=37, lo=1, hi=8000, hq=32, hkv=8, d=128, rot=128),
        # one request, four candidates, an early token: only latency counts
        _attend("attend_few", K=4, prefix_lo=300, prefix_hi=300, own_lo=5, own_hi=20, lse=True),
        # the serving model's sizes: 256 requests, 50 candidates of up to 6 tokens
        _attend("attend_serving", G=256, K=50, prefix_lo=256, prefix_hi=256, own_lo=1, own_hi=6, hq=4, hkv=4, d=32),
        # summaries being written: 32 articles, 16 summaries of each, any of their tokens
        _attend("attend_summaries", G=32, K=16, prefix_lo=600, prefix_hi=1024, own_lo=1, own_hi=64, page=64,
                dtype="f16"),
        # long contexts with grouped heads, a late token
        _attend("attend_long", G=4, K=16, prefix_lo=20000, prefix_hi=32768, own_lo=1, own_hi=500, hq=32, hkv=8, d=128,
                page=64),
        # given summaries read in one pass (to rescore them): many rows per sequence
        _attend("read_summaries", G=32, K=16, prefix_lo=600, prefix_hi=1024, own_lo=33, own_hi=64, rows_lo=33,
                rows_hi=64, page=64, dtype="f16"),
        # long continuations of a long context read in one pass: arithmetic alone counts
        _attend("read_long", G=2, K=8, prefix_lo=8000, prefix_hi=8192, own_lo=200, own_hi=256, rows_lo=200,
                rows_hi=256, hq=32, hkv=8, d=128, page=128),
        # a token of sixteen candidates, the text vocabulary
        _loss("loss_few", T=16),
        # a training step's tokens in fp32, a quarter of them padding
        _loss("loss_step", T=2048, dtype="f32", masked=0.25),
        # a large vocabulary of odd size (rows start anywhere), a temperature
        _loss("loss_wide", T=4099, V=100003, temperature=0.7),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "loss"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "loss":
        V = _log(rng, 1000, 131072)
        T = _log(rng, 1, max(1, min(16384, 4099 * 100003 // V)))
        return _loss(T=T, V=V, dtype=rng.choice(["bf16", "f16", "f32"]) if T * V < 2 ** 27 else dtype,
                     grad=rng.random() < 0.75, ref=rng.random() < 0.5, masked=rng.choice([0.0, 0.3]),
                     temperature=rng.choice([1.0, 0.6, 1.3]))
    d = rng.choice([32, 64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 1, 2, 3, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        S = _log(rng, 1, 4096)
        hi = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 148000 // S))
        hi = min(hi, max(1, 148000 * 48 * 128 // (S * (hq + 2 * hkv) * d)))
        held = _log(rng, 1, 300)
        return _append(S=S, lo=min(hi, rng.choice([0, 1])) if hi > 1 else 1, hi=hi, held_lo=0, held_hi=held, hq=hq,
                       hkv=hkv, d=d, page=page, rot=rng.choice([d, d, d // 2]), pairs=rng.choice(["half", "interleaved"]),
                       dtype=dtype)
    while True:
        G, K = _log(rng, 1, 256), _log(rng, 1, 64)
        P = _log(rng, 1, 32768)
        rows = 1 if rng.random() < 0.6 else _log(rng, 2, 256)
        hi = rows + rng.choice([0, 0, _log(rng, 1, 500)])
        lo = max(rows, 1 + hi // 3) if rng.random() < 0.7 else rows
        scores = G * K * rows * hq * (P + hi)
        held = (G * P + G * K * hi) * hkv * d
        if scores <= 1.1e9 and held <= 4e8 and 4 * d * scores <= 5e11:
            return _attend(G=G, K=K, prefix_lo=rng.choice([0, P // 2, P]), prefix_hi=P, own_lo=lo, own_hi=hi,
                           rows_lo=rows if rng.random() < 0.5 else max(1, rows // 2), rows_hi=rows, hq=hq, hkv=hkv,
                           d=d, page=page, dtype=dtype, lse=rng.random() < 0.5)


def _lengths(salt, n, lo, hi):
    """n lengths from lo to hi, the longest among them, the same ones each time."""
    r = np.random.RandomState(1000 * salt + n % 997 + lo)
    v = r.randint(lo, hi + 1, n)
    v[n // 2] = hi
    return v.astype(np.int64)


def _plan(case):
    """The ragged sizes of a case, as host arrays."""
    if case["op"] == "append":
        rows = _lengths(1, case["S"], case["lo"], case["hi"])
        return dict(rows=rows, first=_lengths(2, case["S"], case["held_lo"], case["held_hi"]),
                    start=np.concatenate([[0], np.cumsum(rows)]))
    S = case["G"] * case["K"]
    own_len = _lengths(3, S, case["own_lo"], case["own_hi"])
    rows = np.minimum(_lengths(4, S, case["rows_lo"], case["rows_hi"]), np.maximum(own_len, 1))
    return dict(rows=rows, own=own_len, start=np.concatenate([[0], np.cumsum(rows)]),
                prefix=_lengths(5, case["G"], case["prefix_lo"], case["prefix_hi"]))


def work(case):
    if case["op"] == "loss":
        kept = case["T"] - _masked(case).sum()
        n = float(kept) * case["V"]
        # logits in, gradient out (zeros where a token is masked); an exponent, a sum, a maximum, the gradient's product
        grad = float(case["T"]) * case["V"] if case["grad"] else 0.0
        return {"bytes": (n + grad) * SIZES[case["dtype"]] + 24.0 * case["T"], "flops": (6.0 if case["grad"] else 4.0) * n}
    p, e, d = _plan(case), SIZES[case["dtype"]], case["d"]
    T = float(p["start"][-1])
    if case["op"] == "append":
        top = int((p["first"] + p["rows"]).max())
        return {"bytes": 2.0 * T * (case["hq"] + 2 * case["hkv"]) * d * e + min(T, top) * case["rot"] * 4.0,
                "flops": 3.0 * T * (case["hq"] + case["hkv"]) * case["rot"]}
    n, ln = p["rows"].astype(float), p["own"].astype(float)
    seen = n * np.repeat(p["prefix"], case["K"]) + n * ln - n * (n - 1) / 2
    kv = 2.0 * float(p["prefix"].sum() + ln.sum()) * case["hkv"] * d * e
    return {"bytes": 2.0 * T * case["hq"] * d * e + kv + (4.0 * T * case["hq"] if case["lse"] else 0.0),
            "flops": 4.0 * d * case["hq"] * float(seen.sum())}


# ---------------------------------------------------------------------------- inputs


def _masked(case):
    r = np.random.RandomState(case["T"] % 9973)
    m = r.random_sample(case["T"]) < case["masked"]
    m[0] = False
    return m


def _ints(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def _rope(n, rot):
    """cos and sin of position p and pair i at [p, i]: angle p 10000^(-2 i / rot)."""
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)[None, :]
    return torch.tensor(np.stack([np.cos(a), np.sin(a)], -1), dtype=torch.float32, device=DEV).contiguous()


def _pages(rng, lens, page, taken):
    """A page table whose used entries come from `taken`, a shuffled list of pages; -1 elsewhere."""
    n = -(-lens // page)
    table = np.full((len(lens), max(1, int(n.max()))), -1, np.int64)
    at = np.concatenate([[0], np.cumsum(n)])
    table[np.arange(table.shape[1])[None, :] < n[:, None]] = taken[: at[-1]]
    return table, taken[at[-1]:]


def prepare(case, seed):
    rng = np.random.RandomState(seed % (2 ** 31))
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)

    dt = DTYPES[case["dtype"]]
    if case["op"] == "loss":
        T, V = case["T"], case["V"]
        logits = torch.empty(T, V, dtype=dt, device=DEV)
        step = max(1, 2 ** 27 // V)
        for i in range(0, T, step):  # a model's logits: a few tokens stand out
            x = torch.randn(min(step, T - i), V, generator=g, device=DEV)
            logits[i:i + step] = x.mul_(2.0)
        y = torch.randint(0, V, (T,), generator=g, device=DEV)
        boost = torch.rand(T, generator=g, device=DEV) * 14
        rows = torch.arange(T, device=DEV)
        logits[rows, y] = (logits[rows, y].float() + boost).to(dt)
        lp = torch.empty(T, device=DEV)
        for i in range(0, T, step):
            x = logits[i:i + step].float() / case["temperature"]
            lp[i:i + step] = x.gather(1, y[i:i + step, None])[:, 0] - torch.logsumexp(x, 1)
        w = torch.tensor(np.where(_masked(case), 0.0, 1.0 / T), dtype=torch.float32, device=DEV)
        # how far the policy has moved; no ratio within a rounding of a clip bound, where the slope jumps
        moved = normal(T, std=0.15)
        for bound in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
            moved = torch.where((moved - bound).abs() < 1e-3, moved + 4e-3, moved)
        return dict(case=case, logits=logits, tokens=y.int(), old=lp - moved,
                    ref=lp + normal(T, std=0.3) if case["ref"] else None, adv=normal(T) + 0.5, w=w)
    p = _plan(case)
    T = int(p["start"][-1])
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    if case["op"] == "append":
        lens = p["first"] + p["rows"]
        n_pages = int((-(-lens // page)).sum()) + 3
        table, _ = _pages(rng, lens, page, rng.permutation(n_pages))
        kv = [normal(n_pages, hkv, page, d, dtype=dt) for _ in range(2)]
        # q, k and v are parts of one projection's rows, as a model has them
        rows = normal(T, hq + 2 * hkv, d, dtype=dt)
        st = dict(case=case, kc=kv[0], vc=kv[1], q=rows[:, :hq], k=rows[:, hq:hq + hkv], v=rows[:, hq + hkv:],
                  row_start=_ints(p["start"]), first=_ints(p["first"]), pages=_ints(table),
                  rope=_rope(int(lens.max()), case["rot"]))
    else:
        n_pre, n_own = -(-p["prefix"] // page), -(-p["own"] // page)
        n_pages = int(n_pre.sum() + n_own.sum()) + 3
        free = rng.permutation(n_pages)
        pre, free = _pages(rng, p["prefix"], page, free)
        table, free = _pages(rng, p["own"], page, free)
        kv = [normal(n_pages, hkv, page, d, dtype=dt) for _ in range(2)]
        # rows that nothing was written to yet hold whatever was there: some of them no number at all
        stale = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
        for lens, tab in ((p["prefix"], pre), (p["own"], table)):
            last = lens % page
            at = np.maximum(lens - 1, 0) // page
            rows = np.arange(page)[None, :] >= np.where(last == 0, page, last)[:, None]
            use = lens > 0
            stale[torch.tensor(tab[np.arange(len(lens)), at][use], device=DEV)] = torch.tensor(rows[use], device=DEV)
        for x in kv:
            x.masked_fill_(stale[:, None, :, None], float("nan"))
        q = normal(T, hq, d, dtype=dt)
        # some directions matter more than others: softmax weights from even to peaked
        q *= (torch.rand(T, hq, 1, generator=g, device=DEV) * 2.0).to(dt)
        st = dict(case=case, kc=kv[0], vc=kv[1], q=q, row_start=_ints(p["start"]), lens=_ints(p["own"]),
                  pages=_ints(table), group_start=_ints(np.arange(case["G"] + 1) * case["K"]),
                  prefix=_ints(p["prefix"]), prefix_pages=_ints(pre), most=(int(p["prefix"].max()), int(p["own"].max()),
                                                                           int(p["rows"].max())))
    return st


# ---------------------------------------------------------------------------- one pass


def run(st):
    op = st["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "loss": _own_loss}[op](st)
    return {"append": _plain_append, "attend": _plain_attend, "loss": _plain_loss}[op](st)


def _cache(st):
    if "cache" not in st:  # the handle that a program keeps
        from paper_2603_02565_gb300 import PagedKV
        st["cache"] = PagedKV(st["kc"], st["vc"])
    return st["cache"]


def _own_append(st):
    q = _cache(st).append(st["k"], st["v"], st["row_start"], st["first"], st["pages"], q=st["q"], rope=st["rope"],
                          pairs=st["case"]["pairs"])
    return st["kc"], st["vc"], q


def _own_attend(st):
    return _cache(st).attend(st["q"], st["row_start"], st["lens"], st["pages"], st["group_start"], st["prefix"],
                             st["prefix_pages"], with_lse=st["case"]["lse"])


def _own_loss(st):
    from paper_2603_02565_gb300 import policy_loss
    r = policy_loss(st["logits"], st["tokens"], st["adv"], st["w"], old_logp=st["old"], ref_logp=st["ref"], clip=CLIP,
                    beta=BETA, temperature=st["case"]["temperature"], with_grad=st["case"]["grad"], grad_scale=SCALE)
    return (r.loss, r.logp, r.grad) if st["case"]["grad"] else (r.loss, r.logp)


def _rotate(x, cs, pairs):
    r = 2 * cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    x = x.float()
    if pairs == "half":
        a, b = x[..., : r // 2], x[..., r // 2: r]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., r:]], -1)


def _plain_append(st):
    case, dt = st["case"], st["kc"].dtype
    t = torch.arange(st["k"].shape[0], device=DEV, dtype=torch.int32)
    s = torch.searchsorted(st["row_start"], t, right=True) - 1
    at = st["first"][s] + t - st["row_start"][s]
    page, place = st["pages"][s, at // case["page"]].long(), (at % case["page"]).long()
    cs = st["rope"][at]
    st["kc"][page, :, place] = _rotate(st["k"], cs, case["pairs"]).to(dt)
    st["vc"][page, :, place] = st["v"]
    return st["kc"], st["vc"], _rotate(st["q"], cs, case["pairs"]).to(dt)


def _plain_keys(cache, table, lens, most):
    """Rows 0 .. most - 1 of each paged sequence in 32 bits, [n, heads, most, d], zeros past its length, and which are valid."""
    x = cache[table.clamp(min=0).long()].transpose(1, 2).flatten(2, 3)[:, :, :most].float()
    valid = torch.arange(most, device=DEV)[None, :] < lens[:, None]
    return torch.where(valid[:, None, :, None], x, torch.zeros((), device=DEV)), valid


def _plain_attend(st):
    case, q = st["case"], st["q"]
    G, K, hkv, d = case["G"], case["K"], case["hkv"], case["d"]
    most_prefix, most_own, nq = (max(1, n) for n in st["most"])
    T, hq = q.shape[:2]
    hr = hq // hkv
    row_start, lens = st["row_start"].long(), st["lens"].long()
    n = row_start[1:] - row_start[:-1]
    j = torch.arange(nq, device=DEV)
    qs = q.float()[(row_start[:-1, None] + j).clamp(max=T - 1)] * (1.0 / math.sqrt(d))
    qs = qs.view(G * K, nq, hkv, hr, d).permute(0, 2, 1, 3, 4).reshape(G * K, hkv, nq * hr, d)
    qg = qs.view(G, K, hkv, nq * hr, d).transpose(1, 2).reshape(G, hkv, K * nq * hr, d)
    minus = float("-inf")
    kp, valid = _plain_keys(st["kc"], st["prefix_pages"], st["prefix"], most_prefix)
    s1 = (qg @ kp.transpose(2, 3)).masked_fill_(~valid[:, None, None, :], minus)
    del kp
    ks, valid = _plain_keys(st["kc"], st["pages"], st["lens"], most_own)
    seen = valid[:, None, :] & (torch.arange(most_own, device=DEV) <= (lens - n)[:, None, None] + j[None, :, None])
    s2 = (qs @ ks.transpose(2, 3)).view(G * K, hkv, nq, hr, most_own)
    s2 = s2.masked_fill_(~seen[:, None, :, None, :], minus)
    s2 = s2.view(G, K, hkv, nq * hr, most_own).transpose(1, 2).reshape(G, hkv, K * nq * hr, most_own)
    m = torch.maximum(s1.amax(-1, keepdim=True), s2.amax(-1, keepdim=True))
    m0 = m.masked_fill(m == minus, 0.0)
    s1.sub_(m0).exp_()
    s2.sub_(m0).exp_()
    total = s1.sum(-1, keepdim=True) + s2.sum(-1, keepdim=True)
    o = s1 @ _plain_keys(st["vc"], st["prefix_pages"], st["prefix"], most_prefix)[0]
    vs = _plain_keys(st["vc"], st["pages"], st["lens"], most_own)[0]
    s2 = s2.view(G, hkv, K, nq * hr, most_own).transpose(1, 2).reshape(G * K, hkv, nq * hr, most_own)
    o = o.view(G, hkv, K, nq * hr, d).transpose(1, 2) + (s2 @ vs).view(G, K, hkv, nq * hr, d)
    total = total.view(G, hkv, K, nq * hr, 1).transpose(1, 2)
    o = torch.where(total > 0, o / total, torch.zeros((), device=DEV))
    t = torch.arange(T, device=DEV)
    s = torch.searchsorted(row_start, t, right=True) - 1
    at = t - row_start[s]
    o = o.reshape(G * K, hkv, nq, hr, d)[s, :, at].reshape(T, hq, d).to(q.dtype)
    if not case["lse"]:
        return o
    lse = m0.reshape(G, hkv, K, nq * hr, 1).transpose(1, 2) + total.log()
    return o, lse.reshape(G * K, hkv, nq, hr)[s, :, at].reshape(T, hq)


def _plain_loss(st):
    case, w, adv = st["case"], st["w"], st["adv"]
    temperature, y = case["temperature"], st["tokens"].long()[:, None]
    kept = w != 0
    x = st["logits"].float() / temperature
    m = x.amax(1, keepdim=True)
    lse = m + (x - m).exp_().sum(1, keepdim=True).log()
    logp = (x.gather(1, y) - lse)[:, 0]
    ratio = torch.exp(logp - st["old"])
    clipped = ratio.clamp(1 - CLIP[0], 1 + CLIP[1])
    loss, coef = -torch.minimum(ratio * adv, clipped * adv), -adv * ratio * (ratio * adv <= clipped * adv)
    if st["ref"] is not None:
        e = torch.exp(st["ref"] - logp)
        loss, coef = loss + BETA * (e - (st["ref"] - logp) - 1), coef + BETA * (1 - e)
    zero = torch.zeros((), device=DEV)
    loss = torch.where(kept, w * loss, zero).sum()
    logp = torch.where(kept, logp, zero)
    if not case["grad"]:
        return loss, logp
    coef = (torch.where(kept, w * coef, zero) * (SCALE / temperature))[:, None]
    grad = x.sub_(lse).exp_().mul_(-coef).scatter_add_(1, y, coef)
    return loss, logp, torch.where(kept[:, None], grad, zero).to(st["logits"].dtype)


# ---------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "loss": _exact_loss}[case["op"]](st, _plan_of(case))


def _plan_of(case):
    return None if case["op"] == "loss" else _plan(case)


def _exact_turned(x, cs, pairs):
    """Rows [n, heads, d] in 64 bits: pairs as complex numbers, each times its position's unit number."""
    r = 2 * cs.shape[1]
    unit = torch.view_as_complex(cs.double())[:, None, :]
    x = x.double()
    a = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if pairs == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
    a = torch.view_as_real(torch.view_as_complex(a.contiguous()) * unit)
    a = a.transpose(-1, -2).flatten(-2) if pairs == "half" else a.flatten(-2)
    return torch.cat([a, x[..., r:]], -1)


def _exact_append(st, p):
    case = st["case"]
    kc, vc, q = st["kc"].double(), st["vc"].double(), torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    table, page = st["pages"].tolist(), case["page"]
    at = np.concatenate([np.arange(f, f + n) for f, n in zip(p["first"], p["rows"])])
    seq = np.repeat(np.arange(case["S"]), p["rows"])
    cs = st["rope"][torch.tensor(at, device=DEV)]
    where = torch.tensor([table[s][c // page] * page + c % page for s, c in zip(seq.tolist(), at.tolist())], device=DEV)
    for h in range(case["hkv"]):
        rows = kc[:, h].clone().view(-1, case["d"])
        rows[where] = _exact_turned(st["k"][:, h:h + 1], cs, case["pairs"])[:, 0]
        kc[:, h] = rows.view(-1, page, case["d"])
        rows = vc[:, h].clone().view(-1, case["d"])
        rows[where] = st["v"][:, h].double()
        vc[:, h] = rows.view(-1, page, case["d"])
    for h in range(case["hq"]):
        q[:, h] = _exact_turned(st["q"][:, h:h + 1], cs, case["pairs"])[:, 0]
    return kc, vc, q


def _exact_attend(st, p):
    """Group by group: the keys of the prefix and of every sequence of the group in one row, others' keys masked."""
    case = st["case"]
    hkv, d, page, K = case["hkv"], case["d"], case["page"], case["K"]
    T, hq = st["q"].shape[:2]
    hr = hq // hkv
    pre, own_pages = st["prefix_pages"].tolist(), st["pages"].tolist()
    o = torch.zeros(T, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((T, hq), float("-inf"), dtype=torch.float64, device=DEV)
    for g in range(case["G"]):
        seqs = range(g * K, (g + 1) * K)
        rows = [pre[g][c // page] * page + c % page for c in range(int(p["prefix"][g]))]
        owner, place = [-1] * len(rows), list(range(len(rows)))
        for s in seqs:
            n = int(p["own"][s])
            rows += [own_pages[s][c // page] * page + c % page for c in range(n)]
            owner += [s] * n
            place += list(range(n))
        if not rows:
            continue
        rows, owner, place = (torch.tensor(x, device=DEV) for x in (rows, owner, place))
        a, b = int(p["start"][g * K]), int(p["start"][(g + 1) * K])
        mine = torch.tensor(np.repeat(np.arange(g * K, (g + 1) * K), p["rows"][g * K:(g + 1) * K]), device=DEV)
        last = torch.tensor(np.concatenate([p["own"][s] - p["rows"][s] + np.arange(p["rows"][s]) for s in seqs]), device=DEV)
        seen = (owner == -1)[None, :] | ((owner[None, :] == mine[:, None]) & (place[None, :] <= last[:, None]))
        seen = seen[:, None, :].expand(-1, hr, -1).reshape((b - a) * hr, -1)
        for h in range(hkv):
            k = st["kc"][rows // page, h, rows % page].double()
            v = st["vc"][rows // page, h, rows % page].double()
            x = st["q"][a:b, h * hr:(h + 1) * hr].double().reshape(-1, d) @ k.T / math.sqrt(d)
            x = x.masked_fill_(~seen, float("-inf"))
            z = torch.logsumexp(x, 1)
            w = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[:, None])
            o[a:b, h * hr:(h + 1) * hr] = (w @ v).view(b - a, hr, d)
            lse[a:b, h * hr:(h + 1) * hr] = z.view(b - a, hr)
    return (o, lse) if case["lse"] else o


def _exact_loss(st, p):
    case = st["case"]
    T, t = case["T"], case["temperature"]
    logp = torch.zeros(T, dtype=torch.float64, device=DEV)
    grad = torch.zeros(T, case["V"], dtype=torch.float64, device=DEV) if case["grad"] else None
    w, adv, old = st["w"].double(), st["adv"].double(), st["old"].double()
    loss = torch.zeros((), dtype=torch.float64, device=DEV)
    step = max(1, 2 ** 26 // case["V"])
    for i in range(0, T, step):
        b = slice(i, min(T, i + step))
        z = torch.log_softmax(st["logits"][b].double() / t, 1)
        y = st["tokens"][b].long()
        lp = z[torch.arange(len(y), device=DEV), y]
        r, A = torch.exp(lp - old[b]), adv[b]
        over = torch.where(A >= 0, r > 1 + CLIP[1], r < 1 - CLIP[0])  # the clipped value is the smaller one
        value = -A * torch.where(over, torch.where(A >= 0, 1.0 + CLIP[1], 1.0 - CLIP[0]), r)
        slope = -A * torch.where(over, 0.0, r)
        if st["ref"] is not None:
            gap = st["ref"][b].double() - lp
            value = value + BETA * (torch.expm1(gap) - gap)
            slope = slope - BETA * torch.expm1(gap)
        kept = w[b] != 0
        loss += (w[b] * value)[kept].sum()
        logp[b] = torch.where(kept, lp, 0.0)
        if grad is not None:
            hot = torch.nn.functional.one_hot(y, case["V"]).double()
            c = torch.where(kept, w[b] * slope, 0.0) * (SCALE / t)
            grad[b] = c[:, None] * (hot - z.exp())
    return (loss, logp, grad) if case["grad"] else (loss, logp)
