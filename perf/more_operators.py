"""Performance cases of the operators for groups of rollouts: decoding behind a shared prompt, and the policy loss's terms.

  shared  one query row per sequence attends over its history in the paged 8-bit cache; the sequences of a group have
          their first positions in common, in the same pages (`attention_shared_kv8`)
  lin     log-probability of a given token per row of hidden states, under the softmax of their products with the
          vocabulary's weights, and the entropy: the logits are never stored (`linear_logprobs`)
  lingrad the gradient of both with respect to the hidden states and the weights (`linear_logprobs_backward`)

The cache: pages of 128 positions, codes [pages][2 (K, V)][KV heads][128][head dim] in e4m3 or int8, one fp32 scale (a power of two)
per 32 positions, KV head and K or V: [pages][2][KV heads][4].  A sequence's pages stand in its row of a table.  A group's shared
positions are those before its prefix length, read through the table row of the group's first sequence.  With `own` false the same
operators are computed by elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

PAGE, BLOCK = 128, 32          # positions of a page, of a scale
TOP = {"e4m3": 448.0, "int8": 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # the last prompt of a round: its 8 rollouts at their median length behind a prompt of some 400 tokens: latency
        {"name": "shared 1 x 8", "kind": "shared", "groups": 1, "k": 8, "prefix": 384, "past": 758, "heads": 12, "kv": 2, "hd": 128,
         "code": "e4m3", "type": "bf16"},
        # a round's probes: two rollouts to a prompt, mid-way
        {"name": "shared 13 x 2", "kind": "shared", "groups": 13, "k": 2, "prefix": 384, "past": 758, "heads": 12, "kv": 2, "hd": 128,
         "code": "int8", "type": "fp16"},
        # a full batch of 64 prompts of about a thousand tokens with 8 rollouts each
        {"name": "shared 64 x 8", "kind": "shared", "groups": 64, "k": 8, "prefix": 1024, "past": 512, "heads": 32, "kv": 8, "hd": 128,
         "code": "e4m3", "type": "bf16"},
        # wide sampling behind long documents: 64 answers each, just begun
        {"name": "shared 8 x 64", "kind": "shared", "groups": 8, "k": 64, "prefix": 32768, "past": 128, "heads": 32, "kv": 8, "hd": 128,
         "code": "e4m3", "type": "bf16"},
        # the smallest model's last hidden states: latency
        {"name": "lin 32 x 128 x 512", "kind": "lin", "rows": 32, "dim": 128, "vocab": 512, "type": "bf16", "scale": 1.0},
        # one token, as a server scores it
        {"name": "lin 1 x 2048 x 151936", "kind": "lin", "rows": 1, "dim": 2048, "vocab": 151936, "type": "fp16", "scale": 1.0},
        # a decode step's rows: bound by reading the weights
        {"name": "lin 26 x 1536 x 151936", "kind": "lin", "rows": 26, "dim": 1536, "vocab": 151936, "type": "bf16", "scale": 1.25},
        # a batch of rollouts scored for the policy loss, a tenth of the rows padding
        {"name": "lin 4096 x 1536 x 151936", "kind": "lin", "rows": 4096, "dim": 1536, "vocab": 151936, "type": "bf16", "scale": 1.0},
        # the smallest model's loss gradient: latency
        {"name": "lingrad 32 x 128 x 512", "kind": "lingrad", "rows": 32, "dim": 128, "vocab": 512, "type": "bf16", "scale": 1.0,
         "entropy": True},
        # a small policy's: odd vocabulary and row count
        {"name": "lingrad 301 x 2048 x 32001", "kind": "lingrad", "rows": 301, "dim": 2048, "vocab": 32001, "type": "fp16", "scale": 1.0,
         "entropy": True},
        # the policy loss's gradient of a batch at the 1.5B shape
        {"name": "lingrad 4096 x 1536 x 151936", "kind": "lingrad", "rows": 4096, "dim": 1536, "vocab": 151936, "type": "bf16",
         "scale": 1.0, "entropy": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "lin", "lingrad"])
    if kind == "shared":
        c = {"kind": kind, "k": _log_int(rng, 1, 128), "kv": rng.choice([1, 2, 2, 4, 8]), "hd": rng.choice([32, 64, 128, 128]),
             "code": rng.choice(["e4m3", "int8"]), "type": rng.choice(["bf16", "fp16"])}
        c["groups"] = _log_int(rng, 1, min(128, max(1, 1024 // c["k"])))
        c["heads"] = c["kv"] * rng.choice([1, 2, 3, 4, 6, 8])
        width, rows = c["kv"] * c["hd"], c["groups"] * c["k"]
        # at most the shared positions, own positions and products of the largest listed cases
        most = min(8 * 32768 * 1024 // (c["groups"] * width), 512 * 32 * 128 * 32768 // (rows * c["heads"] * c["hd"]))
        c["prefix"] = _log_int(rng, 1, min(100000, max(1, most)))
        c["past"] = _log_int(rng, 1, min(16384, max(1, 512 * 512 * 1024 // (rows * width))))
        return c
    c = {"kind": kind, "rows": _log_int(rng, 1, 8192), "dim": 8 * _log_int(rng, 8, 512), "type": rng.choice(["bf16", "bf16", "fp16"]),
         "vocab": rng.choice([151936, 512, _log_int(rng, 300, 152000), 32000 + rng.randrange(999)]), "scale": rng.choice([1.0, 1.0, 1.25])}
    cells = min(4096 * 151936, 4096 * 1536 * 151936 // c["dim"])
    c["rows"] = min(c["rows"], max(1, cells // c["vocab"]))
    if kind == "lingrad":
        c["entropy"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(n, mean):
    """Ragged lengths of a given mean, lognormal as rollouts' are; the case's own, so that every seed has the same sizes."""
    x = np.exp(0.5 * np.random.default_rng([n, mean]).standard_normal(n))
    return np.maximum(np.rint(x * (mean * n / x.sum())), 1).astype(np.int64)


def _sizes(case):
    """Sequences of each group: k, fewer in a quarter of the groups, whose others have ended."""
    g = np.random.default_rng([case["groups"], case["k"]])
    few = g.integers(1, case["k"] + 1, case["groups"])
    return np.where(g.random(case["groups"]) < 0.25, few, case["k"]).astype(np.int64)


def _pool(g, case, pages):
    """A cache of random codes: K and V ~ N(0, 1) in units of their block's spread, scales that differ by block."""
    kv, hd, code = case["kv"], case["hd"], case["code"]
    codes = torch.empty((pages, 2, kv, PAGE, hd), dtype=CODES[code], device="cuda")
    std = TOP[code] / 5.0
    step = max(1, (1 << 27) // (2 * kv * PAGE * hd))
    for a in range(0, pages, step):
        x = torch.randn((min(step, pages - a), 2, kv, PAGE, hd), generator=g, device="cuda").mul_(std)
        x.clamp_(-TOP[code], TOP[code])
        codes[a:a + step].copy_(x.round_().to(torch.int8) if code == "int8" else x.to(torch.float8_e4m3fn))
    e = torch.randint(-1, 2, (pages, 2, kv, PAGE // BLOCK), generator=g, device="cuda") - round(math.log2(std))
    return codes, torch.exp2(e.float())


def _cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _prepare_shared(case, seed):
    g, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    sizes, prefix = _sizes(case), _lengths(case["groups"], case["prefix"])
    start = np.concatenate([[0], np.cumsum(sizes)])
    n = int(start[-1])
    ctx = np.repeat(prefix, sizes) + _lengths(n, case["past"])
    if n >= 16:
        ctx[n // 3] = 0  # a slot of the batch without a sequence
    # whole pages of the prefix are a group's, the others (the one in which the prefix ends among them) a sequence's own
    per = np.maximum(-(-ctx // PAGE), np.where(np.isin(np.arange(n), start[:-1]), np.repeat(-(-prefix // PAGE), sizes), 0))
    whole = prefix // PAGE
    table = np.full((n, max(1, int(per.max()))), -1, np.int32)
    pages = int(whole.sum() + np.maximum(per - np.repeat(whole, sizes), 0).sum())
    ids, at = rng.permutation(pages + 3).astype(np.int32), 0
    for j in range(case["groups"]):
        w = int(whole[j])
        common = ids[at:at + w]
        at += w
        for i in range(int(start[j]), int(start[j + 1])):
            m = max(int(per[i]) - w, 0)
            table[i, :w] = common
            table[i, w:w + m] = ids[at:at + m]
            at += m
    st = {"case": case, "lens": (start, prefix, ctx)}
    st["codes"], st["scales"] = _pool(g, case, pages + 3)
    st["q"] = torch.randn((n, case["heads"], case["hd"]), generator=g, device="cuda", dtype=TYPES[case["type"]])
    st["table"], st["ctx"], st["start"], st["prefix"] = _cuda(table), _cuda(ctx), _cuda(start), _cuda(prefix)
    if own:  # scratch that a serving loop keeps from step to step
        import paper_2607_26253_gb300 as sara
        st["workspace"] = sara.attention_shared_kv8_workspace(n, case["groups"], case["heads"], case["kv"], case["hd"])
    return st


def prepare(case, seed):
    if case["kind"] == "shared":
        return _prepare_shared(case, seed)
    # hidden states behind a last norm, each leaning towards its token's weights so that the token's logit stands out in
    # most rows, as a trained policy's does; a tenth of the rows is padding (token -1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    r, d, v = case["rows"], case["dim"], case["vocab"]
    st = {"case": case}
    w = torch.randn((v, d), generator=g, device="cuda").mul_(0.02)
    h = torch.randn((r, d), generator=g, device="cuda")
    tok = torch.randint(0, v, (r,), generator=g, device="cuda")
    peak = 4.0 * torch.randn((r,), generator=g, device="cuda") + 9.0
    h += w[tok] * (peak / w[tok].square().sum(-1))[:, None]
    if r >= 8:
        tok[torch.rand((r,), generator=g, device="cuda") < 0.1] = -1
    st["hidden"], st["weight"], st["tokens"] = h.to(TYPES[case["type"]]), w.to(TYPES[case["type"]]), tok.int()
    del h, w
    if case["kind"] == "lingrad":
        # what the forward pass left: each row's maximum, the logarithm of its sum, its entropy
        st["stats"], st["entropy"] = torch.empty((r, 2), device="cuda"), torch.empty((r,), device="cuda")
        for a in range(0, r, 1024):
            m, ls, e = _row_sums(_logits(st, a, a + 1024))
            st["stats"][a:a + 1024], st["entropy"][a:a + 1024] = torch.stack([m, ls], dim=1), e
        st["glp"] = torch.randn((r,), generator=g, device="cuda")
        st["gent"] = torch.randn((r,), generator=g, device="cuda").mul_(0.01) if case["entropy"] else None
    if own:  # scratch that a training loop keeps from step to step
        import paper_2607_26253_gb300 as sara
        st["workspace"] = sara.linear_logprobs_workspace(r, d, v, backward=case["kind"] == "lingrad")
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _run_own(state)
    if kind == "shared":
        return _plain_shared(state)
    return _plain_lin(state) if kind == "lin" else _plain_lingrad(state)


def _run_own(st):
    import paper_2607_26253_gb300 as sara
    kind = st["case"]["kind"]
    if kind == "shared":
        return sara.attention_shared_kv8(st["q"], st["codes"], st["scales"], st["table"], st["ctx"], st["start"], st["prefix"],
                                         workspace=st["workspace"])
    scale = st["case"]["scale"]
    if kind == "lin":
        o = sara.linear_logprobs(st["hidden"], st["weight"], st["tokens"], scale=scale, workspace=st["workspace"])
        return {"logprob": o.logprob, "entropy": o.entropy, "stats": o.stats}
    gh, gw = sara.linear_logprobs_backward(st["hidden"], st["weight"], st["tokens"], st["stats"], st["entropy"], st["glp"], st["gent"],
                                           scale=scale, workspace=st["workspace"])
    return {"hidden": gh, "weight": gw}


def _plain_values(st, seq, pos):
    """K and V at (sequence, position) pairs: [..., 2, kv, hd] in 32 bits."""
    page, slot = st["table"].long()[seq, pos // PAGE], pos % PAGE
    c = st["codes"].view(torch.uint8)[page, :, :, slot].view(st["codes"].dtype)
    return c.float() * st["scales"][page, :, :, slot // BLOCK][..., None]


def _part(q, x, live):
    """Maximum, sum and weighted values of q [b, kv, G, hd] over x [b, n, 2, kv, hd], where live [b or 1, ..., n]."""
    k, v = x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)
    s = (q @ k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    s = torch.where(live, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    return m, p.sum(-1, keepdim=True), p @ v


def _plain_shared(st):
    case = st["case"]
    start, prefix, ctx = st["lens"]
    n, kv, hd, G = len(ctx), case["kv"], case["hd"], case["heads"] // case["kv"]
    q = st["q"].float().view(n, kv, G, hd)
    group = torch.searchsorted(st["start"][1:].long(), torch.arange(n, device="cuda"), right=True)
    first = st["prefix"].long()[group]
    # the sequences' own positions
    cap = int(max(1, (ctx - np.repeat(prefix, np.diff(start))).max()))
    pos = first[:, None] + torch.arange(cap, device="cuda")
    live = pos < st["ctx"][:, None]
    x = _plain_values(st, torch.arange(n, device="cuda")[:, None], torch.where(live, pos, 0))
    m, l, o = _part(q, torch.where(live[:, :, None, None, None], x, 0.0), live[:, None, None])
    # the groups' shared ones: the rows of a group side by side, [1, kv, rows * G, positions]
    out = torch.empty_like(q)
    for j in range(case["groups"]):
        a, b, c = int(start[j]), int(start[j + 1]), int(prefix[j])
        pos = torch.arange(c, device="cuda")
        x = _plain_values(st, torch.full((1, c), a, device="cuda"), pos[None])
        qg = q[a:b].transpose(0, 1).reshape(1, kv, (b - a) * G, hd)
        live = (pos < st["ctx"][a:b, None]).repeat_interleave(G, 0)[None, None]
        m2, l2, o2 = (t.view(kv, b - a, G, -1).transpose(0, 1) for t in _part(qg, x, live))
        top = torch.maximum(m[a:b], m2)
        top = torch.where(top > -math.inf, top, 0.0)
        f1, f2 = torch.exp(m[a:b] - top), torch.exp(m2 - top)
        out[a:b] = (f1 * o[a:b] + f2 * o2) / (f1 * l[a:b] + f2 * l2).clamp_min(1e-30)
    return out.reshape(n, case["heads"], hd).to(st["q"].dtype)


def _logits(st, a=0, b=None):
    return (st["hidden"][a:b].float() @ st["weight"].float().t()) * st["case"]["scale"]


def _row_sums(z):
    """Maximum, logarithm of the sum of e^(z - max), entropy of each row."""
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1, keepdim=True)
    ls = torch.log(s)
    return m[:, 0], ls[:, 0], (ls - (e * d).sum(-1, keepdim=True) / s)[:, 0]


def _plain_lin(st):
    z, tok = _logits(st), st["tokens"].long()
    live = tok >= 0
    m, ls, h = _row_sums(z)
    lp = z.gather(1, tok.clamp_min(0)[:, None])[:, 0] - m - ls
    return {"logprob": torch.where(live, lp, 0.0), "entropy": torch.where(live, h, 0.0),
            "stats": torch.where(live[:, None], torch.stack([m, ls], dim=1), 0.0)}


def _plain_lingrad(st):
    tok, scale = st["tokens"].long(), st["case"]["scale"]
    live = (tok >= 0)[:, None]
    logp = _logits(st).sub_(st["stats"][:, :1]).sub_(st["stats"][:, 1:])
    p = torch.exp(logp)
    d = p * -st["glp"][:, None]
    d.scatter_add_(1, tok.clamp_min(0)[:, None], st["glp"][:, None])
    if st["gent"] is not None:
        d -= st["gent"][:, None] * p * (logp + st["entropy"][:, None])
    d = torch.where(live, d * scale, 0.0)
    h = torch.where(live, st["hidden"].float(), 0.0)
    return {"hidden": (d @ st["weight"].float()).to(st["hidden"].dtype), "weight": (d.t() @ h).to(st["weight"].dtype)}


# ------------------------------------------------------------------------------------------------ necessary work
def work(case):
    if case["kind"] == "shared":
        sizes, prefix = _sizes(case), _lengths(case["groups"], case["prefix"])
        n = int(sizes.sum())
        past = int(_lengths(n, case["past"]).sum())
        at = (int(prefix.sum()) + past) * case["kv"]
        return {"bytes": at * (2 * case["hd"] + 8 / BLOCK) + 4 * n * case["heads"] * case["hd"],
                "flops": 4 * (int((sizes * prefix).sum()) + past) * case["heads"] * case["hd"]}
    r, d, v = case["rows"], case["dim"], case["vocab"]
    live = 0.9 * r if r >= 8 else r
    if case["kind"] == "lin":
        return {"bytes": 2 * d * (live + v) + 20 * r, "flops": 2 * live * d * v}
    return {"bytes": 4 * d * (r + v) + 24 * r, "flops": 6 * live * d * v}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _exact_history(st, i, a, b):
    """Positions a..b in sequence i's pages, [2, kv, b - a, hd] in 64 bits."""
    pages = st["table"][i, a // PAGE:-(-b // PAGE)].long()
    x = st["codes"].view(torch.uint8)[pages].view(st["codes"].dtype).double().unflatten(3, (PAGE // BLOCK, BLOCK))
    x = (x * st["scales"][pages].double()[..., None, None]).permute(1, 2, 0, 3, 4, 5).flatten(2, 4)
    return x[:, :, a % PAGE:a % PAGE + b - a]


def _exact_shared(case, seed):
    st = prepare(case, seed)
    start, prefix, ctx = st["lens"]
    G = case["heads"] // case["kv"]
    if 4e-12 * float((np.diff(start) * prefix).sum() + ctx.sum()) * case["heads"] * case["hd"] > 10:
        return None
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for j in range(case["groups"]):
        common = _exact_history(st, int(start[j]), 0, int(prefix[j]))
        for i in range(int(start[j]), int(start[j + 1])):
            c, n = int(prefix[j]), int(ctx[i])
            if n == 0:
                continue
            x = common[:, :, :n] if n <= c else torch.cat([common, _exact_history(st, i, c, n)], 2)
            q = st["q"][i].double().unflatten(0, (case["kv"], G))
            p = torch.softmax(torch.einsum("khd,knd->khn", q, x[0]) / math.sqrt(case["hd"]), dim=-1)
            out[i] = torch.einsum("khn,knd->khd", p, x[1]).flatten(0, 1)
    return out


def exact(case, seed):
    if case["kind"] == "shared":
        return _exact_shared(case, seed)
    st = prepare(case, seed)
    w, grad = st["weight"].double(), case["kind"] == "lingrad"
    gw, rows = torch.zeros_like(w) if grad else None, []
    for a in range(0, case["rows"], 512):
        tok = st["tokens"][a:a + 512].long()
        live = tok >= 0
        h = st["hidden"][a:a + 512].double()[live]
        z = (h @ w.t()) * case["scale"]
        logp = torch.log_softmax(z, dim=-1)
        ent = -(logp.exp() * logp).sum(-1)
        if not grad:
            o = {"logprob": logp.gather(1, tok[live][:, None])[:, 0], "entropy": ent,
                 "stats": torch.stack([z.amax(-1), torch.logsumexp(z, -1) - z.amax(-1)], dim=1)}
        else:
            glp = st["glp"][a:a + 512].double()[live, None]
            d = torch.zeros_like(z).scatter_(1, tok[live][:, None], glp) - glp * logp.exp()
            if st["gent"] is not None:
                d -= st["gent"][a:a + 512].double()[live, None] * logp.exp() * (logp + ent[:, None])
            d *= case["scale"]
            gw += d.t() @ h
            o = {"hidden": d @ w}
        rows.append({k: torch.zeros((len(tok),) + x.shape[1:], dtype=torch.float64, device="cuda").index_put((live,), x)
                     for k, x in o.items()})
    whole = {k: torch.cat([o[k] for o in rows]) for k in rows[0]}
    if grad:
        whole["weight"] = gw
    return whole
