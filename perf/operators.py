"""Performance cases of the kernel-level operators over an 8-bit KV cache and over the logits of sampled tokens.

  write   new tokens' keys and values enter a paged 8-bit cache (`kv8_write`), and the scale blocks they touched are
          read back (`kv8_read`), which gives the values that the codes stand for
  read    sequences' histories come back from the cache in 16 bits (`kv8_read`)
  attn    one query row per sequence attends over its history in that cache (`attention_decode_kv8`)
  score   log-probability of a given token per row of logits, the row's entropy, the top alternatives (`logprobs`)
  grad    the gradient of log-probability and entropy with respect to the logits (`logprobs_backward`)

The cache: pages of 128 positions, codes [pages][2 (K, V)][KV heads][128][head dim] in e4m3 or int8, one fp32 scale per
32 positions, KV head and K or V: [pages][2][KV heads][4], a power of two.  A sequence's pages stand in its row of a
table.  With `own` false the same operators are computed by elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

PAGE, BLOCK = 128, 32          # positions of a page, tokens of a scale
TOP = {"e4m3": 448.0, "int8": 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
LOWEST_EXPONENT = -100
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a decode step of a mid-round batch appends one token to each of 26 ragged rollouts: latency
        {"name": "write 26 x 1", "kind": "write", "rows": 26, "new": 1, "past": 758, "kv": 2, "hd": 128, "code": "e4m3",
         "type": "bf16"},
        # fresh prompts of a round: 64 of 1,024 tokens at 8 KV heads
        {"name": "write 64 x 1024", "kind": "write", "rows": 64, "new": 1024, "past": 0, "kv": 8, "hd": 128,
         "code": "int8", "type": "fp16"},
        # the histories of a mid-round batch, one layer, to go on with in 16 bits
        {"name": "read 26 x 758", "kind": "read", "rows": 26, "ctx": 758, "kv": 2, "hd": 128, "code": "int8",
         "type": "fp16"},
        # a large pool of long histories at 8 KV heads
        {"name": "read 48 x 4096", "kind": "read", "rows": 48, "ctx": 4096, "kv": 8, "hd": 128, "code": "e4m3",
         "type": "bf16"},
        # the last live rollout of a round: a single row, latency
        {"name": "attn 1 x 758", "kind": "attn", "rows": 1, "ctx": 758, "heads": 12, "kv": 2, "hd": 128, "code": "e4m3",
         "type": "bf16", "window": 0},
        # the mean number of live rows of the 1.5B-shaped workload at its median context
        {"name": "attn 26 x 758", "kind": "attn", "rows": 26, "ctx": 758, "heads": 12, "kv": 2, "hd": 128,
         "code": "int8", "type": "fp16", "window": 0},
        # a full batch of long histories, bound by reading the cache
        {"name": "attn 64 x 8192", "kind": "attn", "rows": 64, "ctx": 8192, "heads": 32, "kv": 8, "hd": 128,
         "code": "e4m3", "type": "bf16", "window": 0},
        # two very long histories: the work of a row has to be split
        {"name": "attn 2 x 200000", "kind": "attn", "rows": 2, "ctx": 200000, "heads": 16, "kv": 2, "hd": 128,
         "code": "int8", "type": "fp16", "window": 0},
        # a decode step's logits, with the alternatives that a user asks for: latency
        {"name": "score 26 rows top 8", "kind": "score", "rows": 26, "vocab": 151936, "type": "fp32", "top": 8,
         "masked": False},
        # a batch of rollouts scored for the policy loss, a tenth of the rows padding
        {"name": "score 2048 rows", "kind": "score", "rows": 2048, "vocab": 151936, "type": "bf16", "top": 0,
         "masked": False},
        # a small policy's training rows: odd vocabulary, rows that start off every alignment
        {"name": "grad 300 x 32001", "kind": "grad", "rows": 300, "vocab": 32001, "type": "bf16", "entropy": True,
         "masked": True},
        # the policy loss's gradient at the 1.5B shape's vocabulary
        {"name": "grad 2048 x 151936", "kind": "grad", "rows": 2048, "vocab": 151936, "type": "fp32", "entropy": True,
         "masked": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "read", "attn", "attn", "score", "grad"])
    if kind in ("write", "read", "attn"):
        c = {"kind": kind, "rows": _log_int(rng, 1, 256), "kv": rng.choice([1, 2, 2, 4, 8]), "hd": rng.choice([32, 64, 128, 128]),
             "code": rng.choice(["e4m3", "int8"]), "type": rng.choice(["bf16", "fp16"])}
        width = c["kv"] * c["hd"]
        if kind == "attn":  # at most the positions of the largest listed case
            c["heads"] = c["kv"] * rng.choice([1, 2, 3, 4, 6, 8])
            c["ctx"] = _log_int(rng, 1, min(200000, max(1, 64 * 8192 * 1024 // (c["rows"] * width * 2))))
            c["window"] = rng.choice([0, 0, 0, 500])
        elif kind == "read":
            c["ctx"] = _log_int(rng, 1, min(50000, max(1, 48 * 4096 * 1024 // (c["rows"] * width * 2))))
        else:
            c["past"] = rng.choice([0, _log_int(rng, 1, 4000)])
            c["new"] = rng.choice([1, _log_int(rng, 1, max(1, min(16384, 64 * 1024 * 1024 // (c["rows"] * width))))])
        return c
    vocab = rng.choice([151936, 512, _log_int(rng, 300, 152000), 32000 + rng.randrange(999)])
    c = {"kind": kind, "rows": _log_int(rng, 1, max(1, min(16384, 2048 * 151936 // (2 * vocab)))), "vocab": vocab,
         "type": rng.choice(["fp32", "bf16", "bf16", "fp16"]), "masked": rng.random() < 0.3}
    if kind == "score":
        c["top"] = rng.choice([0, 1, 5, 20, 32]) if c["rows"] * vocab <= 32 * 151936 else 0
    else:
        c["entropy"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(n, mean):
    """Ragged lengths of a given mean, lognormal as rollouts' are; the case's own, so that every seed has the same sizes."""
    x = np.exp(0.5 * np.random.default_rng([n, mean]).standard_normal(n))
    return np.maximum(np.rint(x * (mean * n / x.sum())), 1).astype(np.int64)


def _table(rng, lens):
    """Pages of n sequences, shuffled over a pool that has a few more; unused entries of the table are -1."""
    per = -(-lens // PAGE)
    table = np.full((len(lens), max(1, int(per.max()))), -1, np.int32)
    ids = rng.permutation(int(per.sum()) + 3).astype(np.int32)
    used = np.arange(table.shape[1])[None, :] < per[:, None]
    table[used] = ids[:int(per.sum())]
    return table, len(ids)


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


def _logits(case, seed):
    """Logits of a trained policy's kind: N(0, 2) with the sampled token standing out in most rows; where `masked`, a
    tenth of the vocabulary is not allowed (-inf); a tenth of the rows is padding (token -1)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r, v = case["rows"], case["vocab"]
    z = torch.empty((r, v), dtype=TYPES[case["type"]], device="cuda")
    tok = torch.randint(0, v, (r,), generator=g, device="cuda")
    peak = 4.0 * torch.randn((r,), generator=g, device="cuda") + 9.0
    off = torch.rand((v,), generator=g, device="cuda") < 0.1
    for a in range(0, r, 256):
        x = torch.randn((min(256, r - a), v), generator=g, device="cuda").mul_(2.0)
        if case["masked"]:
            x[:, off] = -math.inf
        z[a:a + 256].copy_(x)
    z[torch.arange(r, device="cuda"), tok] = peak.to(z.dtype)
    if r >= 8:
        tok[torch.rand((r,), generator=g, device="cuda") < 0.1] = -1
    return g, z, tok.int()


def prepare(case, seed):
    st = {"case": case}
    kind = case["kind"]
    if kind in ("score", "grad"):
        g, st["logits"], st["tokens"] = _logits(case, seed)
        if kind == "grad":
            # what the forward pass left: each row's maximum, the logarithm of its sum, its entropy
            r = case["rows"]
            st["stats"] = torch.empty((r, 2), device="cuda")
            st["entropy"] = torch.empty((r,), device="cuda")
            for a in range(0, r, 256):
                m, ls, h = _row_sums(st["logits"][a:a + 256].float())
                st["stats"][a:a + 256], st["entropy"][a:a + 256] = torch.stack([m, ls], dim=1), h
            st["glp"] = torch.randn((r,), generator=g, device="cuda")
            st["gent"] = torch.randn((r,), generator=g, device="cuda").mul_(0.01) if case["entropy"] else None
        return st
    g, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    n = case["rows"]
    if kind == "write":
        pos0 = _lengths(n, case["past"]) if case["past"] else np.zeros(n, np.int64)
        new = _lengths(n, case["new"]) if case["new"] > 1 else np.full(n, 1)
        table, pages = _table(rng, pos0 + new)
        st["codes"], st["scales"] = _pool(g, case, pages)
        start = np.concatenate([[0], np.cumsum(new)])
        first = pos0 // BLOCK * BLOCK  # the scale blocks touched, from their first token on
        rstart = np.concatenate([[0], np.cumsum(pos0 + new - first)])
        # keys and values as views of one projection's rows, q | k | v
        width = case["kv"] * case["hd"]
        qkv = torch.randn((int(start[-1]), 3 * width), generator=g, device="cuda", dtype=TYPES[case["type"]])
        st["k"] = qkv[:, width:2 * width].unflatten(1, (case["kv"], case["hd"]))
        st["v"] = qkv[:, 2 * width:].unflatten(1, (case["kv"], case["hd"]))
        st["pos0"], st["start"], st["total"] = _cuda(pos0), _cuda(start), int(start[-1])
        st["rpos0"], st["rstart"], st["rtotal"] = _cuda(first), _cuda(rstart), int(rstart[-1])
    else:
        lens = _lengths(n, case["ctx"])
        if kind == "attn" and n >= 16:
            lens[n // 3] = 0  # a slot of the batch without a sequence
        table, pages = _table(rng, lens)
        st["codes"], st["scales"] = _pool(g, case, pages)
        if kind == "read":
            st["rpos0"], st["rstart"] = _cuda(np.zeros(n)), _cuda(np.concatenate([[0], np.cumsum(lens)]))
            st["rtotal"] = int(lens.sum())
        else:
            st["q"] = torch.randn((n, case["heads"], case["hd"]), generator=g, device="cuda", dtype=TYPES[case["type"]])
            st["ctx"], st["first"], st["cap"] = _cuda(lens), None, int(lens.max())
            if case["window"]:
                st["first"] = _cuda(np.maximum(lens - case["window"], 0))
            if own:  # scratch that a serving loop keeps from step to step
                import paper_2607_26253_gb300 as sara
                st["workspace"] = sara.attention_kv8_workspace(n, case["heads"], case["kv"], case["hd"])
    st["table"] = _cuda(table)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "write":
        _plain_write(state)
        k, v = _plain_read(state)
        return {"k": k, "v": v, "scales": state["scales"]}
    if kind == "read":
        return _plain_read(state)
    if kind == "attn":
        return _plain_attention(state)
    return _plain_score(state) if kind == "score" else _plain_grad(state)


def _run_own(st):
    import paper_2607_26253_gb300 as sara
    case = st["case"]
    kind = case["kind"]
    if kind == "write":
        sara.kv8_write(st["codes"], st["scales"], st["table"], st["k"], st["v"], st["pos0"], st["start"])
        k, v = sara.kv8_read(st["codes"], st["scales"], st["table"], st["rpos0"], st["rstart"], st["rtotal"], TYPES[case["type"]])
        return {"k": k, "v": v, "scales": st["scales"]}
    if kind == "read":
        return sara.kv8_read(st["codes"], st["scales"], st["table"], st["rpos0"], st["rstart"], st["rtotal"], TYPES[case["type"]])
    if kind == "attn":
        return sara.attention_decode_kv8(st["q"], st["codes"], st["scales"], st["table"], st["ctx"], first=st["first"],
                                         workspace=st["workspace"])
    if kind == "score":
        o = sara.logprobs(st["logits"], st["tokens"], top=case["top"])
        out = {"logprob": o.logprob, "entropy": o.entropy, "stats": o.stats}
        if case["top"]:
            out["top_token"], out["top_logprob"] = o.top_token, o.top_logprob
        return out
    return sara.logprobs_backward(st["logits"], st["tokens"], st["stats"], st["entropy"], st["glp"], st["gent"])


def _positions(start, pos0, total):
    """Sequence and position of each of `total` packed tokens."""
    t = torch.arange(total, device="cuda")
    seq = torch.searchsorted(start[1:].long(), t, right=True)
    return seq, pos0.long()[seq] + t - start.long()[seq]


def _exponent(amax, code):
    """The smallest e with amax <= top * 2^e: amax = f * 2^x with f in [1/2, 1), 448 = 7/8 * 2^9, 127 = 127/128 * 2^7."""
    f, x = torch.frexp(amax)
    e = x - 9 + (f > 0.875) if code == "e4m3" else x - 7 + (f > 127 / 128)
    return torch.where(amax > 0, e, LOWEST_EXPONENT).clamp_min(LOWEST_EXPONENT)


def _encode(x, code):
    return (x.to(torch.float8_e4m3fn) if code == "e4m3" else x.round().to(torch.int8)).view(torch.uint8)


def _decode(c, code):
    return c.view(CODES[code]).float()


def _plain_write(st):
    code, kv, hd = st["case"]["code"], st["case"]["kv"], st["case"]["hd"]
    raw, scales, table = st["codes"].view(torch.uint8), st["scales"], st["table"].long()
    pages = raw.shape[0]
    seq, pos = _positions(st["start"], st["pos0"], st["total"])
    page, slot = table[seq, pos // PAGE], pos % PAGE
    block = page * (PAGE // BLOCK) + slot // BLOCK
    x = torch.stack([st["k"], st["v"]], dim=1).float()                     # [T, 2, kv, hd]
    amax = x.abs().amax(-1)                                                # [T, 2, kv]
    new = torch.full((pages * PAGE // BLOCK, 2, kv), -1.0, device="cuda")
    new.scatter_reduce_(0, block[:, None, None].expand_as(amax), amax, "amax")
    touched = new >= 0
    begun = torch.zeros(pages * PAGE // BLOCK, dtype=torch.int32, device="cuda")
    begun = begun.scatter_reduce_(0, block, (slot % BLOCK == 0).int(), "amax") > 0  # written from its first token
    old = torch.frexp(scales)[1].transpose(-1, -2).transpose(-2, -3).reshape(-1, 2, kv) - 1
    e = _exponent(new, code)
    e = torch.where(touched, torch.where(begun[:, None, None], e, torch.maximum(e, old)), old)
    # codes before the first new token of a block that has some
    p0 = st["pos0"].long()
    last = table.shape[1] - 1
    opage = table.gather(1, (p0 // PAGE).clamp_max(last)[:, None])[:, 0]
    oslot = (p0 % PAGE // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device="cuda")
    oblock = opage * (PAGE // BLOCK) + p0 % PAGE // BLOCK
    at = (opage[:, None], slice(None), slice(None), oslot)
    have = raw[at]                                                         # [rows, 32, 2, kv, hd]
    shift = torch.exp2((old - e)[oblock].float())[:, None, :, :, None]
    keep = (torch.arange(BLOCK, device="cuda") < (p0 % BLOCK)[:, None])[:, :, None, None, None]
    raw[at] = torch.where(keep, _encode(_decode(have, code) * shift, code), have)
    raw[page, :, :, slot] = _encode(x * torch.exp2(-e[block].float())[..., None], code)
    scales.copy_(torch.exp2(e.float()).view(pages, PAGE // BLOCK, 2, kv).permute(0, 2, 3, 1))


def _plain_values(st, seq, pos):
    """K and V at (sequence, position) pairs: [..., 2, kv, hd] in 32 bits."""
    page, slot = st["table"].long()[seq, pos // PAGE], pos % PAGE
    c = st["codes"].view(torch.uint8)[page, :, :, slot]
    return _decode(c, st["case"]["code"]) * st["scales"][page, :, :, slot // BLOCK][..., None]


def _plain_read(st):
    seq, pos = _positions(st["rstart"], st["rpos0"], st["rtotal"])
    x = _plain_values(st, seq, pos).to(TYPES[st["case"]["type"]])
    return x[:, 0].contiguous(), x[:, 1].contiguous()


def _plain_attention(st):
    case = st["case"]
    n, kv, hd, G = case["rows"], case["kv"], case["hd"], case["heads"] // case["kv"]
    pos = torch.arange(st["cap"], device="cuda").expand(n, -1)
    live = pos < st["ctx"][:, None]
    if st["first"] is not None:
        live = live & (pos >= st["first"][:, None])
    x = _plain_values(st, torch.arange(n, device="cuda")[:, None], torch.where(live, pos, 0))   # [n, cap, 2, kv, hd]
    k, v = x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)                                # [n, kv, cap, hd]
    q = st["q"].float().view(n, kv, G, hd)
    s = (q @ k.transpose(-1, -2)) / math.sqrt(hd)                                               # [n, kv, G, cap]
    s = torch.where(live[:, None, None], s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    o = (p @ v) / p.sum(-1, keepdim=True).clamp_min(1e-30)
    return o.reshape(n, case["heads"], hd).to(st["q"].dtype)


def _row_sums(z):
    """Maximum, logarithm of the sum of e^(z - max), entropy of each row."""
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1, keepdim=True)
    ls = torch.log(s)
    return m[:, 0], ls[:, 0], (ls - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / s)[:, 0]


def _plain_score(st):
    z, tok, top = st["logits"].float(), st["tokens"].long(), st["case"]["top"]
    live = tok >= 0
    m, ls, h = _row_sums(z)
    lp = z.gather(1, tok.clamp_min(0)[:, None])[:, 0] - m - ls
    out = {"logprob": torch.where(live, lp, 0.0), "entropy": torch.where(live, h, 0.0),
           "stats": torch.where(live[:, None], torch.stack([m, ls], dim=1), 0.0)}
    if top:
        # one whole number for value and place, so that equal values go by the lowest place
        b = (z + 0.0).view(torch.int32).long()
        key = torch.where(b < 0, -(b & 0x7fffffff), b) * (1 << 32) + (z.shape[1] - 1 - torch.arange(z.shape[1], device="cuda"))
        at = z.shape[1] - 1 - (key.topk(top, dim=1).values & 0xffffffff)
        out["top_token"] = torch.where(live[:, None], at, -1).int()
        out["top_logprob"] = torch.where(live[:, None], z.gather(1, at) - m[:, None] - ls[:, None], -math.inf)
    return out


def _plain_grad(st):
    z, tok = st["logits"].float(), st["tokens"].long()
    live = tok >= 0
    logp = z - st["stats"][:, :1] - st["stats"][:, 1:]
    p = torch.exp(logp)
    d = -st["glp"][:, None] * p
    d.scatter_add_(1, tok.clamp_min(0)[:, None], st["glp"][:, None])
    if st["gent"] is not None:
        d = d - torch.where(p > 0, st["gent"][:, None] * p * (logp + st["entropy"][:, None]), 0.0)
    return torch.where(live[:, None], d, 0.0).to(st["logits"].dtype)


# ------------------------------------------------------------------------------------------------ necessary work
def work(case):
    kind = case["kind"]
    if kind in ("score", "grad"):
        live = 0.9 if case["rows"] >= 8 else 1.0
        cells = case["rows"] * case["vocab"]
        size = 4 if case["type"] == "fp32" else 2
        if kind == "score":
            return {"bytes": live * cells * size + case["rows"] * (20 + 8 * case["top"]), "flops": 5 * live * cells}
        return {"bytes": (1 + live) * cells * size + 24 * case["rows"], "flops": 8 * live * cells}
    width = case["kv"] * case["hd"]
    scales = 2 * 4 * case["kv"] / BLOCK  # bytes of scales per position
    if kind == "write":
        new = case["rows"] * case["new"]
        back = new + case["rows"] * (BLOCK / 2 if case["past"] else 0)
        return {"bytes": new * width * 2 * (2 + 1) + back * width * 2 * 2 + back * scales, "flops": 2 * new * width * 2}
    pos = case["rows"] * case["ctx"]
    if kind == "read":
        return {"bytes": pos * (width * 2 * (1 + 2) + scales), "flops": 2 * pos * width}
    if case["window"]:
        pos = case["rows"] * min(case["ctx"], case["window"])
    return {"bytes": pos * (width * 2 + scales) + 4 * case["rows"] * case["heads"] * case["hd"],
            "flops": 4 * pos * case["heads"] * case["hd"]}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _to_grid(x, code):
    """x rounded to the nearest value of the code's grid (ties to even), in 64 bits."""
    if code == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)  # 3 bits behind the first; subnormal below 2^-6
    return torch.round(x / step) * step


def _exact_write(case, seed):
    st = prepare(case, seed)
    code, kv, hd, n = case["code"], case["kv"], case["hd"], case["rows"]
    host = {k: st[k].cpu().numpy() for k in ("table", "pos0", "start", "rstart")}
    scales = st["scales"].double()
    ks, vs = [], []
    for i in range(n):
        p0, a, b = int(host["pos0"][i]), int(host["start"][i]), int(host["start"][i + 1])
        first, end = p0 // BLOCK * BLOCK, p0 + b - a
        blocks = -(-(end - first) // BLOCK)
        ids = torch.from_numpy(host["table"][i].astype(np.int64)).cuda()
        at = first + BLOCK * torch.arange(blocks, device="cuda")
        page, part = ids[at // PAGE], at % PAGE // BLOCK
        fresh = torch.stack([st["k"][a:b], st["v"][a:b]]).double()         # [2, new, kv, hd]
        gap = p0 - first
        x = torch.zeros((2, blocks * BLOCK, kv, hd), dtype=torch.float64, device="cuda")
        x[:, gap:gap + b - a] = fresh
        x = x.view(2, blocks, BLOCK, kv, hd)
        need = x.abs().amax((2, 4)) / TOP[code]                            # [2, blocks, kv]
        e = torch.ceil(torch.log2(need.clamp_min(2.0 ** LOWEST_EXPONENT)))
        e = torch.where(torch.exp2(e) < need, e + 1, e)
        if gap:
            was = scales[page[0], :, :, part[0]]                           # [2, kv]
            e[:, 0] = torch.maximum(e[:, 0], torch.log2(was).round())
            s0 = int(part[0]) * BLOCK
            held = st["codes"][int(page[0]), :, :, s0:s0 + gap].double() * was[:, :, None, None]
            x[:, 0, :gap] = held.transpose(1, 2)
        s = torch.exp2(e)[:, :, None, :, None]
        y = (_to_grid(x / s, code) * s).view(2, blocks * BLOCK, kv, hd)[:, :end - first]
        scales[page, :, :, part] = torch.exp2(e).transpose(0, 1)
        ks.append(y[0])
        vs.append(y[1])
    return {"k": torch.cat(ks), "v": torch.cat(vs), "scales": scales}


def _exact_history(st, i, a, b):
    """Positions a..b of sequence i, [2, kv, b - a, hd] in 64 bits."""
    pages = st["table"][i, a // PAGE:-(-b // PAGE)].long()
    x = st["codes"].view(torch.uint8)[pages].view(st["codes"].dtype).double().unflatten(3, (PAGE // BLOCK, BLOCK)) * st["scales"][pages].double()[..., None, None]
    x = x.permute(1, 2, 0, 3, 4, 5).flatten(2, 4)
    return x[:, :, a % PAGE:a % PAGE + b - a]


def exact(case, seed):
    kind = case["kind"]
    if kind == "write":
        return _exact_write(case, seed)
    st = prepare(case, seed)
    if kind == "read":
        at = st["rstart"].tolist()
        got = [_exact_history(st, i, 0, at[i + 1] - at[i]) for i in range(case["rows"])]
        return tuple(torch.cat([x[j].transpose(0, 1) for x in got]) for j in (0, 1))
    if kind == "attn":
        G = case["heads"] // case["kv"]
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        ctx = st["ctx"].tolist()
        first = st["first"].tolist() if st["first"] is not None else [0] * len(ctx)
        for i, (a, b) in enumerate(zip(first, ctx)):
            if a >= b:
                continue
            k, v = _exact_history(st, i, a, b)
            for h in range(case["heads"]):
                p = torch.softmax(k[h // G] @ st["q"][i, h].double() / math.sqrt(case["hd"]), dim=0)
                out[i, h] = p @ v[h // G]
        return out
    rows = []
    for r in range(0, case["rows"], 64):
        z, tok = st["logits"][r:r + 64].double(), st["tokens"][r:r + 64].long()
        logp = torch.log_softmax(z, dim=-1)
        p = logp.exp()
        h = torch.special.entr(p).sum(-1)
        live = tok >= 0
        if kind == "score":
            m = z.amax(-1)
            o = {"logprob": logp.gather(1, tok.clamp_min(0)[:, None])[:, 0] * live, "entropy": h * live,
                 "stats": torch.stack([m, torch.logsumexp(z, -1) - m], dim=1) * live[:, None]}
            if case["top"]:
                top, at = (t[:, :case["top"]] for t in torch.sort(logp, dim=-1, descending=True, stable=True))
                o["top_token"] = torch.where(live[:, None], at, -1).int()
                o["top_logprob"] = torch.where(live[:, None], top, -math.inf)
        else:
            glp = st["glp"][r:r + 64].double()[:, None]
            d = -glp * p
            d[torch.arange(len(tok), device="cuda")[live], tok[live]] += glp[live, 0]
            if st["gent"] is not None:
                d -= st["gent"][r:r + 64].double()[:, None] * (p * h[:, None] - torch.special.entr(p))
            o = {"grad": torch.where(live[:, None], d, 0.0)}
        rows.append(o)
    whole = {key: torch.cat([o[key] for o in rows]) for key in rows[0]}
    return whole if kind == "score" else whole["grad"]
