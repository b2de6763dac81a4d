"""Log-probabilities, entropy, alternatives and their gradient on the GPU against the 64-bit oracle, within bounds that follow
from 32-bit arithmetic."""
import numpy as np
import pytest

import synth
from oracle import scoring as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    p.load()
    return p


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def _i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _logits(rng, R, V, typ, std=2.0, mean=0.0):
    import torch
    return torch.from_numpy(mean + std * rng.standard_normal((R, V))).cuda().to(_dtype(typ))


def _sum_bound(V):
    # sums of V terms, at most V / 128 in a chain, each term an exponential good to 2^-21
    return (V / 128 + 48) * U


def _close(got, want, tol):
    if not np.isfinite(want):
        return np.isnan(got) if np.isnan(want) else got == want
    return abs(got - want) <= tol


def _check(o, z, tokens, top, alike=False):
    """alike: probabilities so alike that rounding may order them otherwise is no concern here (values compare exactly)."""
    zn = z.double().cpu().numpy()
    V = zn.shape[1]
    lp = o.logprob.double().cpu().numpy() if o.logprob is not None else None
    H, st = o.entropy.double().cpu().numpy(), o.stats.double().cpu().numpy()
    tt, tl = (o.top_token.cpu().numpy(), o.top_logprob.double().cpu().numpy()) if top else (None, None)
    for r in range(len(zn)):
        w = oracle.score(zn[r], None if tokens is None else int(tokens[r]), top)
        d = np.abs(zn[r][np.isfinite(zn[r])] - w["max"]) if np.isfinite(w["max"]) else np.zeros(1)
        b = _sum_bound(V)
        if lp is not None:
            away = abs(w["logprob"]) if np.isfinite(w["logprob"]) else 0.0
            assert _close(lp[r], w["logprob"], b + 4 * U * (away + abs(w["logsum"]) + 1)), (r, lp[r], w)
        # T / S: terms e |d|, where e |d| sums to S times the mean distance
        mean = 0.0
        if np.isfinite(w["entropy"]) and np.isfinite(w["max"]) and len(d):
            mean = float((np.exp(-d) * d).sum() / np.exp(-d).sum())
        assert _close(H[r], w["entropy"], (b + 4 * U) * (1 + 2 * mean + abs(w["logsum"]))), (r, H[r], w["entropy"])
        assert _close(st[r, 0], w["max"], 0) or (np.isnan(w["logsum"]) and not np.isfinite(w["max"])), (r, st[r], w["max"])
        assert _close(st[r, 1], w["logsum"], b + 2 * U * abs(w["logsum"])), (r, st[r], w["logsum"])
        if top:
            assert tt[r].tolist() == w["top_token"], (r, tt[r], w["top_token"])
            for j in range(top):
                away = abs(w["top_logprob"][j]) if np.isfinite(w["top_logprob"][j]) else 0.0
                assert _close(tl[r, j], w["top_logprob"][j], b + 4 * U * (away + abs(w["logsum"]) + 1)), (r, j)


# vocabularies from one token on, around vectors, warps' and CTAs' shares; odd ones leave rows unaligned
@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [1, 2, 5, 8, 31, 32, 33, 127, 512, 2047, 8191, 32001, 131073])
def test_vocabularies(pkg, V, typ):
    rng = np.random.default_rng(V)
    z = _logits(rng, 5, V, typ)
    tok = rng.integers(0, V, 5)
    for top in (0, 3, 32):
        _check(pkg.logprobs(z, _i32(tok), top=top), z, tok, top)


@pytest.mark.parametrize("R,V", [(1, 151936), (26, 151936), (200, 4099), (900, 1003), (5000, 33), (153, 20000), (305, 9000)])
def test_rows(pkg, R, V):
    rng = np.random.default_rng(R)
    z = _logits(rng, R, V, "bf16", 3.0)
    tok = rng.integers(0, V, R)
    tok[R // 2:: 7] = -1
    _check(pkg.logprobs(z, _i32(tok), top=5), z, tok, 5)


# on either side of the lines between a warp, 4 warps, 8 warps and a cluster a row, with and without alternatives
@pytest.mark.parametrize("R,V,typ,top", [(609, 4099, "bf16", 0), (609, 65600, "bf16", 0), (609, 70001, "bf16", 0), (700, 5003, "fp32", 0),
                                        (609, 8190, "bf16", 7), (609, 8300, "fp16", 7), (304, 33000, "fp32", 0), (305, 33000, "fp32", 3),
                                        (1300, 2051, "fp32", 32), (40, 300, "fp32", 1)])
def test_kernels_by_size(pkg, R, V, typ, top):
    rng = np.random.default_rng(R + V)
    z = _logits(rng, R, V, typ, 3.0)
    tok = rng.integers(0, V, R)
    tok[::9] = -1
    keep = rng.permutation(R)[:60]  # (a part of the rows against the oracle)
    o = pkg.logprobs(z, _i32(tok), top=top)
    pick = lambda x: x[_i32(keep).long()] if x is not None else None  # noqa: E731
    _check(pkg.LogProbs(*[pick(x) for x in (o.logprob, o.entropy, o.stats, o.top_token, o.top_logprob)]), pick(z), tok[keep], top)


# rows that just fill the SMs in clusters of two, four and eight, and one more
@pytest.mark.parametrize("typ", ["bf16", "fp32"])
@pytest.mark.parametrize("V,top", [(33001, 0), (33001, 8), (70001, 0)])
@pytest.mark.parametrize("per_sm", [4, 3])
@pytest.mark.parametrize("ctas", [2, 4, 8])
def test_rows_that_fill_the_gpu_in_clusters(pkg, ctas, per_sm, V, top, typ):
    import torch
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for R in (per_sm * sms // ctas, per_sm * sms // ctas + 1):
        rng = np.random.default_rng(R)
        z = torch.empty((R, V), device="cuda").normal_(0.0, 3.0, generator=torch.Generator("cuda").manual_seed(R)).to(_dtype(typ))
        tok = rng.integers(0, V, R)
        keep = np.concatenate([rng.permutation(R - 2)[:6], [R - 2, R - 1]])
        o = pkg.logprobs(z, _i32(tok), top=top)
        pick = lambda x: x[_i32(keep).long()] if x is not None else None  # noqa: E731
        _check(pkg.LogProbs(*[pick(x) for x in (o.logprob, o.entropy, o.stats, o.top_token, o.top_logprob)]), pick(z), tok[keep], top)


# long rows that fill the SMs and some more: the last ones are taken by 2 or 4 CTAs each, in a grid that starts while the others end
@pytest.mark.parametrize("R,V,typ", [(700, 70001, "bf16"), (860, 33001, "fp32"), (912, 65552, "fp16"), (913, 65552, "fp16")])
def test_last_rows_of_many_long_ones(pkg, R, V, typ):
    import torch
    rng = np.random.default_rng(R)
    gen = torch.Generator("cuda").manual_seed(R)
    z = torch.empty((R, V), device="cuda").normal_(0.0, 3.0, generator=gen).to(_dtype(typ))
    tok = rng.integers(0, V, R)
    tok[::11] = -1
    tok[R - 1], tok[R - 3] = 5, V
    keep = np.concatenate([rng.permutation(608)[:20], np.arange(606, 612), np.arange(R - 20, R)])
    o = pkg.logprobs(z, _i32(tok))
    pick = lambda x: x[_i32(keep).long()] if x is not None else None  # noqa: E731
    _check(pkg.LogProbs(*[pick(x) for x in (o.logprob, o.entropy, o.stats, None, None)]), pick(z), tok[keep], 0)
    p = pkg.logprobs(z, None)
    live = _i32(tok).ge(0)
    assert p.logprob is None and torch.equal(p.entropy[live], o.entropy[live]) and torch.equal(p.stats[live], o.stats[live])
    # captured, with a kernel behind it that reads what both grids wrote
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    dtok = _i32(tok)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        c = pkg.logprobs(z, dtok)
        both = c.logprob + c.entropy
    for _ in range(5):
        both.zero_()
        graph.replay()
        assert torch.equal(both.nan_to_num(7.0), (o.logprob + o.entropy).nan_to_num(7.0))


def test_no_rows(pkg):
    import torch
    z, none = torch.empty((0, 50), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    o = pkg.logprobs(z, none, top=3)
    assert o.logprob.shape == (0,) and o.top_token.shape == (0, 3)
    assert pkg.logprobs_backward(z, none, o.stats, o.entropy, o.logprob).shape == (0, 50)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_strided_rows_off_every_alignment(pkg, off, typ):
    import torch
    rng = np.random.default_rng(off)
    z = _logits(rng, 6, 5003, typ)[:, off:off + 4099]
    tok = rng.integers(0, 4099, 6)
    o = pkg.logprobs(z, _i32(tok), top=8)
    _check(o, z, tok, 8)
    g, gh = (torch.from_numpy(rng.standard_normal(6)).float().cuda() for _ in range(2))
    out = torch.full((6, 5001), 7.0, dtype=z.dtype, device="cuda")
    pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh, out=out[:, 1:4100])
    _check_grad(out[:, 1:4100], z, tok, g, gh)
    assert (out[:, 0] == 7).all() and (out[:, 4100:] == 7).all()


# equal values, everywhere and within a few levels: the alternatives go by the lowest token
@pytest.mark.parametrize("V", [40, 4099, 70001])
@pytest.mark.parametrize("levels", [1, 2, 9])
def test_ties(pkg, V, levels):
    import torch
    rng = np.random.default_rng(V)
    z = torch.from_numpy(rng.integers(0, levels, (4, V))).cuda().float()
    z[3] = torch.where(z[3] == 0, -0.0, z[3])  # -0 equals 0
    z[3, ::2] = z[3, ::2].abs()
    tok = rng.integers(0, V, 4)
    _check(pkg.logprobs(z, _i32(tok), top=32), z, tok, 32)


@pytest.mark.parametrize("order", ["rising", "falling"])
def test_sorted_rows(pkg, order):
    # every token raises the maximum and enters the list, or none after the first
    import torch
    z = torch.linspace(-20, 20, 30000, device="cuda").repeat(3, 1)
    z = z.flip(1).contiguous() if order == "falling" else z
    _check(pkg.logprobs(z, _i32([0, 7, 29999]), top=32), z, [0, 7, 29999], 32)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
def test_masked_infinite_and_nan(pkg, typ):
    import torch
    rng = np.random.default_rng(3)
    V = 5003
    z = _logits(rng, 12, V, typ)
    low = torch.finfo(_dtype(typ)).min
    z[0] = -np.inf                      # a row whose mask leaves nothing
    z[1, 1:] = -np.inf                  # one token left
    z[2, :4000] = -np.inf               # the token itself masked
    z[3] = low                          # masked with the type's lowest value, all of it
    z[4, 7:] = low                      # ... or most
    z[5, 100] = np.inf
    z[6, 4000] = np.nan
    z[7] = np.nan
    z[8, ::2] = -np.inf
    z[9, :] = -np.inf
    z[9, [17, 4002]] = z[9, 3] = low    # three left, at the lowest value
    z[10, 0] = torch.finfo(_dtype(typ)).max
    z[11, 5], z[11, 9] = np.inf, np.nan
    tok = np.array([4, 0, 7, 5, 6, 100, 3, 2, 1, 17, 0, 5])
    o = pkg.logprobs(z, _i32(tok), top=10)
    _check(o, z, tok, 10)
    g, gh = (torch.from_numpy(rng.standard_normal(12)).float().cuda() for _ in range(2))
    _check_grad(pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh), z, tok, g, gh)


def test_nan_wherever_it_stands(pkg):
    rng = np.random.default_rng(4)
    V = 40007
    for at in (0, 1, 5, 19999, 20000, V - 2, V - 1):
        z = _logits(rng, 2, V, "bf16")
        z[0, at] = np.nan
        o = pkg.logprobs(z, _i32([3, 3]), top=2)
        assert o.logprob.isnan().tolist() == [True, False] and o.entropy.isnan().tolist() == [True, False]
        assert o.top_token[0].tolist() == oracle.score(z[0].double().cpu().numpy(), 3, 2)["top_token"]


@pytest.mark.parametrize("mean,std", [(1e6, 1.0), (-1e6, 3.0), (3e38, 0.0), (0.0, 40.0), (0.0, 1e-3)])
def test_large_and_peaked_logits(pkg, mean, std):
    import torch
    rng = np.random.default_rng(5)
    z = _logits(rng, 8, 20011, "fp32", std, mean)
    tok = rng.integers(0, 20011, 8)
    tok[:4] = z[:4].argmax(1).cpu().numpy()
    o = pkg.logprobs(z, _i32(tok), top=4)
    _check(o, z, tok, 4)
    g, gh = (torch.from_numpy(rng.standard_normal(8)).float().cuda() for _ in range(2))
    _check_grad(pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh), z, tok, g, gh)


# Masks of finite values, from ones that rounding just reaches to the type's far end, and logits as large: all but three tokens, most of the
# row in one piece (so that threads begin with nothing else), all of it, at random, or two fills in one row.  The sizes take each kernel: a warp,
# 4 warps, a cluster, 8 warps a row, with and without alternatives, the last rows split over CTAs.
FILLS = [-1e6, -3e6, -1e9, -1e10, -1e15, -1e20, -1e30, -1e36, 1e10, 1e20, 1e30]
FILLS_FP16 = [-1e3, -1e4, -3e4, -59904.0, -60032.0, -6.2e4, -65504.0, 1e4, 3e4, 6e4, 65504.0]


def _filled(rng, R, V, typ, r0=0):
    """Rows r0 .. r0 + R of logits N(0, 3), each with its fill and its pattern."""
    z = 3.0 * rng.standard_normal((R, V))
    fills = FILLS_FP16 if typ == "fp16" else FILLS
    for r in range(R):
        fill, pattern = fills[(r0 + r) % len(fills)], (r0 + r) // len(fills) % 5
        keep = np.zeros(V, bool)
        if pattern == 0:
            keep[rng.permutation(V)[:3]] = True
        elif pattern == 1:
            keep[V - V // 10:] = True
        elif pattern == 3:
            keep = rng.random(V) < 0.1
        elif pattern == 4:
            keep[:V // 20] = True
        z[r, ~keep] = fill
        if pattern == 4:
            z[r, V // 2:] = fills[(r0 + r + 3) % len(fills)]
    import torch
    return torch.from_numpy(z).to(_dtype(typ)).cuda()


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,V,top", [(55, 300, 0), (55, 2001, 0), (55, 2001, 5), (55, 8191, 0), (55, 8191, 8), (55, 40007, 0), (55, 40007, 32), (1, 151936, 0),
                                     (640, 5003, 0), (640, 9001, 7), (609, 70001, 0)])
def test_finite_masks(pkg, R, V, top, typ):
    import torch
    rng = np.random.default_rng(R + V)
    live = min(R, 55)  # (the rest: other rows' company, rows of padding)
    z = torch.zeros((R, V), dtype=_dtype(typ), device="cuda")
    at = np.sort(rng.permutation(R)[:live])
    at[-1] = R - 1
    z[_i32(at).long()] = _filled(rng, live, V, typ, 3 if R == 1 else 0)
    tok = np.full(R, -1)
    tok[at] = rng.integers(0, V, live)
    o = pkg.logprobs(z, _i32(tok), top=top)
    pick = lambda x: x[_i32(at).long()].contiguous() if x is not None else None  # noqa: E731
    _check(pkg.LogProbs(*[pick(x) for x in (o.logprob, o.entropy, o.stats, o.top_token, o.top_logprob)]), pick(z), tok[at], top)
    g, gh = (torch.from_numpy(rng.standard_normal(R)).float().cuda() for _ in range(2))
    y = pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh)
    _check_grad(pick(y), pick(z), tok[at], pick(g), pick(gh))


def test_padding_wrong_tokens_and_no_tokens(pkg):
    import torch
    rng = np.random.default_rng(6)
    z = _logits(rng, 6, 3001, "bf16")
    z[1], z[4] = np.nan, np.inf  # (padding is not read)
    tok = np.array([5, -1, 3001, 2 ** 31 - 1, -100, 3000])
    o = pkg.logprobs(z, _i32(tok), top=3)
    _check(o, z, tok, 3)
    g = torch.ones(6, device="cuda")
    y = pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, g)
    _check_grad(y, z, tok, g, g)
    z[1], z[4] = 0, 1
    o = pkg.logprobs(z, None, top=3)
    assert o.logprob is None
    _check(o, z, None, 3)
    _check_grad(pkg.logprobs_backward(z, None, o.stats, o.entropy, None, g), z, None, 0 * g, g)


# ------------------------------------------------------------------------------------------------ gradient
def _check_grad(y, z, tokens, g, gh):
    """p is off by the roundings of z - max - log S (each half a step of what it is) and of the sum, times p."""
    got, zn = y.double().cpu().numpy(), z.double().cpu().numpy()
    gn, ghn = g.double().cpu().numpy(), gh.double().cpu().numpy()
    half = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[str(y.dtype).split(".")[1]]
    least = 2.0 ** -25 if half == 2.0 ** -11 else 2.0 ** -126
    V = zn.shape[1]
    for r in range(len(zn)):
        t = None if tokens is None else int(tokens[r])
        want = oracle.grad(zn[r], t, gn[r], ghn[r])
        if not np.isfinite(want).all():
            assert np.isnan(got[r]).all(), r
            continue
        if (zn[r] == -np.inf).all() or (t is not None and t < 0):
            assert (got[r] == 0).all(), r
            continue
        s = oracle.score(zn[r], 0)
        with np.errstate(invalid="ignore"):
            logp = zn[r] - s["max"] - s["logsum"]
        p = np.exp(logp)
        logp = np.where(p > 0, logp, 0.0)
        dp = p * (_sum_bound(V) + 6 * U * (np.abs(logp) + s["logsum"] + 1))
        mean = float((p * np.abs(logp)).sum())
        tol = abs(gn[r]) * dp + abs(ghn[r]) * (dp * np.abs(logp + s["entropy"])
                                               + p * (_sum_bound(V) * (2 + 2 * mean + s["logsum"]) + 8 * U * (np.abs(logp) + s["entropy"] + 1)))
        tol = tol + half * (1 + 1e-3) * np.abs(want) + 4 * U * abs(gn[r]) * (want != 0) * (np.arange(V) == (-1 if t is None else t)) + least
        bad = np.abs(got[r] - want) > tol
        assert not bad.any(), (r, np.flatnonzero(bad)[:5], got[r][bad][:5], want[bad][:5])


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 7), (4, 8), (6, 33), (3, 512), (7, 2049), (2, 32001), (2, 151936), (700, 130)])
def test_gradient(pkg, R, V, typ):
    import torch
    rng = np.random.default_rng(R + V)
    z = _logits(rng, R, V, typ)
    tok = rng.integers(0, V, R)
    if R > 3:
        tok[1] = -1
    g, gh = (torch.from_numpy(rng.standard_normal(R)).float().cuda() for _ in range(2))
    o = pkg.logprobs(z, _i32(tok))
    zero = torch.zeros_like(g)
    _check_grad(pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh), z, tok, g, gh)
    _check_grad(pkg.logprobs_backward(z, _i32(tok), o.stats, None, g), z, tok, g, zero)
    _check_grad(pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, None, gh), z, tok, zero, gh)
    want = pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh)
    same = pkg.logprobs_backward(z, _i32(tok), o.stats, o.entropy, g, gh, out=z)  # in the logits' own place
    assert same is z and torch.equal(same, want)


@pytest.mark.parametrize("top", [-8.5, -8.875, -9.25, -10.875])
def test_gradient_in_bf16_is_not_off_all_one_way(pkg, top):
    """A row's probabilities share one constant, whose error is all its values'.  Against the correctly rounded gradients, a value that rounds
    the other way is off by one step, 2^-7 of it or less, and values that are off by e do so with probability e 2^7 at most.
    The exponents' own rounding is at most 2^-20 (below 32), ln 2 of it in a value, and as good as independent over the row's
    different logits; the exponential may be off by 2^-22 and what the rows share by four roundings of fp32, all one way."""
    import torch
    R = V = 4096
    grid = np.arange(-255, round(top * 16) + 1) / 16  # (bf16 has them all)
    row = np.resize(grid, V)
    z = torch.from_numpy(row).to(_dtype("bf16")).cuda().repeat(R, 1)
    g = np.exp2(np.random.default_rng(12).random(R)).astype(np.float32)
    ls = np.float32(np.log(np.exp(row - top).sum()))
    stats = torch.tensor([top, ls], dtype=torch.float32, device="cuda").repeat(R, 1)
    y = pkg.logprobs_backward(z, _i32(np.zeros(R)), stats, None, torch.from_numpy(g).cuda())[:, 1:].double()
    p = torch.from_numpy(np.exp(row[1:] - top - np.float64(ls))).cuda()
    want = -torch.from_numpy(g).cuda().double()[:, None] * p
    off = float(((y - want.to(torch.bfloat16).double()) / want).mean())
    e = 2.0 ** -20 * np.log(2)
    tol = 6 * np.sqrt((e + 2.0 ** -22) * 2.0 ** -7 / y.numel()) + 6 * e / np.sqrt(3 * len(grid)) + 2.0 ** -22 + 4 * U
    assert abs(off) <= tol, (off, tol)


def test_gradient_against_differences_of_the_forward(pkg):
    # central differences of the kernel's own outputs: h = 1/4 leaves (h^2 / 6) |third derivative| and rounding / h
    import torch
    rng = np.random.default_rng(8)
    V, h = 37, 0.125
    z = _logits(rng, 1, V, "fp32", 1.0)
    g, gh = 0.8, -0.5
    o = pkg.logprobs(z, _i32([11]))
    y = pkg.logprobs_backward(z, _i32([11]), o.stats, o.entropy, torch.tensor([g], device="cuda"), torch.tensor([gh], device="cuda"))
    steps = torch.eye(V, device="cuda") * h
    up, down = (pkg.logprobs((z + s * steps).contiguous(), _i32([11] * V)) for s in (1, -1))
    f = [g * x.logprob.double() + gh * x.entropy.double() for x in (up, down)]
    diff = (f[0] - f[1]) / (2 * h)
    # third derivatives of log p and H along one logit: polynomials of p < 1 of size at most 1/2 and 1 + max |log p|
    lp = float(V)  # generous for |log p| at these logits
    bound = h * h / 6 * (0.5 * g + abs(gh) * (1 + lp)) + 64 * U / h
    assert float((diff - y[0].double()).abs().max()) <= bound


# ------------------------------------------------------------------------------------------------ together
def test_rollouts_scored_after_teacher_forcing(pkg):
    """Teacher-forced logits of the tiny policy stay on the GPU; the sampled tokens' log-probabilities, entropies and
    alternatives, then the logits' gradient of a policy loss over them, one padded row among them."""
    import ctypes

    import torch
    w = synth.WORKLOADS["tiny"]
    m, n, T = w.model, 4, 6
    weights, si = synth.model_weights(m, w.weight_seed), synth.step_inputs(w)
    cfg = pkg.model_cfg(m, max_prompts=n, max_active=n, max_seqs=n, max_prompt_len=w.prompt_len, max_gen_len=T + 1, max_k=2)
    rng = np.random.default_rng(9)
    with pkg.Handle(cfg, weights) as h:
        prompts = torch.from_numpy(np.ascontiguousarray(si.tokens[:n], np.int32)).cuda()
        forced = torch.from_numpy(rng.integers(0, m.vocab, (n, T)).astype(np.int32)).cuda()
        uid = torch.arange(n, device="cuda")
        z = torch.empty((n, T, m.vocab), device="cuda")
        tok = torch.empty((n, T), dtype=torch.int32, device="cuda")
        p = lambda x: ctypes.c_void_p(x.data_ptr())  # noqa: E731
        assert pkg.load().sara_teacher_force(h._h, n, w.prompt_len, p(prompts), T, p(forced), p(uid), 3, p(z), p(tok), 1) == 0
    z, flat = z.view(n * T, m.vocab), tok.view(-1).clone()
    flat[5] = -1
    o = pkg.logprobs(z, flat, top=4)
    t = flat.cpu().numpy()
    _check(o, z, t, 4)
    adv = torch.from_numpy(rng.standard_normal(n * T)).float().cuda()
    ent = torch.full((n * T,), 0.01, device="cuda")
    _check_grad(pkg.logprobs_backward(z, flat, o.stats, o.entropy, adv, ent), z, t, adv, ent)


def test_captured_replayed_and_on_another_stream(pkg):
    import torch
    rng = np.random.default_rng(10)
    z, tok = _logits(rng, 9, 20001, "bf16"), _i32(rng.integers(0, 20001, 9))
    g = torch.ones(9, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        o = pkg.logprobs(z, tok, top=6)
        y = pkg.logprobs_backward(z, tok, o.stats, o.entropy, g, g)
    for _ in range(3):
        z.copy_(_logits(rng, 9, 20001, "bf16", 4.0))
        tok.copy_(_i32(rng.integers(0, 20001, 9)))
        graph.replay()
        t = tok.cpu().numpy()
        _check(o, z, t, 6)
        _check_grad(y, z, t, g, g)
    with torch.cuda.stream(s):
        o2 = pkg.logprobs(z, tok, top=6)
    torch.cuda.synchronize()
    for a in ("logprob", "entropy", "stats", "top_token", "top_logprob"):  # the same bits again
        assert torch.equal(getattr(o, a), getattr(o2, a))


def test_rows_past_32_bits(pkg):
    # the last rows begin beyond 2^32 bytes
    import torch
    R, V = 15000, 151936
    z = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(11)
    z[-2:] = _logits(rng, 2, V, "bf16")
    tok = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    tok[-2:] = _i32([7, V - 1])
    o = pkg.logprobs(z, tok, top=2)
    last = pkg.LogProbs(o.logprob[-2:], o.entropy[-2:], o.stats[-2:], o.top_token[-2:], o.top_logprob[-2:])
    _check(last, z[-2:], [7, V - 1], 2)
    g = torch.ones(R, device="cuda")
    want = z[-2:].clone()
    y = pkg.logprobs_backward(z, tok, o.stats, o.entropy, g, g, out=z)
    _check_grad(y[-2:], want, [7, V - 1], g[-2:], g[-2:])
    assert float(y[:-2].abs().max()) == 0


def test_most_rows(pkg):
    # 2^31 - 1 rows, of one token each: the last group of eight is not whole
    import torch
    R = 2 ** 31 - 1
    z = torch.zeros((R, 1), dtype=torch.bfloat16, device="cuda")
    z[R - 1] = 3.0
    o = pkg.logprobs(z, None)
    # (the last row: 3 log2(e) is rounded, so its sum is an exponential of the rounding, good to 2^-21 as any: the bound of sums here.  Zeros
    # round nothing: 2^0 is 1, its logarithm 0.)
    assert o.logprob is None and float(o.stats[-1, 0]) == 3.0 and abs(float(o.stats[-1, 1])) <= _sum_bound(1) >= abs(float(o.entropy[-1]))
    for x in (o.entropy[:-1], o.stats[:-1].view(-1)):
        for a in range(0, x.numel(), 1 << 29):
            assert not bool(x[a:a + (1 << 29)].any())


def test_largest_vocabulary(pkg):
    # token ids up to 2^31 - 2
    import torch
    V = 2 ** 31 - 1
    z = torch.full((1, V), -30.0, dtype=torch.bfloat16, device="cuda")
    z[0, V - 1], z[0, 2 ** 30], z[0, 5] = 10.0, 9.0, 8.0
    o = pkg.logprobs(z, _i32([V - 1]), top=4)
    assert o.top_token[0].tolist() == [V - 1, 2 ** 30, 5, 0]
    S = 1 + np.exp(-1.0) + np.exp(-2.0) + (V - 3) * np.exp(-40.0)
    assert abs(float(o.logprob[0]) + np.log(S)) < 1e-5
    g = torch.ones(1, device="cuda")
    y = pkg.logprobs_backward(z, _i32([V - 1]), o.stats, o.entropy, g, out=z)
    assert abs(float(y[0, V - 1]) - (1 - 1 / S)) <= 2.0 ** -8 and abs(float(y[0, 5]) + np.exp(-2) / S) <= 2.0 ** -8 * 0.2
