"""Log-probabilities and entropies from hidden states, and their gradients, on the GPU against the 64-bit oracle, within bounds that
follow from the arithmetic: exact products summed in fp32, dz rounded to the operands' type, one rounding of the results."""
import numpy as np
import pytest

import synth
from oracle import scoring as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"bf16": 2.0 ** -126, "fp16": 2.0 ** -25}


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    p.load()
    return p


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _f32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.float32, device="cuda")


def _inputs(rng, R, d, V, typ, std=2.0):
    """Hidden states N(0, 1) and weights that make logits of spread `std`, on the GPU."""
    import torch
    h = torch.from_numpy(rng.standard_normal((R, d))).cuda().to(_dtype(typ))
    w = torch.from_numpy(rng.standard_normal((V, d)) * (std / np.sqrt(d))).cuda().to(_dtype(typ))
    return h, w


def _np(x):
    return x.double().cpu().numpy()


def _chain(n):
    # relative to the sum of magnitudes: the tensor core adds 16 products at a time and cuts, a step of fp32 each, and a few more inside
    return (n / 16 + 8) * 2 * U


def _logit_error(h, w, scale):
    """Bound on a row's logits' errors, the largest over the vocabulary."""
    a = scale * (np.abs(h) @ np.abs(w).T).max(1)
    return a * (_chain(h.shape[1]) + 2 * U)


def _sum_error(V):
    return (V / 256 + 300) * U  # tiles of 256 in a chain, tiles joined by fewer steps than there are; terms good to 2^-21


def _check(o, h, w, tokens, scale):
    hn, wn = _np(h), _np(w)
    live = np.ones(len(hn), bool) if tokens is None else np.asarray(tokens) >= 0
    want, z = oracle.linear(np.where(live[:, None], hn, 0), wn, tokens, scale)
    e = _logit_error(np.where(live[:, None], hn, 0), wn, scale)
    lp, H, st = None if o.logprob is None else _np(o.logprob), _np(o.entropy), _np(o.stats)
    for r, s in enumerate(want):
        if not live[r]:
            assert (lp is None or lp[r] == 0) and H[r] == 0 and (st[r] == 0).all(), r
            continue
        b = _sum_error(len(wn)) + 2 * e[r]
        if lp is not None:
            if np.isnan(s["logprob"]):
                assert np.isnan(lp[r]), r
            else:
                assert abs(lp[r] - s["logprob"]) <= b + 4 * U * (abs(s["logprob"]) + s["logsum"] + 1), (r, lp[r], s)
        if np.isnan(s["entropy"]):
            assert np.isnan(H[r]) and np.isnan(st[r, 1]), r
            continue
        dist = s["max"] - z[r]
        mean = float((np.exp(-dist) * dist).sum() / np.exp(-dist).sum())
        assert abs(H[r] - s["entropy"]) <= (b + 4 * U) * (2 + 2 * mean + s["logsum"]), (r, H[r], s)
        assert abs(st[r, 0] - s["max"]) <= e[r] + 2 * U * abs(s["max"]) and abs(st[r, 1] - s["logsum"]) <= b + 2 * U * s["logsum"], (r, st[r], s)


def _check_grad(got, h, w, tokens, g, gh, scale, typ, spread=True):
    """spread: inputs as of _inputs, whose errors add up as independent ones do; bounds by magnitudes hold for any."""
    hn, wn, gn, ghn = _np(h), _np(w), _np(g), _np(gh)
    live = np.ones(len(hn), bool) if tokens is None else np.asarray(tokens) >= 0
    dh, dw, dz = oracle.linear_grad(hn, wn, tokens, gn, ghn, scale)
    h0 = np.where(live[:, None], hn, 0)
    wrong = np.isnan(dz).any(1)
    e = 2 * _logit_error(h0, wn, scale) + _sum_error(len(wn))
    ok = ~wrong
    # dz's error: p's (2 e and the exponential's), that of log p + H where it counts, one rounding to the type
    z = scale * (h0 @ wn.T)
    lp = z - z.max(1, keepdims=True)
    lp -= np.log(np.exp(lp).sum(1, keepdims=True))
    H = -(np.exp(lp) * lp).sum(1, keepdims=True)
    near = (e[:, None] + 8 * U * (np.abs(lp) + 1)) * np.exp(lp) * (np.abs(gn)[:, None] + np.abs(ghn)[:, None] * (np.abs(lp + H) + 2 + H))
    near = near + 4 * U * np.abs(dz) + 4 * U * np.abs(gn)[:, None] * (np.arange(len(wn)) == (np.asarray(tokens) if tokens is not None else np.full(len(hn), -1))[:, None])
    err = np.where(live[:, None], near + HALF[typ] * np.abs(dz), 0)
    if typ == "fp16":  # a row's dz below 2^-27 of its largest possible: half a step of fp16 there
        err += np.where(live, 2.0 ** -25 * 2.0 ** -12 * (np.abs(gn) + 16 * np.abs(ghn)), 0)[:, None]
    if got[0] is not None:
        y = _np(got[0])
        assert (y[~live] == 0).all() and np.isnan(y[wrong]).all()
        mag = scale * (np.abs(dz) @ np.abs(wn))
        tol = scale * (err @ np.abs(wn)) + (_chain(len(wn)) + 40 * U) * mag + HALF[typ] * (1 + 1e-3) * np.abs(dh) + LEAST[typ]
        if len(wn) > 0:
            bad = np.abs(y - dh)[ok] > tol[ok]
            assert not bad.any(), (np.argwhere(bad)[:5], y[ok][bad][:5], dh[ok][bad][:5], tol[ok][bad][:5])
        if spread and typ == "bf16" and dh[ok].size > 1000 and np.linalg.norm(dh[ok]):
            assert np.linalg.norm(y[ok] - dh[ok]) <= 1.5 * HALF[typ] * np.linalg.norm(dh[ok])
    if got[1] is not None:
        y = _np(got[1])
        if wrong.any():
            assert np.isnan(y).all()
            return
        low = 0.0
        if typ == "fp16":  # rows lowered by more than 14 powers of two lose bits: half a step of fp16 times what their dz was raised to
            b = np.abs(gn) + 16 * np.abs(ghn)
            low = scale * 2.0 ** -25 * len(hn) * b[live].max() if live.any() else 0.0
        mag = scale * (np.abs(dz).T @ np.abs(h0))
        tol = scale * (err.T @ np.abs(h0)) + (_chain(len(hn)) + 40 * U) * mag + HALF[typ] * (1 + 1e-3) * np.abs(dw) + LEAST[typ] + low
        bad = np.abs(y - dw) > tol
        assert not bad.any(), (np.argwhere(bad)[:5], y[bad][:5], dw[bad][:5], tol[bad][:5])
        if spread and typ == "bf16" and dw.size > 1000 and np.linalg.norm(dw):
            assert np.linalg.norm(y - dw) <= 1.5 * HALF[typ] * np.linalg.norm(dw)


def _both(pkg, h, w, tok, scale, g, gh, typ, spread=True):
    t = None if tok is None else _i32(tok)
    o = pkg.linear_logprobs(h, w, t, scale=scale)
    _check(o, h, w, tok, scale)
    y = pkg.linear_logprobs_backward(h, w, t, o.stats, o.entropy, g if tok is not None else None, gh, scale=scale)
    _check_grad(y, h, w, tok, g if tok is not None else 0 * g, gh, scale, typ, spread)
    return o, y


# rows and tokens around tiles, dims around chunks of 64 and tiles of 256, from the smallest on
@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,d,V", [(1, 8, 1), (1, 64, 256), (2, 72, 3), (5, 16, 255), (31, 128, 512), (32, 200, 257), (127, 256, 700), (128, 264, 1024),
                                   (129, 64, 300), (130, 320, 2001), (255, 520, 513), (256, 1536, 400), (257, 8, 3000), (640, 136, 1111)])
def test_sizes(pkg, R, d, V, typ):
    rng = np.random.default_rng(R + d + V)
    h, w = _inputs(rng, R, d, V, typ)
    tok = rng.integers(0, V, R)
    if R > 3:
        tok[1::7] = -1
    _both(pkg, h, w, tok, [1.0, 1.25, 0.3][R % 3], _f32(rng.standard_normal(R)), _f32(0.1 * rng.standard_normal(R)), typ)


# several pieces of the vocabulary, dH in several parts; the last piece and its parts are shorter
@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,d,V", [(3, 64, 16384), (40, 72, 33000), (200, 128, 40001), (300, 264, 16385)])
def test_pieces(pkg, R, d, V, typ):
    rng = np.random.default_rng(V)
    h, w = _inputs(rng, R, d, V, typ, 3.0)
    tok = rng.integers(0, V, R)
    tok[0] = V - 1
    _both(pkg, h, w, tok, 1.0, _f32(rng.standard_normal(R)), _f32(0.1 * rng.standard_normal(R)), typ)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R", [9, 400])
def test_rows_of_padding(pkg, R, typ):
    import torch
    rng = np.random.default_rng(R)
    h, w = _inputs(rng, R, 96, 1500, typ)
    g, gh = _f32(rng.standard_normal(R)), _f32(rng.standard_normal(R))
    tok = rng.integers(0, 1500, R)
    tok[rng.random(R) < 0.5] = -1
    tok[0] = -7
    dead = _i32(tok) < 0
    h[dead] = torch.tensor([np.nan, np.inf, -np.inf] * 32, device="cuda").to(h.dtype)  # (what they hold does not matter)
    g[dead], gh[dead] = np.nan, np.inf
    o = pkg.linear_logprobs(h, w, _i32(tok))
    _check(o, h, w, tok, 1.0)
    y = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    _check_grad(y, h, w, tok, g.nan_to_num(0, 0, 0), gh.nan_to_num(0, 0, 0), 1.0, typ)
    tok[:] = -1  # nothing but padding
    o = pkg.linear_logprobs(h, w, _i32(tok))
    _check(o, h, w, tok, 1.0)
    a, b = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    assert not a.any() and not b.any()


def test_no_rows(pkg):
    import torch
    w = torch.ones((50, 16), dtype=torch.bfloat16, device="cuda")
    h, none = w[:0], _i32([])
    o = pkg.linear_logprobs(h, w, none)
    assert o.logprob.shape == (0,) and o.stats.shape == (0, 2)
    a, b = pkg.linear_logprobs_backward(h, w, none, o.stats, o.entropy, o.logprob)
    assert a.shape == (0, 16) and b.shape == (50, 16) and not b.any()


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R", [6, 300])
def test_wrong_tokens_no_tokens_and_infinite_logits(pkg, R, typ):
    import torch
    rng = np.random.default_rng(4)
    h, w = _inputs(rng, R, 64, 900, typ)
    g, gh = _f32(rng.standard_normal(R)), _f32(rng.standard_normal(R))
    tok = rng.integers(0, 900, R)
    _both(pkg, h, w, None, 1.0, g, gh, typ)
    tok[1], tok[3] = 900, 2 ** 31 - 1
    _both(pkg, h, w, tok, 1.0, g, gh, typ)
    tok[1], tok[3] = -1, 5
    h[4, 7] = np.nan
    _both(pkg, h, w, tok, 1.0, g, gh, typ)
    h[4, 7] = np.inf  # logits of either sign
    o = pkg.linear_logprobs(h, w, _i32(tok))
    assert o.logprob.isnan().tolist() == o.entropy.isnan().tolist() == [r == 4 for r in range(R)]
    a, b = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    assert a.isnan().any(1).tolist() == [r == 4 for r in range(R)] and bool(b.isnan().all())
    # a token that is nobody's: its weights at -inf for hidden states above 0
    h = h.abs().nan_to_num(1, 1, 1)
    w[100] = -np.inf
    tok[4] = 100
    o = pkg.linear_logprobs(h, w, _i32(tok))
    keep = torch.tensor([v for v in range(900) if v != 100], device="cuda")
    without = pkg.linear_logprobs(h, w[keep].contiguous(), None)
    live = _i32(tok) >= 0
    assert float(o.logprob[4]) == -np.inf and torch.allclose(o.entropy[live], without.entropy[live], rtol=0, atol=1e-4)


def test_large_and_peaked_logits(pkg):
    # logits of thousands, one token far above the others, all alike
    import torch
    rng = np.random.default_rng(5)
    for std in (3000.0, 40.0, 1e-4):
        h, w = _inputs(rng, 140, 64, 1300, "bf16", std)
        _both(pkg, h, w, rng.integers(0, 1300, 140), 1.0, _f32(rng.standard_normal(140)), _f32(0.1 * rng.standard_normal(140)), "bf16", spread=False)
    h, w = _inputs(rng, 10, 64, 1300, "bf16", 0.0)
    o = pkg.linear_logprobs(h, w, _i32(rng.integers(0, 1300, 10)))
    assert torch.allclose(o.entropy, torch.full_like(o.entropy, np.log(1300)), rtol=4e-6)


def test_gradients_of_very_different_rows_in_fp16(pkg):
    # a row's gradient keeps its bits however small its weight beside other rows'
    rng = np.random.default_rng(6)
    R = 150
    h, w = _inputs(rng, R, 64, 2000, "fp16")
    tok = rng.integers(0, 2000, R)
    g = rng.standard_normal(R) * 2.0 ** rng.integers(-30, 30, R)
    g[3], g[5] = 0, 1e-35
    gh = np.where(rng.random(R) < 0.5, 0, g * 0.1)
    o = pkg.linear_logprobs(h, w, _i32(tok))
    dh, _ = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, _f32(g), _f32(gh), scale=1.0, grad_weight=False)
    k = np.abs(g) < 2.0 ** 14  # (the others' results pass fp16)
    want = oracle.linear_grad(_np(h), _np(w), tok, g.astype(np.float32).astype(np.float64), gh.astype(np.float32).astype(np.float64))[0]
    y = _np(dh)
    for r in np.flatnonzero(k):
        assert np.linalg.norm(y[r] - want[r]) <= 2 * HALF["fp16"] * np.linalg.norm(want[r]) + 8 * LEAST["fp16"] * 2, r


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R", [50, 200])
def test_strided_rows_and_given_outputs(pkg, R, typ):
    import torch
    rng = np.random.default_rng(7)
    big_h, big_w = _inputs(rng, R, 160, 777, typ)
    h, w = big_h[:, 8:136], big_w[:, 16:144]
    tok, g, gh = rng.integers(0, 777, R), _f32(rng.standard_normal(R)), _f32(rng.standard_normal(R))
    o = pkg.linear_logprobs(h, w, _i32(tok))
    _check(o, h, w, tok, 1.0)
    oh, ow = (torch.full_like(x, 7.0) for x in (big_h, big_w))
    same = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh, grad_hidden=oh[:, 24:152], grad_weight=ow[:, 32:])
    _check_grad(same, h, w, tok, g, gh, 1.0, typ)
    assert (oh[:, :24] == 7).all() and (oh[:, 152:] == 7).all() and (ow[:, :32] == 7).all()
    for wanted in ((True, False), (False, True)):
        y = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh, grad_hidden=wanted[0], grad_weight=wanted[1])
        assert [x is not None for x in y] == list(wanted)
        for a, b in zip(y, same):
            assert a is None or torch.equal(a, b)


def test_each_weight_alone(pkg):
    import torch
    rng = np.random.default_rng(8)
    h, w = _inputs(rng, 20, 64, 400, "bf16")
    tok, g = rng.integers(0, 400, 20), _f32(rng.standard_normal(20))
    o = pkg.linear_logprobs(h, w, _i32(tok))
    zero = torch.zeros_like(g)
    _check_grad(pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, None, g), h, w, tok, g, zero, 1.0, "bf16")
    _check_grad(pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, None, g), h, w, tok, zero, g, 1.0, "bf16")
    a, b = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, None)
    assert not a.any() and not b.any()


def test_gradient_against_differences_of_the_forward(pkg):
    # steps of the weights and hidden states that bf16 holds exactly: h = 2^-4 leaves (h^2 / 6) |third derivative| and rounding / h
    import torch
    rng = np.random.default_rng(9)
    h = torch.from_numpy(rng.integers(-8, 9, (2, 8)) / 8).cuda().bfloat16()
    w = torch.from_numpy(rng.integers(-8, 9, (5, 8)) / 8).cuda().bfloat16()
    tok, g, gh, step = _i32([1, 4]), _f32([0.75, -0.5]), _f32([0.25, 0.5]), 2.0 ** -4

    def f(h, w):
        o = pkg.linear_logprobs(h, w, tok)
        return float((g.double() * o.logprob.double() + gh.double() * o.entropy.double()).sum())

    o = pkg.linear_logprobs(h, w, tok)
    dh, dw = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g, gh)
    for x, dx, at in ((h, dh, (1, 3)), (h, dh, (0, 0)), (w, dw, (4, 2)), (w, dw, (0, 7))):
        was = x[at].clone()
        x[at] = was + step
        up = f(h, w)
        x[at] = was - step
        down = f(h, w)
        x[at] = was
        # third derivatives along one weight: at most the rows' number times |h|^3 <= 1 times polynomials of p of size 1/2 and 1 + |log p|
        bound = step * step / 6 * (1.25 * 0.5 + 0.75 * (1 + 20)) + 200 * U / step + 3 * HALF["bf16"] * 2
        assert abs((up - down) / (2 * step) - float(dx[at])) <= bound


def test_same_bits_again_on_another_stream_and_captured(pkg):
    import torch
    rng = np.random.default_rng(10)
    R, d, V = 300, 128, 20001
    h, w = _inputs(rng, R, d, V, "bf16")
    tok, g = _i32(rng.integers(-1, V, R)), _f32(rng.standard_normal(R))
    ws, wsb = pkg.linear_logprobs_workspace(R, d, V), pkg.linear_logprobs_workspace(R, d, V, backward=True)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    pkg.linear_logprobs(h, w, tok, workspace=ws)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        o = pkg.linear_logprobs(h, w, tok, workspace=ws)
        y = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g, g, workspace=wsb)
    for _ in range(3):
        h.copy_(_inputs(rng, R, d, 1, "bf16")[0])
        tok.copy_(_i32(rng.integers(-1, V, R)))
        graph.replay()
        with torch.cuda.stream(s):
            o2 = pkg.linear_logprobs(h, w, tok)
            y2 = pkg.linear_logprobs_backward(h, w, tok, o2.stats, o2.entropy, g, g)
        torch.cuda.synchronize()
        for a in ("logprob", "entropy", "stats"):
            assert torch.equal(getattr(o, a), getattr(o2, a))
        assert torch.equal(y[0], y2[0]) and torch.equal(y[1], y2[1])
    _check(o, h, w, tok.cpu().numpy(), 1.0)


def test_workspace_too_small_or_elsewhere(pkg):
    import torch
    h, w = _inputs(np.random.default_rng(11), 200, 64, 600, "bf16")
    tok = _i32(np.zeros(200))
    ws = pkg.linear_logprobs_workspace(200, 64, 600)
    for bad in (ws[:-256], ws[1:], ws.cpu()):
        with pytest.raises(pkg.SaraError):
            pkg.linear_logprobs(h, w, tok, workspace=bad)
    o = pkg.linear_logprobs(h, w, tok, workspace=ws)
    with pytest.raises(pkg.SaraError):  # (in the operand's place)
        pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, o.logprob, grad_hidden=h)
    with pytest.raises(pkg.SaraError):
        pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, o.logprob, grad_weight=w)
    assert not torch.isnan(o.logprob).any()


def test_alike_with_scores_of_stored_logits(pkg):
    """The policy loss of a tiny model's rollouts, by way of the logits and without them."""
    import torch
    m = synth.WORKLOADS["tiny"].model
    rng = np.random.default_rng(12)
    R = 48
    h, w = _inputs(rng, R, m.d_model, m.vocab, "bf16", 3.0)
    z = h.float() @ w.float().t()  # exact products, sums of 128 of them in fp32
    tok = _i32(rng.integers(-1, m.vocab, R))
    a, b = pkg.logprobs(z, tok), pkg.linear_logprobs(h, w, tok)
    e = 2 * float(_logit_error(_np(h), _np(w), 1.0).max()) * 2 + 2 * _sum_error(m.vocab)
    assert float((a.logprob - b.logprob).abs().max()) <= e and float((a.entropy - b.entropy).abs().max()) <= 20 * e
    adv = _f32(rng.standard_normal(R))
    dz = pkg.logprobs_backward(z, tok, a.stats, a.entropy, adv, adv).double()
    dh, dw = pkg.linear_logprobs_backward(h, w, tok, b.stats, b.entropy, adv, adv)
    assert float((dh.double() - dz @ w.double()).norm()) <= 1.5 * HALF["bf16"] * float((dz @ w.double()).norm())
    assert float((dw.double() - dz.t() @ h.double()).norm()) <= 1.5 * HALF["bf16"] * float((dz.t() @ h.double()).norm())


def test_weights_past_32_bits(pkg):
    # the last tokens' weights, and their gradients, begin beyond 2^32 bytes
    import torch
    V, d = 2 ** 19 + 300, 4352
    h = torch.full((2, d), 2.0 ** -6, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    w[V - 1] = 0.25   # logit 17
    w[5] = 0.125      # 8.5
    tok = _i32([V - 1, 5])
    o = pkg.linear_logprobs(h, w, tok)
    S = 1 + np.exp(-8.5) + (V - 2) * np.exp(-17.0)
    assert abs(float(o.logprob[0]) + np.log(S)) < 1e-4 and abs(float(o.logprob[1]) + 8.5 + np.log(S)) < 1e-4
    g = _f32([1.0, 0.0])
    dh, dw = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g)
    p = 1 / S
    assert abs(float(dw[V - 1, d - 1]) - (1 - p) * 2.0 ** -6) <= 2.0 ** -6 * 2.0 ** -7 * (1 - p) + 1e-9
    assert abs(float(dw[V - 2, 0]) + p * np.exp(-17.0) * 2.0 ** -6) <= 2.0 ** -7 * p * np.exp(-17.0) * 2.0 ** -6
    want = (1 - p) * 0.25 - p * np.exp(-8.5) * 0.125
    assert abs(float(dh[0, 0]) - want) <= 2.0 ** -6 * abs(want) and float(dh[1].abs().max()) == 0


def test_a_single_row_has_no_stride(pkg):
    """One row of a matrix whose rows are no multiple of 8 elements apart, and one token of a vocabulary."""
    import torch
    rng = np.random.default_rng(12)
    h = torch.from_numpy(rng.standard_normal((9, 100))).cuda().bfloat16()[8:9, 32:96]  # (8 x 200 + 64 bytes: aligned)
    for w in (torch.from_numpy(rng.standard_normal((300, 64))).cuda().bfloat16(), torch.from_numpy(rng.standard_normal((9, 100))).cuda().bfloat16()[8:9, 32:96]):
        g = torch.ones(1, device="cuda")
        _both(pkg, h, w, [0], 1.0, g, g, "bf16", spread=False)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,d,V,logit", [(1, 944, 3000, 12), (1, 1464, 32570, 22), (2, 96, 513, 9), (200, 512, 2000, 18), (129, 2048, 700, 30)])
def test_gradients_of_tokens_that_are_nearly_certain(pkg, R, d, V, logit, typ):
    """1 - p of 1e-2 to 1e-10: the whole gradient hangs on it.  A row's error: one rounding of each dz but the token's and of the result, the logits'
    errors (2^-24 of them a step of 16 products, and what the formula adds) in the exponents of the others, and twice the same for 1 - p."""
    import torch
    rng = np.random.default_rng(R + d)
    h = torch.from_numpy(rng.standard_normal((R, d))).cuda().to(_dtype(typ))
    w = torch.from_numpy(rng.standard_normal((V, d)) / np.sqrt(d)).cuda().to(_dtype(typ))
    tok = rng.permutation(V)[:R]
    for r in range(R):
        w[tok[r]] = (h[r].double() * (logit / float((h[r].double() ** 2).sum()))).to(w.dtype)
    t = _i32(tok)
    o = pkg.linear_logprobs(h, w, t)
    g, gh = torch.from_numpy(rng.standard_normal(R)).float().cuda(), torch.from_numpy(rng.standard_normal(R)).float().cuda() / 64
    got, _ = pkg.linear_logprobs_backward(h, w, t, o.stats, o.entropy, g, gh)
    want, _, dz = oracle.linear_grad(_np(h), _np(w), tok, _np(g), _np(gh))
    size, mag = np.abs(_np(h) @ _np(w).T).max(1, keepdims=True), np.abs(dz) @ np.abs(_np(w))
    tol = (2 * HALF[typ] + 4 * (d / 16 + 16) * U * (size + 1) + 1e-4) * mag + LEAST[typ]
    b, wn = np.abs(_np(g)) + 16 * np.abs(_np(gh)), np.abs(_np(w))
    if typ == "fp16":  # dz below 2^-27 of a row's largest possible: half a step of fp16 there, as _check_grad has it
        tol += (2.0 ** -25 * 2.0 ** -12 * b)[:, None] * wn.sum(0)
    if R > 128:  # the sum beside the maximum's 1: 64 terms in a chain that it is one of, 66 roundings of 2^-24, in log S and in the entropy
        tol += (66 * U * (np.abs(_np(g)) + 2 * np.abs(_np(gh))))[:, None] * wn[tok]
    assert (np.abs(_np(got) - want) <= tol).all(), np.max(np.abs(_np(got) - want) / tol)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,V,how", [(1023, 300, "any"), (1024, 300, "any"), (1025, 300, "any"), (700, 40, "same"), (1500, 600, "few"), (90, 513, "last"), (2000, 512, "wide")])
def test_rows_found_and_sorted_by_token(pkg, R, V, how, typ):
    """Row counts around what a CTA finds for itself, and many rows to a token: its corrections come from more rows than wait in shared memory."""
    import torch
    rng = np.random.default_rng(R)
    d = 328 if how == "wide" else 64
    h = torch.from_numpy(rng.standard_normal((R, d))).cuda().to(_dtype(typ))
    w = torch.from_numpy(rng.standard_normal((V, d)) / np.sqrt(d)).cuda().to(_dtype(typ))
    tok = {"any": rng.integers(0, V, R), "same": np.full(R, 7), "few": rng.integers(250, 260, R), "last": np.full(R, V - 1), "wide": rng.integers(0, V, R)}[how]
    tok[rng.random(R) < 0.2] = -1
    g, gh = (torch.from_numpy(rng.standard_normal(R)).float().cuda() for _ in range(2))
    _, y = _both(pkg, h, w, tok, 1.0, g, gh, typ, spread=False)
    o = pkg.linear_logprobs(h, w, _i32(tok))
    again = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    assert torch.equal(y[0], again[0]) and torch.equal(y[1], again[1])


def _weights_bound(h, w, tok, g, gh, dz, want):
    """What dW may be off by in fp16 (scale 1): dz by what _check_grad has (its exponents, one rounding but at the row's token, half a step of fp16 below 2^-27 of
    the row's largest possible b = |g| + 16 |g'|), sums of R products in fp32, one rounding of the result; and rows whose b max|h| is far below the
    largest's lose bits of h: 2^-38 of the largest b max|h|, times dz / b."""
    hn, wn, gn, ghn = np.abs(_np(h)), _np(w), np.abs(_np(g))[:, None], np.abs(_np(gh))[:, None]
    z = _np(h) @ wn.T
    lp = z - z.max(1, keepdims=True)
    lp -= np.log(np.exp(lp).sum(1, keepdims=True))
    H = -(np.exp(lp) * lp).sum(1, keepdims=True)
    e = (2 * _logit_error(_np(h), wn, 1.0) + _sum_error(len(wn)))[:, None]
    b, own = gn + 16 * ghn, np.arange(len(wn)) == np.asarray(tok)[:, None]
    err = (e + 8 * U * (np.abs(lp) + 1)) * np.exp(lp) * (gn + ghn * (np.abs(lp + H) + 2 + H)) + 4 * U * np.abs(dz) + 4 * U * gn * own
    err += np.where(own, 0, HALF["fp16"] * np.abs(dz)) + 2.0 ** -25 * 2.0 ** -12 * b
    err += HALF["fp16"] ** 2 * np.abs(dz)
    low = 2.0 ** -38 * (b[:, 0] * hn.max(1)).max() * (np.abs(dz) / np.maximum(b, 1e-300)).sum(0)
    return err.T @ hn + (_chain(len(hn)) + 40 * U) * (np.abs(dz).T @ hn) + HALF["fp16"] * (1 + 1e-3) * np.abs(want) + LEAST["fp16"] + low[:, None]


@pytest.mark.parametrize("R,up,down,big", [(40, 10, -10, 1.0), (300, 12, -12, 1.0), (40, 3, -3, 2.0 ** -10), (200, 14, -14, 1.0), (60, 0, -9, 2.0 ** 5)])
def test_weights_gradient_of_rows_of_small_weight_in_fp16(pkg, R, up, down, big):
    """Rows of small weight beside rows of large weight, whose hidden states have other dims: dW's there is well within fp16, and keeps its bits."""
    import torch
    rng = np.random.default_rng(R)
    d, V = 128, 900
    large = np.arange(R) % 2 == 0
    h, w = rng.standard_normal((R, d)) * big, rng.standard_normal((V, d)) * (2 / np.sqrt(d)) / big
    h[large, d // 2:], h[~large, :d // 2] = 0, 0
    tok = rng.integers(0, V, R)
    h, w = torch.from_numpy(h).cuda().half(), torch.from_numpy(w).cuda().half()
    size = np.where(large, 2.0 ** up, 2.0 ** down)
    g, gh = _f32(rng.choice([-1, 1], R) * size * (0.5 + rng.random(R))), _f32(rng.standard_normal(R) * size / 64)
    o = pkg.linear_logprobs(h, w, _i32(tok))
    _, dw = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    _, want, dz = oracle.linear_grad(_np(h), _np(w), tok, _np(g), _np(gh))
    tol = _weights_bound(h, w, tok, g, gh, dz, want)
    bad = (np.abs(_np(dw) - want) > tol) & (np.abs(want) < 65504)
    assert not bad.any(), np.max(np.abs(_np(dw) - want)[bad] / tol[bad])


def test_weights_gradient_of_very_different_rows_in_fp16(pkg):
    """Weights over 2^-30 .. 2^14, some of them 0, hidden states of very different sizes, some of them 0 too."""
    import torch
    rng = np.random.default_rng(16)
    for R in (90, 250):
        d, V = 64, 700
        h = rng.standard_normal((R, d)) * 2.0 ** rng.integers(-8, 3, R)[:, None]
        h[3], h[5], h[R - 2] = 60000.0, 0, 2.0 ** -24  # (the first of no weight)
        h, w = torch.from_numpy(h).cuda().half(), torch.from_numpy(rng.standard_normal((V, d)) / np.sqrt(d)).cuda().half()
        tok = rng.integers(0, V, R)
        tok[4] = -1
        g = rng.standard_normal(R) * 2.0 ** rng.integers(-30, 15, R)
        g[3], g[7], g[8] = 0, 1e-35, -1e-40
        gh = np.where(rng.random(R) < 0.5, 0, g * 0.1)
        g[4] = 2.0 ** 100  # (padding)
        o = pkg.linear_logprobs(h, w, _i32(tok))
        for size in (1.0, 2.0 ** -20):
            gs, ghs = _f32(g * size), _f32(gh * size)
            _, dw = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, gs, ghs)
            h0 = h.clone()
            h0[4], gs[4], ghs[4] = 0, 0, 0
            _, want, dz = oracle.linear_grad(_np(h0), _np(w), tok, _np(gs), _np(ghs))
            tol = _weights_bound(h0, w, tok, gs, ghs, dz, want)
            bad = (np.abs(_np(dw) - want) > tol) & (np.abs(want) < 60000)
            assert not bad.any(), np.max(np.abs(_np(dw) - want)[bad] / tol[bad])


def test_weights_gradient_does_not_depend_on_calls_before(pkg):
    """One workspace for rows of large weight and of small, in fp16: what a call finds of its rows is not left for the next."""
    import torch
    rng = np.random.default_rng(17)
    R, d, V = 64, 64, 300
    h, w = _inputs(rng, R, d, V, "fp16")
    tok, g = _i32(rng.integers(0, V, R)), _f32(rng.standard_normal(R))
    o = pkg.linear_logprobs(h, w, tok)
    fresh = lambda k: pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g * k, None)  # noqa: E731
    ws = pkg.linear_logprobs_workspace(R, d, V, backward=True)
    for k in (1.0, 2.0 ** 12, 2.0 ** -12, 1.0, 0.0, 2.0 ** -6):
        a, b = fresh(k), pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g * k, None, workspace=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), k


def test_two_likely_tokens_in_fp16(pkg):
    """Logits of 100 and 46 steps of 2^-15 less, exact in fp32 whatever the order: 1 - p of either depends on the difference.  The gradient's first half
    of dims is the first token's, the other half the second's.  Bound: the result's rounding, and 300 steps of fp32 in log S and in exponents."""
    import torch
    d, V = 4096, 300
    for R in (3, 200):
        h = torch.ones((R, d), dtype=torch.float16, device="cuda")
        w = torch.zeros((V, d), dtype=torch.float16, device="cuda")
        w[17, :d // 2], w[250, d // 2:] = 100 / 2048, 100 / 2048
        w[250, d // 2:d // 2 + 46] -= 2.0 ** -15
        for t in (17, 250):
            tok, g = np.full(R, t), _f32(np.ones(R))
            o = pkg.linear_logprobs(h, w, _i32(tok))
            dh, _ = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, grad_weight=False)
            want, _, dz = oracle.linear_grad(_np(h), _np(w), tok, np.ones(R), np.zeros(R))
            own = _np(w)[t][None] != 0  # the other token's dz is rounded to fp16
            tol = (HALF["fp16"] * np.where(own, 1, 2) + 300 * U) * np.abs(want) + LEAST["fp16"]
            assert (np.abs(_np(dh) - want) <= tol).all(), (R, t, np.max(np.abs(_np(dh) - want) / tol))


@pytest.mark.parametrize("R", [4, 256])
def test_logits_of_long_hidden_states_in_bf16(pkg, R):
    """65,536 products of one sign to a logit of 36, which two tokens have: the probability of each is 1/2, and the gradient of a third is minus the weights of
    either, exactly.  An error of p of 1/512 shows; parts of 2,048 products lose at most 2^-15 of the logit, 1.1e-3."""
    import torch
    rng = np.random.default_rng(13)
    d, V = 65536, 300
    h = torch.from_numpy(rng.integers(128, 256, d) * 2.0 ** -7).cuda().bfloat16().repeat(R, 1)
    w = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    w[3] = torch.from_numpy(rng.integers(128, 256, d) * 2.0 ** -19).cuda().bfloat16()
    w[7] = w[3]
    z = float((h[0].double() * w[3].double()).sum())
    assert 35 < z < 37
    tok, g = _i32(np.full(R, 100)), _f32(np.ones(R))
    o = pkg.linear_logprobs(h, w, tok)
    assert abs(float(o.logprob[0]) + z + np.log(2)) < 1e-3
    dh, dw = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g)
    assert torch.equal(dh, -w[3].expand(R, d)), float((dh.float() / w[3].float()).mean())
    assert torch.equal(dw[3], -R / 2 * h[0]) and torch.equal(dw[7], dw[3])


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,d,V,logit", [(3, 4096, 3000, 17), (2, 8192, 2000, 33), (200, 8192, 900, 17), (130, 4096, 700, 34), (1, 2048, 5000, 16.5)])
def test_gradients_of_nearly_certain_tokens_of_long_hidden_states(pkg, R, d, V, logit, typ):
    """Logits next to a power of two, of products of one sign: the sums that the gradient makes again lose the most there."""
    test_gradients_of_tokens_that_are_nearly_certain(pkg, R, d, V, logit, typ)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("R,d,V,logit", [(140, 1024, 2000, 17), (200, 4096, 900, 20)])
def test_scores_in_small_batches_gradients_in_one(pkg, R, d, V, logit, typ):
    """Few rows' logits are summed in other parts than many rows': 1 - p of nearly certain tokens, from the scores of a few rows at a time.  Bounds as in
    test_gradients_of_tokens_that_are_nearly_certain for up to 128 rows."""
    import torch
    rng = np.random.default_rng(R + d)
    h = torch.from_numpy(rng.standard_normal((R, d))).cuda().to(_dtype(typ))
    w = torch.from_numpy(rng.standard_normal((V, d)) / np.sqrt(d)).cuda().to(_dtype(typ))
    tok = rng.permutation(V)[:R]
    for r in range(R):
        w[tok[r]] = (h[r].double() * (logit / float((h[r].double() ** 2).sum()))).to(w.dtype)
    t, step = _i32(tok), 20
    o = [pkg.linear_logprobs(h[a:a + step], w, t[a:a + step]) for a in range(0, R, step)]
    stats, entropy = torch.cat([x.stats for x in o]), torch.cat([x.entropy for x in o])
    g, gh = torch.from_numpy(rng.standard_normal(R)).float().cuda(), torch.from_numpy(rng.standard_normal(R)).float().cuda() / 64
    got, _ = pkg.linear_logprobs_backward(h, w, t, stats, entropy, g, gh)
    want, _, dz = oracle.linear_grad(_np(h), _np(w), tok, _np(g), _np(gh))
    size, mag = np.abs(_np(h) @ _np(w).T).max(1, keepdims=True), np.abs(dz) @ np.abs(_np(w))
    tol = (2 * HALF[typ] + 4 * (d / 16 + 16) * U * (size + 1) + 1e-4) * mag + LEAST[typ]
    if typ == "fp16":
        tol += (2.0 ** -25 * 2.0 ** -12 * (np.abs(_np(g)) + 16 * np.abs(_np(gh))))[:, None] * np.abs(_np(w)).sum(0)
    assert (np.abs(_np(got) - want) <= tol).all(), np.max(np.abs(_np(got) - want) / tol)


@pytest.mark.parametrize("how", ["spread", "few"])
@pytest.mark.parametrize("live", [70000, 131100])
def test_more_rows_than_are_sorted_together(pkg, live, how):
    """Rows are put in their tokens' order 65,536 at a time.  All logits alike, so that p = 1 / V; each token's rows come in groups of 17, 7 of weight 1 and hidden states of
    1 and 10 of 0.7 and -1, whose gradients add up to nothing: what is left of dW in bf16 are the roundings of the other tokens' dz, which are known, and those of the
    rows' own, which are put right row by row (0.02 a group: a row left out, or counted twice, is 0.0006 or 0.0016 off).  Bound: sums of R
    products in steps of 16, each cut off at 2^-23 of a partial sum (of some 1 in a group and what is left of them behind it), and the result's rounding."""
    import torch
    rng = np.random.default_rng(live)
    d, V, n = 64, 300, live // 17
    assert (n + 1) * 17 > 65536
    g17 = np.array([1, -.7, -.7, 1, -.7, 1, -.7, -.7, 1, -.7, 1, -.7, -.7, 1, -.7, 1, -.7])  # (partial sums within 1.2)
    assert abs(g17.sum()) < 1e-9
    tok = np.repeat(rng.integers(0, V, n) if how == "spread" else rng.integers(250, 253, n), 17)
    sign, g = np.tile(np.sign(g17), n), np.tile(np.abs(g17), n)
    R = 17 * n + 3000  # padding among them
    at = np.sort(rng.permutation(R)[:17 * n])
    toks, gs, hs = np.full(R, -1), np.full(R, 5.0), np.full(R, 9.0)
    toks[at], gs[at], hs[at] = tok, g, sign
    h = torch.from_numpy(hs).cuda().bfloat16()[:, None].repeat(1, d)
    w = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    ws, wsb = (pkg.linear_logprobs_workspace(R, d, V, backward=x) for x in (False, True))
    o = pkg.linear_logprobs(h, w, _i32(toks), workspace=ws)
    lp = _np(o.logprob)
    assert (lp[toks < 0] == 0).all() and np.abs(lp[at] + np.log(V)).max() < 1e-5
    dh, dw = pkg.linear_logprobs_backward(h, w, _i32(toks), o.stats, o.entropy, _f32(gs), workspace=wsb)
    assert not dh.any()
    bf16 = lambda x: torch.tensor(x, dtype=torch.float32).bfloat16().double().numpy()  # noqa: E731
    g32 = g.astype(np.float32).astype(np.float64)
    own = np.bincount(tok, sign * g32 * (1 - 1 / V), V)
    other = sign * bf16(-g32 / V)
    want = own + other.sum() - np.bincount(tok, other, V)
    got = _np(dw)
    rows = np.bincount(tok, minlength=V).max()
    part = max(1.2, 0.02 * rows / 17 + abs(other.sum()))
    tol = (live / 16 + 8) * 2.0 ** -23 * part + rows * 2.0 ** -24 * part + HALF["bf16"] * np.abs(want) + 1e-6
    assert (got == got[:, :1]).all()
    assert (np.abs(got[:, 0] - want) <= tol).all(), (np.max(np.abs(got[:, 0] - want) / tol), got[:4, 0], want[:4])


def test_gradients_of_more_rows_than_are_sorted_together(pkg):
    """Some 70,000 rows with logits of their own: a sample of them, and of the tokens, against 64 bits."""
    import torch
    rng = np.random.default_rng(70)
    R, d, V = 70100, 64, 300
    h, w = _inputs(rng, R, d, V, "bf16")
    tok = rng.integers(0, V, R)
    tok[rng.random(R) < 0.02] = -1
    g, gh = _f32(rng.standard_normal(R)), _f32(0.1 * rng.standard_normal(R))
    o = pkg.linear_logprobs(h, w, _i32(tok))
    dh, dw = pkg.linear_logprobs_backward(h, w, _i32(tok), o.stats, o.entropy, g, gh)
    some = np.unique(np.concatenate([rng.integers(0, R, 200), [0, 65535, 65536, 65537, R - 1]]))
    at = torch.from_numpy(some).cuda()
    _check(type(o)(o.logprob[at], o.entropy[at], o.stats[at]), h[at], w, tok[some], 1.0)
    _check_grad((dh[at], None), h[at], w, tok[some], g[at], gh[at], 1.0, "bf16")
    z = h.double() @ w.double().t()
    lp = torch.log_softmax(z, 1)
    dz = -g.double()[:, None] * lp.exp() - gh.double()[:, None] * lp.exp() * (lp - (lp.exp() * lp).sum(1, keepdim=True))
    t = torch.from_numpy(tok).cuda()
    dz[t >= 0, t[t >= 0]] += g.double()[t >= 0]
    dz[t < 0] = 0
    want = dz.t() @ h.double()
    mag = dz.abs().t() @ h.double().abs()
    assert bool(((dw.double() - want).abs() <= (_chain(R) + HALF["bf16"]) * mag + HALF["bf16"] * want.abs()).all())
    assert float((dw.double() - want).norm()) <= 1.5 * HALF["bf16"] * float(want.norm())


@pytest.mark.parametrize("typ,R", [("bf16", 1 << 19), ("fp16", 1 << 18)])
def test_weights_gradient_of_very_many_rows(pkg, typ, R):
    """Every row all but certain of the last token, whose dz is -g in each, and sampled from the others: dW of the last token is minus the sum of all g h, which
    are positive.  Bound: 1 - p below 2^-30, one rounding of the result, 2^-12 of the sum (parts of 4,096 rows lose at most 3 steps of 2^-24 each 16)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(R)
    d, V = 64, 300
    h = (torch.randint(128, 256, (R, d), generator=gen, device="cuda") * 2.0 ** -7).to(_dtype(typ))
    h *= 2.0 ** -8  # (sums within fp16)
    w = torch.zeros((V, d), dtype=h.dtype, device="cuda")
    w[V - 1] = 128.0  # a logit of 48
    tok = torch.randint(0, V - 1, (R,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.randint(128, 256, (R,), generator=gen, device="cuda").float() * 2.0 ** -7
    o = pkg.linear_logprobs(h, w, tok)
    assert float(o.entropy.max()) < 1e-6
    dh, dw = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g)
    want = -(g.double()[:, None] * h.double()).sum(0)
    assert bool(((dw[V - 1].double() - want).abs() <= (HALF[typ] + 2.0 ** -12) * want.abs()).all()), float((dw[V - 1].double() / want).mean())
    some = torch.arange(0, R, 4099, device="cuda")
    assert torch.equal(dh[some], -w[V - 1] * g[some, None].to(h.dtype))


def test_gradient_of_a_very_large_vocabulary(pkg):
    """Half a million tokens alike: dH of a row, whose token is none of the likely ones, is minus the mean of their weights, which are positive."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    R, d, V = 150, 20480, 780000
    h = torch.zeros((R, d), dtype=torch.float16, device="cuda")
    h[:, 0] = 1
    w = (torch.randint(1024, 2048, (V, d), generator=gen, device="cuda", dtype=torch.int16)).to(torch.float16).mul_(2.0 ** -10)
    w[:, 0] = 0
    w[5, 0] = -60
    tok, g = _i32(np.full(R, 5)), _f32(np.full(R, 2.0))
    o = pkg.linear_logprobs(h, w, tok)
    dh, _ = pkg.linear_logprobs_backward(h, w, tok, o.stats, o.entropy, g, grad_weight=False)
    total = torch.zeros(d, dtype=torch.float64, device="cuda")
    for a in range(0, V, 20000):
        total += w[a:a + 20000].double().sum(0)
    want = 2 * (w[5].double() - (total - w[5].double()) / (V - 1))[1:]
    # dz of a token: 2 / (V - 1) in fp16, whose rounding all of them share
    dz = torch.tensor(2.0 * 2 ** 20 / (V - 1)).half().double() * 2.0 ** -20
    off = float(dz * (V - 1) / 2 - 1)
    mean = (2 * (total - w[5].double()) / (V - 1))[1:]
    assert bool(((dh[0, 1:].double() - (want - off * mean)).abs() <= HALF["fp16"] * want.abs() + (2.0 ** -12 + 300 * U) * mean).all()), float((dh[0, 1:].double() - (want - off * mean)).mean())
    assert torch.equal(dh[0], dh[R - 1])


def test_millions_of_rows_of_one_token(pkg):
    """Their roundings are put right one after the other, which takes a CTA seconds while it has another tile to do: no wait of its may run out meanwhile.  Every third row
    weighs -1, the others 1/2, and all hidden states are 1, so that next to nothing is left.  Bound: parts of 4,096 rows lose at most 4 steps of 2^-24 each 16 of a part's
    sum of some 1; corrections, of 2^-10 and less, come in threes of no sum; the result's rounding."""
    import torch
    R, d, V = 1 << 21, 4872, 1000
    g = torch.full((R,), 0.5, device="cuda")
    g[::3] = -1.0
    h, w = torch.ones((R, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    tok = torch.full((R,), 7, dtype=torch.int32, device="cuda")
    stats, entropy = torch.zeros((R, 2), device="cuda"), torch.zeros(R, device="cuda")
    stats[:, 1] = float(np.log(V))
    _, dw = pkg.linear_logprobs_backward(h, w, tok, stats, entropy, g, grad_hidden=False)
    want = torch.full((V,), -float(g.double().sum()) / V, dtype=torch.float64)
    want[7] += float(g.double().sum())
    assert not dw.isnan().any()
    assert bool(((dw.double().cpu() - want[:, None]).abs() <= HALF["bf16"] * want[:, None].abs() + 0.05).all()), (dw[7], want[7])
