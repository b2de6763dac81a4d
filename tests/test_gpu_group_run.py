"""A group of rollouts as it is used: the prompt and the rollouts' own tokens into the 8-bit cache, a decode step behind the common prompt, and
the policy loss's terms and gradients of the heads' outputs, eagerly and captured."""
import numpy as np
import pytest

import test_gpu_linear_logprobs as linear
import test_gpu_shared_kv8 as shared
from test_gpu_kv8 import Cache, _i32, _q, _tokens
from test_gpu_shared_kv8 import route  # noqa: F401  (both)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    p.load()
    return p


@pytest.mark.parametrize("sizes,H,kvh,hd,V,fmt,typ", [([8, 8], 4, 1, 64, 700, "e4m3", "bf16"), ([5, 1, 40, 3], 6, 2, 32, 333, "int8", "fp16"),
                                                      ([90, 70], 4, 2, 128, 1500, "e4m3", "bf16")])
def test_decode_then_score_then_gradient(pkg, sizes, H, kvh, hd, V, fmt, typ):
    import torch
    rng = np.random.default_rng(sum(sizes))
    start = np.concatenate([[0], np.cumsum(sizes)])
    n, blocks = int(start[-1]), 4
    prompt, own = rng.integers(1, 300, len(sizes)), rng.integers(0, 150, n)
    c = Cache(pkg, rng, n, blocks, kvh, hd, fmt)
    c.codes.view(torch.uint8).zero_()
    c.scales.fill_(2.0 ** -100)  # (as kv8_cache gives them: blocks are first written in their middle)
    c.want_codes, c.want_scales = c.values(), c.scales.double().cpu().numpy()
    lead, prefix = shared._groups(n, start, prompt)
    for i in range(n):  # whole pages of the prompt are the first sequence's
        c.table[i, :prefix[i] // 128] = c.table[lead[i], :prefix[i] // 128]
    c.tab = _i32(c.table)
    # the prompts, through their first sequences; then each sequence's own tokens behind its prompt
    at = np.concatenate([[0], np.cumsum(np.where(lead == np.arange(n), prefix, 0))])
    c.write(*_tokens(rng, at[-1], kvh, hd, typ), np.zeros(n, np.int64), at)
    at = np.concatenate([[0], np.cumsum(own)])
    c.write(*_tokens(rng, at[-1], kvh, hd, typ), prefix, at)
    c.check()
    ctx = prefix + own
    q = _q(rng, n, H, hd, typ)
    w = torch.from_numpy(rng.standard_normal((V, H * hd)) / np.sqrt(hd)).cuda().to(q.dtype)
    tok = rng.integers(0, V, n)
    tok[::7] = -1
    g, gh = (torch.from_numpy(rng.standard_normal(n)).float().cuda() for _ in range(2))
    args = _i32(ctx), _i32(start), _i32(prompt), _i32(tok)
    tab = shared._table(c, len(sizes))
    ws = pkg.attention_shared_kv8_workspace(n, len(sizes), H, kvh, hd)
    ws1, ws2 = (pkg.linear_logprobs_workspace(n, H * hd, V, back) for back in (False, True))

    def run():
        out = pkg.attention_shared_kv8(q, c.codes, c.scales, tab, *args[:3], workspace=ws)
        hidden = out.view(n, H * hd)
        s = pkg.linear_logprobs(hidden, w, args[3], scale=2.0, workspace=ws1)
        return out, s, pkg.linear_logprobs_backward(hidden, w, args[3], s.stats, s.entropy, g, gh, scale=2.0, workspace=ws2)

    out, s, grads = run()
    shared._check(c, q, ctx, start, prompt, out, typ)
    hidden = out.view(n, H * hd)
    linear._check(s, hidden, w, tok, 2.0)
    linear._check_grad(grads, hidden, w, tok, g, gh, 2.0, typ, spread=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = run()
    for _ in range(2):
        graph.replay()
        for a, b in zip((out, s.logprob, s.entropy, s.stats, *grads), (again[0], again[1].logprob, again[1].entropy, again[1].stats, *again[2])):
            assert torch.equal(a, b)
