"""Attention behind a common prefix and log-probabilities from hidden states refuse wrong arguments before they touch a device: through the
C ABI with made-up addresses, and through the binding with tensors that are not on a GPU."""
import pytest
import torch

from test_ops_refusals import A, BAD_CACHES, _cache, _refused, lib, pkg  # noqa: F401


def test_shared_attention_refusals(lib):  # noqa: F811
    size = lib.sara_attention_shared_kv8_workspace_bytes
    assert size(0, 1, 8, 2, 64) == 0 and size(4, -1, 8, 2, 64) == 0 and size(4, 1, 0, 2, 64) == 0 and size(4, 1, 8, 0, 64) == 0
    assert size(1 << 28, 1, 16, 2, 64) == 0
    assert 0 < size(4, 1, 8, 2, 64) <= size(5, 1, 8, 2, 64) <= size(5, 3, 8, 2, 64) <= size(5, 3, 16, 2, 64) <= size(5, 3, 16, 2, 128)

    def call(cache=None, n=3, H=8, q=A, qs=512, ctx=A, first=None, groups=2, start=A, prefix=A, out=A, lse=None, typ=0, ws=A, nbytes=1 << 34):
        return lib.sara_attention_shared_kv8(cache or _cache(), n, H, q, qs, ctx, first, groups, start, prefix, out, lse, typ, None, ws, nbytes, None)

    for bad in BAD_CACHES:
        assert call(cache=_cache(**bad)) == -1, bad
    assert lib.sara_attention_shared_kv8(None, 3, 8, A, 512, A, None, 2, A, A, A, None, 0, None, A, 1 << 34, None) == -1
    for bad in (dict(n=-1), dict(H=0), dict(H=7), dict(H=18), dict(q=None), dict(q=A + 8), dict(qs=511), dict(qs=256), dict(ctx=None), dict(groups=-1),
                dict(groups=4), dict(start=None), dict(prefix=None), dict(out=None), dict(out=A + 8), dict(typ=2), dict(typ=-1), dict(ws=None),
                dict(ws=A + 16), dict(nbytes=0), dict(nbytes=size(3, 2, 8, 2, 64) - 1), dict(n=1 << 28, H=16, groups=1),
                dict(cache=_cache(max_blocks=1 << 23, table_stride=1 << 23), n=64)):
        assert call(**bad) == -1, bad
    assert call(n=0, groups=0) == 0  # nothing to do: no device is touched
    assert call(n=0, groups=0, cache=_cache(table=0), q=None, ctx=None, start=None, prefix=None, out=None, ws=None, nbytes=0) == 0


def test_linear_scoring_refusals(lib):  # noqa: F811
    size, big = lib.sara_linear_logprobs_workspace_bytes, 1 << 40
    for back in (0, 1):
        assert size(4, 64, 1000, back) > 0 and size(0, 64, 1000, back) >= 0
        for bad in ((-1, 64, 1000), ((1 << 22) + 1, 64, 1000), (4, 0, 1000), (4, 60, 1000), (4, 65544, 1000), (4, 64, 0), (4, 64, (1 << 24) + 1)):
            assert size(*bad, back) == 0, bad
        # the largest sizes: counted in 64 bits
        assert size(1 << 22, 65536, 1 << 24, back) > 2 * (1 << 22) * 65536 * back

    def fwd(h=A, hs=64, w=A, ws=64, typ=0, R=3, d=64, V=100, tok=A, scale=1.0, lp=A, ent=A, stats=A, scratch=A, n=big):
        return lib.sara_linear_logprobs(h, hs, w, ws, typ, R, d, V, tok, scale, lp, ent, stats, scratch, n, None)

    wrong = (dict(h=None), dict(h=A + 8), dict(hs=60), dict(hs=56), dict(hs=0), dict(hs=-64), dict(w=None), dict(w=A + 2), dict(ws=68), dict(ws=0), dict(typ=2),
             dict(typ=-1), dict(R=-1), dict(R=(1 << 22) + 1), dict(d=0), dict(d=60), dict(d=65544, hs=65544, ws=65544), dict(V=0), dict(V=(1 << 24) + 1),
             dict(tok=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scratch=None),
             dict(scratch=A + 16), dict(n=0))
    for bad in wrong + (dict(n=size(3, 64, 100, 0) - 1),):
        assert fwd(**bad) == -1, bad
    assert fwd(R=0) == 0 and fwd(R=0, h=None, tok=None, scratch=None) == 0

    def bwd(h=A, hs=64, w=2 * A, ws=64, typ=0, R=3, d=64, V=100, tok=A, scale=1.0, stats=A, ent=A, g=A, gh=A, dh=3 * A, dhs=64, dw=4 * A, dws=64,
            scratch=A, n=big):
        return lib.sara_linear_logprobs_backward(h, hs, w, ws, typ, R, d, V, tok, scale, stats, ent, g, gh, dh, dhs, dw, dws, scratch, n, None)

    for bad in wrong + (dict(n=size(3, 64, 100, 1) - 1), dict(stats=None), dict(ent=None), dict(dh=None, dw=None), dict(dh=A + 3 * A // 8 + 8), dict(dhs=60),
                        dict(dhs=56), dict(dw=4 * A + 8), dict(dws=0), dict(dws=65),
                        dict(dh=A), dict(dw=2 * A), dict(dh=2 * A), dict(dw=A), dict(dw=3 * A), dict(dh=A + 256), dict(dh=4 * A + 64 * 198)):  # operands that meet
        assert bwd(**bad) == -1, bad
    assert bwd(R=0, dw=None) == 0


def test_binding_refuses_tensors_that_do_not_fit_a_shared_prefix(pkg):  # noqa: F811
    codes, scales = pkg.kv8_cache(4, 2, 64, device="cpu")
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32)  # noqa: E731
    q = torch.zeros(3, 8, 64, dtype=torch.float16)
    ok = dict(q=q, codes=codes, scales=scales, table=i32(3, 2), ctx=i32(3), group_start=i32(3), prefix=i32(2), workspace=torch.zeros(1024, dtype=torch.uint8))

    def att(**kw):
        return _refused(pkg, pkg.attention_shared_kv8, **{**ok, **kw})

    assert "CUDA" in att()
    assert "CUDA" in att(first=i32(3), out=q.clone(), lse=torch.zeros(3, 8), status=i32(1))
    att(codes=codes.view(torch.uint8))
    att(table=i32(3, 2).long())
    att(q=q.float())
    att(q=q[:2])
    att(q=q[..., :32])
    att(q=q[:, :, ::2])
    att(q=q.transpose(0, 1).contiguous().transpose(0, 1))
    att(ctx=i32(3).long())
    att(ctx=i32(2))
    att(group_start=i32(2))
    att(group_start=i32(3).long())
    att(group_start=i32(6)[::2])
    att(prefix=i32(3))
    att(prefix=i32(2, 1))
    att(prefix=i32(2).long())
    assert "as many groups" in att(prefix=i32(4), group_start=i32(5))
    att(first=i32(2))
    att(out=q.bfloat16())
    att(out=q[:2])
    att(lse=torch.zeros(3, 4))
    att(lse=torch.zeros(3, 8).double())
    att(status=i32(2))
    att(workspace=torch.zeros(2048, dtype=torch.uint8)[::2])
    for bad in ((-1, 1, 8, 2, 64), (2 ** 32 + 5, 1, 8, 2, 64), (4, 2 ** 32 + 1, 8, 2, 64)):
        assert "0 .. 2^31 - 1" in _refused(pkg, pkg.attention_shared_kv8_workspace, *bad, device="cpu")


def test_binding_refuses_tensors_that_do_not_fit_linear_scoring(pkg):  # noqa: F811
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32)  # noqa: E731
    h, w, st, v = torch.zeros(4, 64).bfloat16(), torch.zeros(10, 64).bfloat16(), torch.zeros(4, 2), torch.zeros(4)

    def fwd(hidden=h, weight=w, tokens=i32(4), **kw):
        return _refused(pkg, pkg.linear_logprobs, hidden, weight, tokens, **kw)

    def bwd(hidden=h, weight=w, tokens=i32(4), stats=st, entropy=v, grad_logprob=v, **kw):
        return _refused(pkg, pkg.linear_logprobs_backward, hidden, weight, tokens, stats, entropy, grad_logprob, **kw)

    for f in (fwd, bwd):
        assert "CUDA" in f()
        f(hidden=h.float(), weight=w.float())
        f(hidden=h.half())
        f(hidden=h[0])
        f(hidden=h[:, ::2], weight=w[:, :32])
        f(weight=w[:, :32])
        f(weight=w.t().contiguous().t())
        f(tokens=i32(3))
        f(tokens=i32(4).long())
        f(tokens=i32(8)[::2])
    bwd(stats=st[:, :1])
    bwd(stats=st.double())
    bwd(entropy=v[:3])
    bwd(grad_logprob=v[:1].expand(4))
    bwd(grad_logprob=v.half())
    bwd(grad_entropy=v[:2])
    bwd(grad_hidden=h.half())
    bwd(grad_hidden=h[:3])
    bwd(grad_weight=w.float())
    bwd(grad_weight=w.t().contiguous().t())
    assert "0 .. 2^31 - 1" in _refused(pkg, pkg.linear_logprobs_workspace, -1, 64, 100, device="cpu")


# counts that int32 does not hold are refused before a call could cut them short (tensors without memory)
def test_binding_refuses_more_rows_than_the_calls_count(pkg):  # noqa: F811
    many = 2 ** 32 + 5
    new = lambda *a, t=torch.bfloat16: torch.empty(*a, dtype=t, device="meta")  # noqa: E731
    i32 = lambda *a: new(*a, t=torch.int32)  # noqa: E731
    for R, V, d in ((many, 10, 64), (4, many, 64), (4, 10, many)):
        h, w, v, st = new(R, d), new(V, d), new(R, t=torch.float32), new(R, 2, t=torch.float32)
        assert "2^31" in _refused(pkg, pkg.linear_logprobs, h, w, i32(R))
        assert "2^31" in _refused(pkg, pkg.linear_logprobs_backward, h, w, i32(R), st, v, v)
        assert "2^31" in _refused(pkg, pkg.linear_logprobs_workspace, R, d, V)
    codes, scales = pkg.kv8_cache(4, 2, 64, device="meta")
    assert "2^31" in _refused(pkg, pkg.attention_shared_kv8, new(many, 8, 64), codes, scales, i32(many, 1), i32(many), i32(2), i32(1))


def test_scales_whose_exponents_leave_fp32_are_refused(lib):  # noqa: F811
    for scale, rc in ((2.0 ** 127, 0), (1.0000002 * 2.0 ** 127, -1), (3.4e38, -1), (1e-45, 0)):
        assert lib.sara_linear_logprobs(A, 64, A, 64, 0, 0, 64, 100, A, scale, A, A, A, A, 1 << 40, None) == rc, scale
        assert lib.sara_linear_logprobs_backward(A, 64, 2 * A, 64, 0, 0, 64, 100, A, scale, A, A, A, A, 3 * A, 64, None, 64, A, 1 << 40, None) == rc, scale
