"""The cache and scoring operators refuse wrong arguments before they touch a device: through the C ABI with made-up
addresses, and through the binding with tensors that are not on a GPU."""
import ctypes

import pytest
import torch

import __graft_entry__

A = 1 << 20  # an aligned address that a refused call never follows


@pytest.fixture(scope="module")
def pkg():
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    return p


@pytest.fixture(scope="module")
def lib(pkg):
    return pkg.load()


def _cache(**kw):
    import paper_2607_26253_gb300.sara as s
    f = dict(codes=A, scales=A, table=A, table_stride=4, n_blocks=8, max_blocks=4, n_kv_heads=2, head_dim=64, format=0)
    f.update(kw)
    return ctypes.byref(s.Kv8Cache(*[f[n] for n, _ in s.Kv8Cache._fields_]))


BAD_CACHES = [dict(codes=0), dict(scales=0), dict(table=0), dict(codes=A + 8), dict(scales=A + 2), dict(table_stride=3), dict(n_blocks=0),
              dict(max_blocks=0), dict(max_blocks=1 << 24, table_stride=1 << 24), dict(n_kv_heads=0), dict(head_dim=48), dict(head_dim=256),
              dict(format=2), dict(format=-1)]


def test_write_and_read_refusals(lib):
    def call(fn, cache=None, n=2, pos0=A, start=A, total=4, k=A, ks=128, v=A, vs=128, typ=0):
        return fn(cache or _cache(), n, pos0, start, total, k, ks, v, vs, typ, None, None)

    for fn, types in ((lib.sara_kv8_write, (0, 1)), (lib.sara_kv8_read, (0, 1, 2))):
        assert fn(None, 2, A, A, 4, A, 128, A, 128, 0, None, None) == -1
        for bad in BAD_CACHES:
            assert call(fn, cache=_cache(**bad)) == -1, bad
        for bad in (dict(n=-1), dict(total=-1), dict(pos0=None), dict(start=None), dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2),
                    dict(ks=127), dict(ks=132), dict(vs=120), dict(vs=0), dict(typ=-1), dict(typ=max(types) + 1)):
            assert call(fn, **bad) == -1, bad
        for t in types:  # nothing to do: no device is touched
            assert call(fn, n=0, typ=t) == 0 and call(fn, total=0, typ=t) == 0
            assert call(fn, cache=_cache(table=0), n=0, typ=t, pos0=None, start=None) == 0


def test_write_and_read_refuse_more_sequences_than_their_search_counts(lib):
    # 32-bit sums of its steps would pass 2^31 shortly before the last int32, and its loads leave the starts
    for fn in (lib.sara_kv8_write, lib.sara_kv8_read):
        for n in ((1 << 30) + 1, 2 ** 31 - 31, 2 ** 31 - 1):
            assert fn(_cache(n_kv_heads=1), n, A, A, 1, A, 64, A, 64, 0, None, None) == -1


def test_attention_refusals(lib):
    assert lib.sara_attention_kv8_workspace_bytes(0, 8, 2, 64) == 0
    assert lib.sara_attention_kv8_workspace_bytes(4, 8, 0, 64) == 0

    def call(cache=None, n=2, H=8, q=A, qs=512, ctx=A, out=A, typ=0, ws=A, nbytes=1 << 30):
        return lib.sara_attention_decode_kv8(cache or _cache(), n, H, q, qs, ctx, None, out, None, typ, None, ws, nbytes, None)

    for bad in BAD_CACHES:
        assert call(cache=_cache(**bad)) == -1, bad
    for bad in (dict(n=-1), dict(H=0), dict(H=7), dict(H=18), dict(q=None), dict(q=A + 8), dict(qs=511), dict(qs=256), dict(ctx=None),
                dict(out=None), dict(out=A + 8), dict(typ=2), dict(typ=-1), dict(ws=None), dict(ws=A + 8), dict(nbytes=0), dict(n=1 << 28, H=16)):
        assert call(**bad) == -1, bad
    assert call(n=0) == 0 and call(n=0, cache=_cache(table=0)) == 0
    for n, blocks in ((64, 1 << 23), (1 << 29, 1), (1 << 27, 4)):  # 2^30 blocks and heads of them
        assert call(n=n, H=2, cache=_cache(max_blocks=blocks, table_stride=blocks)) == -1
    # a workspace that was laid out for fewer rows is enough only where the larger batch wants no more
    size = [lib.sara_attention_kv8_workspace_bytes(n, 8, 2, 64) for n in (1, 50, 799, 800, 5000)]
    assert size == sorted(size) and size[0] == size[2] < size[3] == size[4]
    assert call(n=800, nbytes=size[2]) == -1 and call(n=1, nbytes=size[0] - 1) == -1


def test_scoring_refusals(lib):
    def fwd(z=A, stride=100, typ=0, R=3, V=100, tok=A, top=0, lp=A, ent=A, stats=A, tt=None, tl=None):
        return lib.sara_logprobs(z, stride, typ, R, V, tok, top, lp, ent, stats, tt, tl, None)

    for bad in (dict(z=None), dict(z=A + 1), dict(z=A + 2, typ=2), dict(stride=99), dict(stride=0), dict(typ=3), dict(typ=-1), dict(R=-1),
                dict(V=0), dict(tok=None), dict(top=-1), dict(top=33, tt=A, tl=A), dict(top=1), dict(top=1, tt=A), dict(top=1, tl=A)):
        assert fwd(**bad) == -1, bad
    assert fwd(R=0) == 0

    def bwd(z=A, stride=100, typ=0, R=3, V=100, tok=A, stats=A, ent=A, g=A, gh=A, out=2 * A, os=100):
        return lib.sara_logprobs_backward(z, stride, typ, R, V, tok, stats, ent, g, gh, out, os, None)

    for bad in (dict(z=None), dict(z=A + 1), dict(stride=99), dict(typ=3), dict(R=-1), dict(V=0), dict(tok=None), dict(stats=None),
                dict(ent=None), dict(out=None), dict(out=A + 1), dict(os=99), dict(os=0), dict(out=A, os=120)):
        assert bwd(**bad) == -1, bad
    assert bwd(R=0) == 0


def _refused(pkg, f, *a, **kw):
    with pytest.raises(pkg.SaraError) as e:
        f(*a, **kw)
    assert e.value.code == pkg.SARA_EINVAL
    return str(e.value)


def test_binding_refuses_tensors_that_do_not_fit(pkg):
    codes, scales = pkg.kv8_cache(4, 2, 64, device="cpu")
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32)  # noqa: E731
    table, k = i32(3, 2), torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    ok = dict(codes=codes, scales=scales, table=table, k=k, v=k, pos0=i32(3), seq_start=i32(4))

    def write(**kw):
        return _refused(pkg, pkg.kv8_write, **{**ok, **kw})

    assert "CUDA" in write()
    write(codes=codes.view(torch.uint8))
    write(codes=codes[:, :1])
    write(codes=codes.transpose(2, 3))
    write(scales=scales[:3])
    write(scales=scales.half())
    write(table=table.long())
    write(table=table[0])
    write(table=i32(2, 3).t())
    write(table=table[:1].expand(3, 2))
    write(k=k.float(), v=k.float())
    write(k=k.half())
    write(k=k[:4])
    write(k=k[:, :1])
    write(k=k.transpose(0, 1).contiguous().transpose(0, 1), v=k)
    write(pos0=i32(4))
    write(pos0=i32(3).long())
    write(seq_start=i32(3))
    write(seq_start=i32(8)[::2])
    write(status=i32(2))
    rd = lambda **kw: _refused(pkg, pkg.kv8_read, **{**dict(codes=codes, scales=scales, table=table, pos0=i32(3), seq_start=i32(4), total=5), **kw})  # noqa: E731
    assert "CUDA" in rd()
    rd(out=(k, k[:4]))
    rd(out=(k, k.half()))
    rd(dtype=torch.float64)
    q = torch.zeros(3, 8, 64, dtype=torch.float16)
    base = dict(q=q, codes=codes, scales=scales, table=table, ctx=i32(3), workspace=torch.zeros(1024, dtype=torch.uint8))
    att = lambda **kw: _refused(pkg, pkg.attention_decode_kv8, **{**base, **kw})  # noqa: E731
    assert "CUDA" in att()
    att(q=q.float())
    att(q=q[:2])
    att(q=q[..., :32])
    att(q=q[:, :, ::2])
    att(ctx=i32(3).long())
    att(first=i32(2))
    att(out=q.bfloat16())
    att(out=q[:2])
    att(lse=torch.zeros(3, 4))
    att(lse=torch.zeros(3, 8).double())
    z = torch.zeros(4, 10)
    assert "CUDA" in _refused(pkg, pkg.logprobs, z, i32(4))
    _refused(pkg, pkg.logprobs, z, i32(3))
    _refused(pkg, pkg.logprobs, z, i32(4).long())
    _refused(pkg, pkg.logprobs, z.double(), i32(4))
    _refused(pkg, pkg.logprobs, z.t(), i32(10))
    _refused(pkg, pkg.logprobs, z[0], i32(4))
    _refused(pkg, pkg.logprobs, z, i32(4), top=33)
    st, h = torch.zeros(4, 2), torch.zeros(4)
    assert "CUDA" in _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h, h, h)
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st[:, :1], h, h, h)
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h[:3], h, h)
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h, h.double(), h)
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h, h[:1].expand(4), h)  # (not broadcast)
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h, h, h, out=z.half())
    _refused(pkg, pkg.logprobs_backward, z, i32(4), st, h, h, h, out=z[:3])


# counts that int32 does not hold are refused before a call could cut them short (tensors without memory)
def test_binding_refuses_more_rows_than_the_calls_count(pkg):
    many = 2 ** 32 + 5
    codes, scales = pkg.kv8_cache(4, 2, 64, device="meta")
    i32 = lambda *a: torch.empty(*a, dtype=torch.int32, device="meta")  # noqa: E731
    assert "2^31" in _refused(pkg, pkg.kv8_read, codes, scales, i32(many, 1), i32(many), i32(many + 1), 5)
    assert "2^31" in _refused(pkg, pkg.kv8_read, codes, scales, i32(3, 2), i32(3), i32(4), many)
    assert "total" in _refused(pkg, pkg.kv8_read, codes, scales, i32(3, 2), i32(3), i32(4), -1)
    k = torch.empty((many, 2, 64), dtype=torch.bfloat16, device="meta")
    assert "2^31" in _refused(pkg, pkg.kv8_write, codes, scales, i32(3, 2), k, k, i32(3), i32(4))
    for shape in ((1, many), (many, 1)):
        z = torch.empty(shape, dtype=torch.bfloat16, device="meta")
        assert "2^31" in _refused(pkg, pkg.logprobs, z, i32(shape[0]))
        v = torch.empty(shape[0], device="meta")
        assert "2^31" in _refused(pkg, pkg.logprobs_backward, z, i32(shape[0]), torch.empty((shape[0], 2), device="meta"), v, v)
