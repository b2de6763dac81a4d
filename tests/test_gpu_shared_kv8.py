"""Attention of groups behind a common prefix over the 8-bit cache, on the GPU against the 64-bit oracle, within bounds that follow from
the arithmetic."""
import numpy as np
import pytest

from oracle import kv8 as oracle
from test_gpu_kv8 import HALF_STEP, Cache, _i32, _q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    p.load()
    return p


ALONE = 160 << 20  # bytes that the table's rows have room for, less those of two rows a group, up to which every row attends by itself


@pytest.fixture(params=["alone", "shared"], autouse=True)
def route(request, monkeypatch):
    """Both ways to the results: small tables, and the same ones with room for more positions (their ids wrong, and not read)."""
    monkeypatch.setattr(Cache, "wide", request.param == "shared", raising=False)


def _table(c, groups):
    import torch
    n = len(c.tab)
    more = max(0, ALONE // ((n - 2 * groups) * c.kvh * 256 * c.hd) + 1 - c.tab.shape[1]) if c.wide and n > 2 * groups else 0
    return torch.cat([c.tab, torch.full((n, more), -7, dtype=torch.int32, device="cuda")], 1)


def _groups(n, start, prefix):
    """Each row's first row of its group and its shared positions (itself and 0 without a group)."""
    lead, shared = np.arange(n), np.zeros(n, np.int64)
    for g in range(len(prefix)):
        lead[start[g]:start[g + 1]], shared[start[g]:start[g + 1]] = start[g], prefix[g]
    return lead, shared


def _check(c, q, ctx, start, prefix, out, typ, first=None, lse=None, rows=None):
    """Bounds: scores off by (hd + 24) roundings of 32 bits of sum |q k| / sqrt(hd); probabilities times scales in 11 bits, or within 2^-31
    of the largest; sums of at most a quarter of the positions in a chain; two states joined; the result rounded once."""
    got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    lead, shared = _groups(len(ctx), start, prefix)
    for i in range(len(ctx)) if rows is None else rows:
        a, n = 0 if first is None else first[i], ctx[i]
        cut = min(max(shared[i], a), max(n, a))
        parts = [oracle.read(c.want_codes, c.want_scales, c.table[lead[i]], a, cut), oracle.read(c.want_codes, c.want_scales, c.table[i], cut, max(n, cut))]
        k, v = (np.concatenate([x[j] for x in parts]) for j in (0, 1))
        want, wl, mag, pv = oracle.attention(qn[i], k, v)
        ds = (c.hd + 24) * 2.0 ** -24 * mag[:, None]
        vmax = np.abs(v).max() if len(v) else 0.0
        tol = HALF_STEP[typ] * np.abs(want) + (2.0 ** -11 + 2 * ds + 2.0 ** -19 + (len(k) / 4 + 64) * 2.0 ** -24) * pv \
            + max(1, len(k)) * 2.0 ** -31 * vmax + 2.0 ** -25
        assert (np.abs(got[i] - want) <= tol).all(), (i, n, np.max(np.abs(got[i] - want) - tol))
        if lse is not None:
            l = lse[i].double().cpu().numpy()
            if n <= a:
                assert (l == -np.inf).all(), i
            else:
                assert (np.abs(l - wl) <= ds[:, 0] + (len(k) / 4 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(wl))).all(), (i, l, wl)


def _run(pkg, c, q, ctx, start, prefix, first=None, **kw):
    import torch
    lse, status = torch.empty(q.shape[:2], device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = pkg.attention_shared_kv8(q, c.codes, c.scales, _table(c, len(prefix)), _i32(ctx), _i32(start), _i32(prefix), first=None if first is None else _i32(first),
                                   lse=lse, status=status, **kw)
    return out, lse, int(status)


# prefixes that end in and between scale blocks and pages; rows that end in their prefix, at its end, behind it, or hold nothing
@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,kvh,hd", [(6, 1, 128), (8, 1, 64), (2, 1, 32), (4, 4, 128), (9, 3, 32), (14, 2, 64), (15, 3, 128), (32, 4, 128)])
def test_edges(pkg, H, kvh, hd, fmt, typ):
    rng = np.random.default_rng(hd + H)
    prefix = [1, 31, 32, 33, 100, 127, 128, 129, 255, 256, 300, 0, 640]
    sizes = [2, 3, 1, 4, 5, 2, 2, 7, 3, 2, 6, 3, 4]
    start = np.concatenate([[0], np.cumsum(sizes)])
    n = int(start[-1])
    lead, shared = _groups(n, start, prefix)
    ctx = np.minimum(np.maximum(shared + rng.choice([0, -1, 1, 2, 31, 32, 33, 100, 127, 128], n), 0), 768)
    ctx[5], ctx[17] = 0, 768
    c = Cache(pkg, rng, n, 6, kvh, hd, fmt)
    q = _q(rng, n, H, hd, typ)
    out, lse, status = _run(pkg, c, q, ctx, start, prefix)
    assert status == 0
    _check(c, q, ctx, start, prefix, out, typ, lse=lse)


# few and many queries of a group: one tile, two, several; long prefixes split over CTAs, short ones many to a CTA
@pytest.mark.parametrize("fmt,typ", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("sizes,H,kvh,hd,blocks", [([64], 8, 1, 128, 3), ([16, 17], 8, 1, 128, 2), ([33], 16, 2, 64, 40), ([90, 2], 6, 1, 128, 5), ([3] * 40, 4, 2, 64, 3),
                                                   ([130], 4, 1, 32, 9), ([2, 200, 2], 2, 1, 128, 4), ([8] * 12, 12, 2, 128, 12), ([40] * 5, 28, 4, 128, 6),
                                                   ([42] * 6, 16, 8, 128, 40), ([20] * 5, 24, 4, 128, 60), ([69, 30, 128], 2, 2, 32, 170), ([40] * 9, 32, 8, 64, 30)])
def test_group_sizes(pkg, sizes, H, kvh, hd, blocks, fmt, typ):
    import torch
    rng = np.random.default_rng(sum(sizes) + hd)
    start = np.concatenate([[0], np.cumsum(sizes)])
    n = int(start[-1])
    prefix = rng.integers(1, 128 * blocks - 100, len(sizes))
    prefix[0] = 128 * blocks - 100
    lead, shared = _groups(n, start, prefix)
    ctx = shared + rng.integers(0, 100, n)
    c = Cache(pkg, rng, 20, blocks, kvh, hd, fmt)
    c.table = rng.integers(0, c.codes.shape[0], (n, blocks)).astype(np.int32)
    c.tab = _i32(c.table)
    q = _q(rng, n, H, hd, typ)
    ws = pkg.attention_shared_kv8_workspace(n, len(sizes), H, kvh, hd)
    out, lse, status = _run(pkg, c, q, ctx, start, prefix, workspace=ws)
    assert status == 0
    _check(c, q, ctx, start, prefix, out, typ, lse=lse, rows=np.unique(np.concatenate([rng.integers(0, n, 30), start[:-1], start[1:] - 1])))
    for _ in range(3):  # the same bits again, from the same workspace
        again, lse2, _ = _run(pkg, c, q, ctx, start, prefix, workspace=ws)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_nan_reaches_its_rows_alone(pkg, hd, fmt):
    """Scales of NaN, and in e4m3 codes of NaN, among keys and values: a row is NaN where it attends to the block of 32, whichever way,
    and as it would be without them where it does not."""
    import torch
    rng = np.random.default_rng(hd)
    n, prefix = 40, 700
    ctx = np.array([(37 * i) % 760 for i in range(n)])
    first = np.where(np.arange(n) % 3 == 0, (53 * np.arange(n)) % 600, 0)
    c = Cache(pkg, rng, n, 6, 2, hd, fmt)
    q = _q(rng, n, 12, hd, "bf16")
    want = _run(pkg, c, q, ctx, [0, n], [prefix], first)[:2]
    shared = c.table[0]
    for at, kv, how in ((10, 0, "scale"), (300, 1, "scale"), (420, 0, "code"), (640, 1, "code"), (127, 1, "code"), (128, 0, "scale"), (699, 1, "code")):
        page, slot = shared[at // 128], at % 128
        codes, scales = c.codes.view(torch.uint8).clone(), c.scales.clone()
        if how == "scale":
            scales[page, kv, :, slot // 32] = float("nan")
            hit = (first < at // 32 * 32 + 32) & (np.minimum(ctx, prefix) > at // 32 * 32) & (first < ctx)
        else:
            if fmt == "int8" or not c.wide:  # (a row by itself: as the decode attention, whose value of NaN makes its dim NaN)
                continue
            codes[page, kv, :, slot, hd // 2] = 0xff
            hit = (first < at // 32 * 32 + 32) & (np.minimum(ctx, prefix) > at // 32 * 32) & (first < ctx)
        lse, status = torch.empty((n, 12), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = pkg.attention_shared_kv8(q, codes.view(c.codes.dtype), scales, _table(c, 1), _i32(ctx), _i32([0, n]), _i32([prefix]), first=_i32(first), lse=lse, status=status)
        assert int(status) == 0
        for i in range(n):
            if hit[i]:
                assert bool(out[i].isnan().all()), (at, kv, how, i)
                assert bool(lse[i].isnan().all()) or (kv == 1 and not c.wide), (at, kv, how, i)  # (values have no part in it)
            else:
                assert torch.equal(out[i], want[0][i]) and torch.equal(lse[i], want[1][i]), (at, kv, how, i)


def _batch(pkg, rng, fmt="e4m3", typ="bf16", hd=64, H=8, kvh=2, blocks=6):
    """Rows of no group before, between empty groups' places and behind, a group of one, groups of several."""
    start = [2, 2, 7, 8, 8, 40, 45]
    prefix = [100, 300, 200, 128, 513, 64]
    n = 48
    c = Cache(pkg, rng, n, blocks, kvh, hd, fmt)
    ctx = rng.integers(0, 128 * blocks + 1, n)
    ctx[9], ctx[10], ctx[11], ctx[12] = 0, 513, 512, 514
    return c, _q(rng, n, H, hd, typ), ctx, start, prefix


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_windows_strides_and_rows_of_no_group(pkg, hd, fmt, typ):
    import torch
    rng = np.random.default_rng(hd + 3)
    c, q, ctx, start, prefix = _batch(pkg, rng, fmt, typ, hd)
    n, H = q.shape[:2]
    # windows from in the prefix, at its end, behind it, at and behind the row's end
    first = np.maximum(0, rng.choice([0, 1, 31, 33, 127, 128, 200, 300, 512, 513, 520, 700], n))
    first[14], first[15], first[16], ctx[14], ctx[15], ctx[16] = 513, 512, 700, 600, 600, 650
    wide = torch.full((n, 3 * H * hd + 8), float("nan"), dtype=q.dtype, device="cuda")
    strided = wide[:, 8:8 + H * hd].view(n, H, hd)
    strided.copy_(q)
    out = torch.full_like(q, 7.0)
    got, lse, status = _run(pkg, c, strided, ctx, start, prefix, first, out=out)
    assert got is out and status == 0
    _check(c, q, ctx, start, prefix, out, typ, first=first, lse=lse)
    again = pkg.attention_shared_kv8(q, c.codes, c.scales, _table(c, len(prefix)), _i32(ctx), _i32(start), _i32(prefix), first=_i32(first))
    assert torch.equal(again, out)
    alone, lse, status = _run(pkg, c, q, ctx, [0], [], first)  # no groups
    assert status == 0
    _check(c, q, ctx, [0], [], alone, typ, first=first, lse=lse)


def test_the_others_tables_do_not_matter_in_the_prefix(pkg):
    import torch
    rng = np.random.default_rng(8)
    n, prefix = 20, 500
    c = Cache(pkg, rng, n, 6, 2, 128, "e4m3")
    q = _q(rng, n, 8, 128, "bf16")
    ctx = rng.integers(prefix, 700, n)
    want = _run(pkg, c, q, ctx, [0, n], [prefix])
    c.tab[1:, :3] = 1 << 30  # (pages wholly in the prefix)
    got = _run(pkg, c, q, ctx, [0, n], [prefix])
    assert got[2] == 0 and torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("hd", [32, 128])
def test_wrong_groups_prefixes_lengths_and_blocks_are_nan_and_reported(pkg, hd):
    import torch
    rng = np.random.default_rng(hd + 1)
    c, q, ctx, start, prefix = _batch(pkg, rng, hd=hd)
    n = len(ctx)
    want = _run(pkg, c, q, ctx, start, prefix)
    assert want[2] == 0
    lead, shared = _groups(n, start, prefix)

    def check(got, bad):
        assert got[2] == pkg.SARA_EINVAL
        assert bool(got[0][bad].isnan().all()) and bool(got[1][bad].isnan().all())
        # (the others' sums may be cut elsewhere)
        _check(c, q, ctx, start, prefix, got[0], "bf16", lse=got[1], rows=np.flatnonzero(~bad))

    for wrong in ([2, 2, 1, 8, 8, 40, 45], [-1, 2, 7, 8, 8, 40, 45], [2, 2, 7, 8, 8, 40, 49], [2, 2, 7, 8, 1 << 30, 40, 45], [2, 2, 7, 8, -(1 << 31), 40, 45]):
        check(_run(pkg, c, q, ctx, wrong, prefix), np.ones(n, bool))
    most = _table(c, len(prefix)).shape[1] * 128
    for bad in (-1, most + 1, 2 ** 31 - 1, -2 ** 31):
        check(_run(pkg, c, q, ctx, start, prefix[:4] + [bad] + prefix[5:]), (np.arange(n) >= 8) & (np.arange(n) < 40))
    for bad in (-1, most + 1):
        wrong = ctx.copy()
        wrong[20] = bad
        check(_run(pkg, c, q, wrong, start, prefix), np.arange(n) == 20)
    for bad in (-1, c.codes.shape[0], 2 ** 31 - 1):
        was = int(c.tab[8, 2])
        c.tab[8, 2] = bad
        check(_run(pkg, c, q, ctx, start, prefix), (np.arange(n) >= 8) & (np.arange(n) < 40) & (ctx > 256))
        c.tab[8, 2] = was
    assert torch.equal(_run(pkg, c, q, ctx, start, prefix)[0], want[0])


@pytest.mark.parametrize("fmt,typ", [("e4m3", "fp16"), ("int8", "bf16")])
def test_maxima_that_move_and_scales_without_weight(pkg, fmt, typ):
    """Scores that rise and fall by hundreds from page to page, values' scales over 60 powers of two in either direction: the error is
    bounded by the largest probability times scale, not by scales that no probability goes with."""
    import torch
    rng = np.random.default_rng(4)
    n, prefix, blocks, hd = 40, 1500, 12, 64
    c = Cache(pkg, rng, n, blocks, 1, hd, fmt)
    c.scales[:, 0] *= torch.exp2(_i32(rng.integers(-2, 6, c.scales[:, 0].shape)).float())
    c.scales[:, 1] = torch.exp2(_i32(rng.integers(-30, 31, c.scales[:, 1].shape)).float())
    c.want_scales = c.scales.double().cpu().numpy()
    q = _q(rng, n, 4, hd, typ)
    ctx = rng.integers(prefix - 100, 1536, n)
    out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix])
    assert status == 0
    got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    for i in range(n):
        cut = min(prefix, ctx[i])
        parts = [oracle.read(c.want_codes, c.want_scales, c.table[0], 0, cut), oracle.read(c.want_codes, c.want_scales, c.table[i], cut, max(ctx[i], cut))]
        k, v = (np.concatenate([x[j] for x in parts]) for j in (0, 1))
        want, wl, mag, pv = oracle.attention(qn[i], k, v)
        z = np.einsum("hd,pd->hp", qn[i], k[:, 0]) / np.sqrt(hd)
        p = np.exp(z - wl[:, None])
        s = np.concatenate([c.want_scales[c.table[0]][:, 1, 0].reshape(-1)[:(cut + 31) // 32].repeat(32)[:cut],
                            c.want_scales[c.table[i]][:, 1, 0].reshape(-1).repeat(32)[cut:max(ctx[i], cut)]])
        ds = (hd + 24) * 2.0 ** -24 * mag[:, None]
        tol = HALF_STEP[typ] * np.abs(want) + (2.0 ** -11 + 2 * ds + 2.0 ** -19 + (len(k) / 4 + 64) * 2.0 ** -24) * pv \
            + len(k) * 2.0 ** -31 * 448 * (p * s).max(1)[:, None] + (2.0 ** -25 if typ == "fp16" else 0)
        ok = np.abs(want) < 65504 if typ == "fp16" else np.ones(want.shape, bool)  # (fp16 holds no more)
        assert (np.abs(got[i] - want)[ok] <= tol[ok]).all(), (i, np.max((np.abs(got[i] - want) / tol)[ok]))


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
def test_queries_of_every_size(pkg, typ):
    import torch
    rng = np.random.default_rng(6)
    n, prefix = 24, 400
    c = Cache(pkg, rng, n, 4, 2, 128, "e4m3")
    q = _q(rng, n, 8, 128, typ)
    size = torch.exp2(_i32(np.arange(n) % 12 * 3 - 24).float()) if typ == "fp16" else torch.exp2(_i32((np.arange(n) % 12 - 10) * 12).float())
    q = (q.float() * size[:, None, None]).to(q.dtype)
    q[3] = 0
    ctx = rng.integers(300, 512, n)
    out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix])
    assert status == 0
    _check(c, q, ctx, [0, n], [prefix], out, typ, lse=lse)
    broken = q.clone()  # of one sequence, and of one of its heads: the others do not notice
    broken[5], broken[7, 2, 9], broken[8, 1, 0] = float("nan"), float("inf"), float("nan")
    got, lse2, _ = _run(pkg, c, broken, ctx, [0, n], [prefix])
    assert bool(got[5].isnan().all()) and bool(got[8, 1].isnan().all())
    hit = torch.zeros(n, 8, dtype=torch.bool, device="cuda")
    hit[5], hit[7, 2], hit[8, 1] = True, True, True
    assert torch.equal(got[~hit], out[~hit]) and torch.equal(lse2[~hit], lse[~hit])


@pytest.mark.parametrize("most", [2, 7])
def test_more_groups_than_a_block_plans_at_once(pkg, most):
    rng = np.random.default_rng(7)
    sizes = rng.integers(0, most + 1, 2300)
    start = np.concatenate([[0], np.cumsum(sizes)])
    n = int(start[-1])
    prefix = rng.integers(0, 257, 2300)
    prefix = prefix[:n] if len(prefix) > n else prefix
    start = start[:len(prefix) + 1]
    ctx = rng.integers(0, 257, n)
    c = Cache(pkg, rng, 10, 2, 1, 32, "int8")
    c.table = rng.integers(0, c.codes.shape[0], (n, 2)).astype(np.int32)
    c.tab = _i32(c.table)
    q = _q(rng, n, 3, 32, "fp16")
    out, lse, status = _run(pkg, c, q, ctx, start, prefix)
    assert status == 0
    _check(c, q, ctx, start, prefix, out, "fp16", lse=lse, rows=np.unique(rng.integers(0, n, 400)))


def test_a_cache_past_32_bits(pkg):
    import torch
    rng = np.random.default_rng(9)
    n, prefix = 12, 300
    c = Cache(pkg, rng, n, 4, 8, 128, "int8")
    q = _q(rng, n, 16, 128, "bf16")
    ctx = rng.integers(250, 512, n)
    want = _run(pkg, c, q, ctx, [0, n], [prefix])
    nb, many = c.codes.shape[0], (1 << 32) // (2 * 8 * 128 * 128) + 300
    codes = torch.zeros((many, *c.codes.shape[1:]), dtype=c.codes.dtype, device="cuda")
    scales = torch.full((many, *c.scales.shape[1:]), float("nan"), device="cuda")
    codes[many - nb:], scales[many - nb:] = c.codes, c.scales
    c.codes, c.scales, c.tab = codes, scales, c.tab + (many - nb)
    got = _run(pkg, c, q, ctx, [0, n], [prefix])
    assert got[2] == 0 and torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_captured_on_another_stream_and_two_calls_at_once(pkg):
    import torch
    rng = np.random.default_rng(10)
    c, q, ctx, start, prefix = _batch(pkg, rng, hd=128)
    n, H = q.shape[:2]
    args = [_table(c, len(prefix)), _i32(ctx), _i32(start), _i32(prefix)]
    want, lse, _ = _run(pkg, c, q, ctx, start, prefix)
    new = lambda: pkg.attention_shared_kv8_workspace(n + 5, len(prefix) + 2, H, 2, 128)  # noqa: E731  (room for more)
    shared, streams = new(), [torch.cuda.Stream() for _ in range(2)]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], [torch.zeros_like(q) for _ in range(2)]
    q2 = torch.zeros_like(q)
    for g, out, x in zip(graphs, outs, (q, q2)):  # two graphs that share a workspace, replayed in turn
        with torch.cuda.graph(g, stream=streams[0]):
            pkg.attention_shared_kv8(x, c.codes, c.scales, *args, workspace=shared, out=out)
    for _ in range(3):
        q2.copy_(q.flip(0) if _ == 1 else q)
        for g in graphs:
            g.replay()
        assert torch.equal(outs[0], want)
        assert torch.equal(outs[1], want) == (_ != 1)
    spaces = [new() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):  # two streams, each its own workspace
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                outs[k].append(pkg.attention_shared_kv8(q, c.codes, c.scales, *args, workspace=spaces[k]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for k in range(2) for x in outs[k])


def test_the_same_sequence_in_every_row(pkg):
    import torch
    rng = np.random.default_rng(11)
    n = 33
    c = Cache(pkg, rng, 1, 5, 2, 64, "e4m3")
    c.table = np.repeat(c.table, n, 0)
    c.tab = _i32(c.table)
    q = _q(rng, 1, 8, 64, "fp16").expand(n, 8, 64).contiguous()
    out, lse, status = _run(pkg, c, q, [600] * n, [0, n], [555])
    assert status == 0
    _check(c, q, [600] * n, [0, n], [555], out, "fp16", lse=lse)
    assert pkg.attention_shared_kv8(q[:0], c.codes, c.scales, c.tab[:0], _i32([]), _i32([0]), _i32([])).shape == (0, 8, 64)


def _unwritten(c, used, scale):
    """Scales of blocks that hold no position of `used` (pairs of a row of the table and a range), as memory that nobody has written may have them."""
    import torch
    keep = torch.zeros(c.scales.shape[0], 4, dtype=torch.bool)
    for row, a, b in used:
        for x in range(a // 32, -(-b // 32)):
            keep[row[x // 4], x % 4] = True
    c.scales = torch.where(keep.cuda()[:, None, None, :], c.scales, torch.tensor(scale, device="cuda"))
    c.want_scales = c.scales.double().cpu().numpy()


@pytest.mark.parametrize("scale", [0.0, -0.0, -1.0, -2.0 ** 100, 2.0 ** -100, 1e-45, 2.0 ** 120, float("inf"), float("nan")])
@pytest.mark.parametrize("hd,fmt,typ", [(128, "e4m3", "bf16"), (64, "int8", "fp16"), (32, "e4m3", "bf16")])
def test_scales_of_blocks_that_nobody_attends_to_do_not_matter(pkg, hd, fmt, typ, scale):
    """Prefixes, rows and windows that end and begin in each block of a page."""
    rng = np.random.default_rng(hd)
    n, blocks = 24, 6
    for prefix, lo in ((400, 0), (390, 0), (416, 33), (449, 70), (500, 97), (16, 0), (33, 32), (512, 64), (530, 300)):
        c = Cache(pkg, rng, n, blocks, 2, hd, fmt)
        ctx = np.maximum(prefix - rng.integers(0, 3, n), lo + 1)  # rollouts just begun
        ctx[::5] = prefix + 1
        first = np.full(n, lo)
        _unwritten(c, [(c.table[0], lo, prefix)] + [(c.table[i], prefix, ctx[i]) for i in range(n) if ctx[i] > prefix], scale)
        q = _q(rng, n, 8, hd, typ)
        q[2], q[3, 1] = 0, 0
        out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix], first)
        assert status == 0
        _check(c, q, ctx, [0, n], [prefix], out, typ, first=first, lse=lse)


@pytest.mark.parametrize("typ,size", [("bf16", 0.0), ("bf16", 2.0 ** -133), ("bf16", 2.0 ** -126), ("bf16", 2.0 ** -60), ("fp16", 0.0), ("fp16", 2.0 ** -24)])
@pytest.mark.parametrize("hd", [32, 128])
def test_queries_and_keys_next_to_nothing(pkg, hd, typ, size):
    """Heads of zeros and of the least elements over keys of zeros, which have the lowest scale, and over others; rows that end in each block."""
    import torch
    rng = np.random.default_rng(hd + 1)
    n, prefix = 20, 400
    for k_scale in (2.0 ** -100, 2.0 ** -126, 0.0, 2.0 ** -8):
        c = Cache(pkg, rng, n, 5, 2, hd, "e4m3")
        c.scales[:, 0] = k_scale
        if k_scale == 2.0 ** -100:
            c.codes.view(torch.uint8)[:, 0] = 0
        c.want_codes, c.want_scales = c.values(), c.scales.double().cpu().numpy()
        q = _q(rng, n, 8, hd, typ)
        small = (q.float().sign() * size).to(q.dtype)
        q[:, ::2] = small[:, ::2]
        ctx = rng.integers(300, 430, n)
        out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix])
        assert status == 0
        _check(c, q, ctx, [0, n], [prefix], out, typ, lse=lse)


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_keys_of_a_scale_below_zero(pkg, hd):
    """None that is ever written: rows that attend to its block are NaN, or have it as a factor where they go by themselves; the others do not notice."""
    rng = np.random.default_rng(3)
    n, prefix = 40, 450
    c = Cache(pkg, rng, n, 4, 2, hd, "int8")
    q = _q(rng, n, 8, hd, "bf16")
    ctx, first = rng.integers(200, 500, n), rng.choice([0, 100, 300], n)
    first = np.minimum(first, ctx)
    want = _run(pkg, c, q, ctx, [0, n], [prefix], first)
    c.scales[c.table[0, 1], 0, :, 2] *= -1  # positions 192 .. 223
    c.want_scales = c.scales.double().cpu().numpy()
    out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix], first)
    assert status == 0
    hit = (first < 224) & (ctx > 192) & (first < ctx)
    if c.wide:
        assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    else:
        _check(c, q, ctx, [0, n], [prefix], out, "bf16", first=first, lse=lse)
    assert (out[~hit] == want[0][~hit]).all() and (lse[~hit] == want[1][~hit]).all()


@pytest.mark.parametrize("fmt,typ", [("e4m3", "bf16"), ("int8", "fp16")])
def test_wrong_blocks_that_no_row_attends_to_are_not_reported(pkg, fmt, typ):
    """Windows that leave a gap among a group's shared positions, its pages none of the cache's; then one row that attends to one of them."""
    rng = np.random.default_rng(12)
    n, prefix = 24, 900
    c = Cache(pkg, rng, n, 8, 2, 64, fmt)
    early = np.arange(n) % 2 == 0
    first = np.where(early, 0, 650)
    ctx = np.where(early, 200, 950)
    ctx[4] = 250
    c.tab[0, 2:5] = _i32([-1, 1 << 30, c.codes.shape[0]])  # positions 256 .. 639
    q = _q(rng, n, 8, 64, typ)
    out, lse, status = _run(pkg, c, q, ctx, [0, n], [prefix], first)
    assert status == 0
    _check(c, q, ctx, [0, n], [prefix], out, typ, first=first, lse=lse)
    for row, a, b in ((4, 0, 257), (7, 639, 950), (9, 639, 640)):
        first2, ctx2 = first.copy(), ctx.copy()
        first2[row], ctx2[row] = a, b
        out, lse, status = _run(pkg, c, q, ctx2, [0, n], [prefix], first2)
        assert status == pkg.SARA_EINVAL
        assert bool(out[row].isnan().all()) and bool(lse[row].isnan().all())
        _check(c, q, ctx2, [0, n], [prefix], out, typ, first=first2, lse=lse, rows=[i for i in range(n) if i != row])
