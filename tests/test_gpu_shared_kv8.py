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
    out = pkg.attention_shared_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), _i32(start), _i32(prefix), first=None if first is None else _i32(first),
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
            if fmt == "int8":
                continue
            codes[page, kv, :, slot, hd // 2] = 0xff
            hit = (first < at // 32 * 32 + 32) & (np.minimum(ctx, prefix) > at // 32 * 32) & (first < ctx)
        lse, status = torch.empty((n, 12), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = pkg.attention_shared_kv8(q, codes.view(c.codes.dtype), scales, c.tab, _i32(ctx), _i32([0, n]), _i32([prefix]), first=_i32(first), lse=lse, status=status)
        assert int(status) == 0
        for i in range(n):
            if hit[i]:
                assert bool(out[i].isnan().all()) and bool(lse[i].isnan().all()), (at, kv, how, i)
            else:
                assert torch.equal(out[i], want[0][i]) and torch.equal(lse[i], want[1][i]), (at, kv, how, i)
