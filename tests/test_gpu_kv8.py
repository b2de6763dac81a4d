"""The 8-bit paged KV cache on the GPU against its 64-bit oracle: codes and scales exactly, attention within bounds that
follow from the arithmetic."""
import numpy as np
import pytest

from oracle import kv8 as oracle

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_26253_gb300 as p
    p.load()
    return p


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn,
            "int8": torch.int8}[name]


def _i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Cache:
    """A cache on the GPU and its oracle twin, filled with the same random codes, pages handed out in random order."""

    def __init__(self, pkg, rng, n_seq, max_blocks, kvh, hd, fmt, spare=2):
        import torch
        self.pkg, self.fmt, self.kvh, self.hd = pkg, fmt, kvh, hd
        nb = n_seq * max_blocks + spare
        self.table = rng.permutation(nb)[:n_seq * max_blocks].reshape(n_seq, max_blocks).astype(np.int32)
        raw = rng.integers(-127, 128, (nb, 2, kvh, 128, hd)).astype(np.int8)
        if fmt == "e4m3":
            raw = np.where((raw & 0x7f) == 0x7f, 0, raw).astype(np.int8)  # (no NaN)
        self.codes = torch.from_numpy(raw).cuda().view(_dtype(fmt))
        self.scales = torch.exp2(torch.from_numpy(rng.integers(-9, -3, (nb, 2, kvh, 4))).float()).cuda()
        self.want_codes, self.want_scales = self.values(), self.scales.double().cpu().numpy()
        self.tab = _i32(self.table)

    def values(self):
        return self.codes.float().double().cpu().numpy()

    def write(self, k, v, pos0, start, status=None):
        self.pkg.kv8_write(self.codes, self.scales, self.tab, k, v, _i32(pos0), _i32(start), status=status)
        kn, vn = k.double().cpu().numpy(), v.double().cpu().numpy()
        for i in range(len(pos0)):
            a, b = start[i], start[i + 1]
            oracle.write(self.want_codes, self.want_scales, self.fmt, self.table[i], pos0[i], kn[a:b], vn[a:b])

    def check(self):
        assert np.array_equal(self.scales.double().cpu().numpy(), self.want_scales, equal_nan=True)
        assert np.array_equal(self.values(), self.want_codes)


def _tokens(rng, n, kvh, hd, typ, std=1.0):
    import torch
    return [torch.from_numpy(rng.standard_normal((n, kvh, hd)) * std).cuda().to(_dtype(typ)) for _ in range(2)]


LENGTHS = [1, 31, 32, 33, 0, 127, 128, 129, 300, 2]


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd,kvh", [(32, 2), (64, 1), (128, 3)])
def test_write_whole_sequences(pkg, hd, kvh, fmt, typ):
    rng = np.random.default_rng(hd + kvh)
    c = Cache(pkg, rng, len(LENGTHS), 3, kvh, hd, fmt)
    start = np.concatenate([[0], np.cumsum(LENGTHS)])
    k, v = _tokens(rng, start[-1] + 5, kvh, hd, typ)  # (rows behind the last sequence are not read)
    k[start[-1]:] = float("nan")
    c.write(k, v, np.zeros(len(LENGTHS), int), start)
    c.check()  # codes behind the tokens and pages of nobody are as they were


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_appends_raise_scales_and_keep_older_tokens(pkg, hd, fmt):
    # sizes of one token to several pages, from every place in a scale block, magnitudes that rise and fall
    rng = np.random.default_rng(hd)
    n, kvh = 4, 2
    c = Cache(pkg, rng, n, 5, kvh, hd, fmt)
    pos = np.zeros(n, int)
    kept = [[] for _ in range(n)]
    for step, std in enumerate([1, 0.1, 3, 100, 1, 1e-3, 7, 300, 2000, 1, 1]):
        new = rng.choice([0, 1, 1, 5, 31, 33, 70], n)
        start = np.concatenate([[0], np.cumsum(new)])
        k, v = _tokens(rng, start[-1], kvh, hd, "bf16", std)
        c.write(k, v, pos, start)
        for i in range(n):
            kept[i].append(k[start[i]:start[i + 1]].double().cpu().numpy())
        pos = pos + new
        c.check()
    for i in range(n):  # the promised error: half a step of the value, and one smallest step of the final scale
        x = np.concatenate(kept[i])
        got, _ = oracle.read(c.want_codes, c.want_scales, c.table[i], 0, pos[i])
        p = np.arange(pos[i])
        s = c.want_scales[c.table[i][p // 128], 0, :, p % 128 // 32][..., None]
        assert (np.abs(got - x) <= (np.abs(x) * 2.0 ** -4 + s * 2.0 ** -9 if fmt == "e4m3" else s)).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_extreme_values(pkg, fmt):
    import torch
    rng = np.random.default_rng(5)
    c = Cache(pkg, rng, 9, 1, 1, 32, fmt)
    k, v = _tokens(rng, 9 * 40, 1, 32, "bf16")
    big = torch.finfo(torch.bfloat16)
    k[0:40] = 0                                   # zeros: the lowest scale
    k[40:80] *= big.max / 8                       # up to the type's largest
    k[50, 0, 3] = big.max
    k[80:120] = big.tiny                          # far below the lowest scale's first code
    k[120, 0, 0] = float("nan")                   # one block of NaN, the next one not
    k[165, 0, 31] = float("inf")
    k[200, 0, 7] = float("-inf")
    k[240:280], k[241] = 0, 448.0                 # the top itself, and just above it
    k[280:320], k[281] = 0, 450.0
    k[320:360], k[321] = 0, 127.0
    start = np.arange(0, 361, 40)
    c.write(k, v, np.zeros(9, int), start)
    s = c.scales[:, 0, 0].cpu().numpy()[c.table[:, 0]]
    assert np.isnan(s[3, 0]) and np.isfinite(s[3, 1]) and np.isnan(s[4, 0]) and np.isnan(s[5, 0])
    assert s[0, 0] == 2.0 ** -100 and s[2, 0] == 2.0 ** -100
    bad = np.isnan(c.want_scales)
    assert np.array_equal(np.isnan(c.scales.cpu().numpy()), bad)
    ok = ~np.repeat(bad, 32, axis=3)
    assert np.array_equal(c.scales.double().cpu().numpy()[~bad], c.want_scales[~bad])
    assert np.array_equal(c.values()[ok], c.want_codes[ok])
    # a NaN block stays one when tokens join it, and is a new block when it is written from its first position on
    k2, v2 = _tokens(rng, 9, 1, 32, "bf16")
    c.write(k2, v2, np.full(9, 20), np.arange(10))
    assert np.isnan(c.scales[c.table[3, 0], 0, 0, 0].item())
    c.write(k2, v2, np.zeros(9, int), np.arange(10))
    assert np.isfinite(c.scales[c.table[:, 0], 0, 0, 0].cpu().numpy()).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_first_tokens_of_an_empty_cache_anywhere_in_a_block(pkg, fmt):
    # a sequence that begins at position 5: the block has held nothing, so its scale is the tokens' own
    rng = np.random.default_rng(24)
    codes, scales = pkg.kv8_cache(2, 2, 64, dtype=_dtype(fmt))
    k, v = _tokens(rng, 40, 2, 64, "bf16", 1e-3)
    pkg.kv8_write(codes, scales, _i32([[1]]), k, v, _i32([5]), _i32([0, 40]))
    got = pkg.kv8_read(codes, scales, _i32([[1]]), _i32([5]), _i32([0, 40]), 40, dtype=_dtype("fp32"))
    for x, y in zip((k, v), got):
        x, y = x.double().cpu().numpy(), y.double().cpu().numpy()
        parts = ((0, 27), (27, 40))  # rows of a scale block
        for a, b in parts:
            amax = np.abs(x[a:b]).max((0, 2), keepdims=True)
            # half a step of the value, or of the smallest code at a scale of at most 2 amax / top
            tol = np.abs(x[a:b]) * 2.0 ** -4 + amax / 448 * 2.0 ** -9 if fmt == "e4m3" else amax / 127
            assert (np.abs(y[a:b] - x[a:b]) <= tol).all()


def test_write_again_from_an_earlier_position(pkg):
    # tokens taken back (a rejected draft): the positions are written again, the scale only rises
    rng = np.random.default_rng(6)
    c = Cache(pkg, rng, 2, 2, 2, 64, "e4m3")
    k, v = _tokens(rng, 200, 2, 64, "fp16", 50.0)
    c.write(k, v, [0, 0], [0, 100, 200])
    k, v = _tokens(rng, 30, 2, 64, "fp16", 0.5)
    c.write(k, v, [90, 40], [0, 10, 30])
    c.check()


def test_write_views_of_a_projection_and_many_sequences(pkg):
    import torch
    rng = np.random.default_rng(7)
    n, kvh, hd = 1100, 2, 32  # three steps of the search
    c = Cache(pkg, rng, n, 1, kvh, hd, "int8")
    new = rng.choice([0, 1, 1, 2, 40], n)
    start = np.concatenate([[0], np.cumsum(new)])
    qkv = torch.from_numpy(rng.standard_normal((start[-1], 5 * kvh * hd))).cuda().half()
    k, v = (qkv[:, a * kvh * hd:(a + 1) * kvh * hd].unflatten(1, (kvh, hd)) for a in (2, 4))
    c.write(k, v, rng.integers(0, 80, n), start)
    c.check()


def test_wrong_ranges_and_blocks_are_skipped_and_reported(pkg):
    import torch
    rng = np.random.default_rng(8)
    c = Cache(pkg, rng, 6, 2, 1, 32, "e4m3")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = _tokens(rng, 60, 1, 32, "bf16")
    good = c.table.copy()
    before = c.codes.view(torch.uint8).clone()

    def call(pos0, start, table=None):
        status.zero_()
        pkg.kv8_write(c.codes, c.scales, _i32(good if table is None else table), k, v, _i32(pos0), _i32(start), status=status)
        out = tuple(torch.full((60, 1, 32), 7.0, dtype=torch.float32, device="cuda") for _ in range(2))
        code = int(status)
        status.zero_()
        pkg.kv8_read(c.codes, c.scales, _i32(good if table is None else table), _i32(pos0), _i32(start), 60, status=status, out=out)
        return code, int(status), out[0][:, 0, 0].cpu().numpy()

    start = np.arange(0, 61, 10)
    assert call(np.zeros(6), start)[:2] == (0, 0)
    c.codes.view(torch.uint8).copy_(before)
    for pos0 in (-1, 247, 2 ** 31 - 5):  # before the table, past its end, past 32 bits
        w, r, x = call([pos0, 0, 0, 0, 0, 0], start)
        assert (w, r) == (pkg.SARA_EINVAL, pkg.SARA_EINVAL)
        assert np.isnan(x[:10]).all() and np.isfinite(x[10:]).all()
    for bad in (-1, c.codes.shape[0], 2 ** 31 - 1):
        t = good.copy()
        t[2, 0] = bad
        w, r, x = call(np.zeros(6), start, t)
        assert (w, r) == (pkg.SARA_EINVAL, pkg.SARA_EINVAL)
        assert np.isnan(x[20:30]).all() and np.isfinite(np.delete(x, slice(20, 30))).all()
    # starts that leave the tokens or fall: nothing outside them is touched
    for bad in ([0, 10, 20, 30, 40, 50, 61], [0, 10, 20, 30, 40, 50, 2 ** 31 - 1], [-5, 10, 20, 30, 40, 50, 60], [0, 30, 20, 30, 40, 50, 60],
                [0, 60, 0, 60, 0, 60, 0], [60, 50, 40, 30, 20, 10, 0], [0, 2 ** 31 - 1, -2 ** 31, 3, 4, 5, 6], [0, 10, 20, 30, 40, 61, 60]):
        w, r, x = call(np.zeros(6), bad)
        assert (w, r) == (pkg.SARA_EINVAL, pkg.SARA_EINVAL)
    spare = np.setdiff1d(np.arange(c.codes.shape[0]), good[:, 0])
    assert torch.equal(c.codes.view(torch.uint8)[spare], before[spare])


@pytest.mark.parametrize("typ", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd,kvh", [(32, 3), (64, 2), (128, 1)])
def test_read(pkg, hd, kvh, fmt, typ):
    import torch
    rng = np.random.default_rng(hd)
    c = Cache(pkg, rng, 7, 4, kvh, hd, fmt)
    pos0 = np.array([0, 5, 31, 127, 100, 384, 32])
    lens = np.array([1, 300, 2, 130, 0, 128, 64])
    start = np.concatenate([[0], np.cumsum(lens)])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    total = int(start[-1]) + 3
    out = tuple(torch.full((total, 2 * kvh, hd), 7.0, dtype=_dtype(typ), device="cuda")[:, :kvh] for _ in range(2))
    k, v = pkg.kv8_read(c.codes, c.scales, c.tab, _i32(pos0), _i32(start), total, out=out, status=status)
    assert int(status) == 0
    for i in range(7):
        for got, want in zip((k, v), oracle.read(c.want_codes, c.want_scales, c.table[i], pos0[i], pos0[i] + lens[i])):
            assert torch.equal(got[start[i]:start[i + 1]].cpu(), torch.from_numpy(want).to(_dtype(typ)))
    assert (k[start[-1]:] == 7).all() and (v[start[-1]:] == 7).all()
    k2, v2 = pkg.kv8_read(c.codes, c.scales, c.tab, _i32(pos0), _i32(start), int(start[-1]), dtype=_dtype(typ))
    assert torch.equal(k2, k[:start[-1]]) and torch.equal(v2, v[:start[-1]])


# ------------------------------------------------------------------------------------------------ attention
def _check_attention(c, q, ctx, out, typ, first=None, lse=None, chains=4):
    """Bounds: scores off by (hd + 4 + |s| terms) roundings of 32 bits of sum |q k| / sqrt(hd); probabilities in 21 bits or more
    and multiples of 2^-32 of the maximum; sums of at most a quarter (1 / chains) of the positions in a chain; the result rounded once."""
    got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    for i, n in enumerate(ctx):
        a = 0 if first is None else first[i]
        k, v = oracle.read(c.want_codes, c.want_scales, c.table[i], a, max(a, n))
        want, wl, mag, pv = oracle.attention(qn[i], k, v)
        ds = (c.hd + 8) * 2.0 ** -24 * mag[:, None]
        vmax = np.abs(v).max() if len(v) else 0.0
        tol = HALF_STEP[typ] * np.abs(want) + (2 * ds + 2.0 ** -20 + (len(k) / chains + 32) * 2.0 ** -24) * pv \
            + max(1, len(k)) * 2.0 ** -32 * vmax + 2.0 ** -25
        ok = bool((np.abs(got[i] - want) <= tol).all())
        assert ok, (i, n, np.max(np.abs(got[i] - want) - tol))
        if lse is not None:
            l = lse[i].double().cpu().numpy()
            if n <= a:
                assert (l == -np.inf).all()
            else:
                assert (np.abs(l - wl) <= ds[:, 0] + (len(k) / chains + 32) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(wl))).all()


def _q(rng, n, H, hd, typ, std=1.0):
    import torch
    return torch.from_numpy(rng.standard_normal((n, H, hd)) * std).cuda().to(_dtype(typ))


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 0, 100, 127, 128, 129, 255, 256, 257, 700]


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,kvh,hd", [(6, 1, 128), (8, 1, 64), (2, 1, 32), (4, 4, 128), (9, 3, 32), (14, 2, 64), (15, 3, 128),
                                      (8, 2, 128)])
def test_attention_edges(pkg, H, kvh, hd, fmt, typ):
    import torch
    rng = np.random.default_rng(H + hd)
    c = Cache(pkg, rng, len(EDGES), 6, kvh, hd, fmt)
    q = _q(rng, len(EDGES), H, hd, typ)
    lse = torch.empty((len(EDGES), H), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(EDGES), lse=lse, status=status)
    assert int(status) == 0
    _check_attention(c, q, EDGES, out, typ, lse=lse)


# the first visible position before, in and behind a page, a scale block, a warp's step; rows without a position
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_attention_window(pkg, hd, fmt):
    import torch
    rng = np.random.default_rng(hd)
    ctx = [700, 700, 700, 300, 300, 129, 129, 17, 50, 0, 640, 5]
    first = [0, 1, 127, 128, 299, 128, 129, 16, 700, 0, 500, 2 ** 31 - 1]
    c = Cache(pkg, rng, len(ctx), 6, 2, hd, fmt)
    q = _q(rng, len(ctx), 12, hd, "fp16")
    lse = torch.empty((len(ctx), 12), device="cuda")
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), first=_i32(first), lse=lse)
    _check_attention(c, q, ctx, out, "fp16", [min(f, 768) for f in first], lse)


# one long row, few and many: work split over a row, whole rows, rows that end inside a CTA's share
@pytest.mark.parametrize("ctxs", [[12288], [5000, 1, 9000], list(range(1, 200)), [128] * 300, [40] * 700])
def test_attention_lengths_and_rows(pkg, ctxs):
    rng = np.random.default_rng(len(ctxs))
    c = Cache(pkg, rng, len(ctxs), -(-max(ctxs) // 128), 2, 64, "e4m3")
    q = _q(rng, len(ctxs), 12, 64, "bf16")
    ws = pkg.attention_kv8_workspace(len(ctxs), 12, 2, 64)
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctxs), workspace=ws)
    _check_attention(c, q, ctxs, out, "bf16")
    for _ in range(3):  # the same bits again, from the same workspace
        import torch
        assert torch.equal(out, pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctxs), workspace=ws))


def _shared_pages(c, rng, n, blocks):
    """Another table for the cache: n rows of `blocks` of its pages, shared at random."""
    c.table = rng.integers(0, c.codes.shape[0], (n, blocks)).astype(np.int32)
    c.tab = _i32(c.table)


# many rows, of all lengths, seen from 0 or from some position on: shares of a warp from 1,600 (row, KV head) pairs on, those of a CTA
# below; rows counted by every warp for itself (up to 32) or in parts of 32 or 64
@pytest.mark.parametrize("fmt,typ", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("n,H,kvh,hd", [(1700, 6, 1, 128), (820, 16, 2, 64), (410, 12, 4, 32), (211, 64, 8, 128), (1600, 1, 1, 32), (1599, 1, 1, 32),
                                        (2100, 3, 1, 64), (33, 4, 2, 64), (1025, 2, 1, 128)])
def test_attention_many_rows(pkg, n, H, kvh, hd, fmt, typ):
    import torch
    rng = np.random.default_rng(n + hd)
    c = Cache(pkg, rng, 20, 3, kvh, hd, fmt)
    _shared_pages(c, rng, n, 6)
    ctx = rng.choice(EDGES, n)
    first = np.where(rng.random(n) < 0.5, 0, rng.integers(0, 300, n))
    q, lse, status = _q(rng, n, H, hd, typ), torch.empty((n, H), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = pkg.attention_kv8_workspace(n, H, kvh, hd)
    for f in (None, first):
        call = lambda: pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), first=None if f is None else _i32(f),  # noqa: E731
                                                workspace=ws, lse=lse, status=status)
        out = call()
        assert int(status) == 0
        _check_attention(c, q, ctx, out, typ, f, lse=lse, chains=1)
        assert torch.equal(out, call())


# one row that most of the shares hold, among many of one position: joins over three levels; the workspace then serves a batch of few rows
@pytest.mark.parametrize("hd,long", [(128, 20000), (64, 60000), (32, 300)])
def test_attention_one_long_row_among_many(pkg, hd, long):
    import torch
    rng = np.random.default_rng(hd)
    n = 1700
    c = Cache(pkg, rng, 1, 40, 1, hd, "e4m3")
    _shared_pages(c, rng, n, -(-long // 128))
    q, ws = _q(rng, n, 5, hd, "fp16"), pkg.attention_kv8_workspace(n, 5, 1, hd)
    few, ctx = None, np.ones(n, dtype=np.int64)
    for at in (900, 0, n - 1):
        ctx[:] = 1
        ctx[at] = long
        out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), workspace=ws)
        _check_attention(c, q, ctx, out, "fp16", chains=1)
        assert torch.equal(out, pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), workspace=ws))
        out = pkg.attention_decode_kv8(q[:3], c.codes, c.scales, c.tab[:3], _i32([long, 5, long]), workspace=ws)
        if few is None:
            _check_attention(c, q[:3], [long, 5, long], out, "fp16")
            few = out
        assert torch.equal(out, few)


def test_attention_many_rows_some_of_them_wrong(pkg):
    import torch
    rng = np.random.default_rng(23)
    n, H, kvh, hd = 900, 4, 2, 64
    c = Cache(pkg, rng, 10, 4, kvh, hd, "int8")
    _shared_pages(c, rng, n, 4)
    q, ctx = _q(rng, n, H, hd, "bf16"), rng.integers(1, 513, n)
    first = np.zeros(n)
    table = c.table.copy()
    ctx[[3, 500]] = [513, -1]
    first[[77, 899]] = [-1, -2 ** 31]
    ctx[[200, 640]] = 300
    table[200, 2], table[640, 0] = -1, c.codes.shape[0]
    table[300, 3], ctx[300] = 2 ** 31 - 1, 384  # (a page that is not read)
    status, lse = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((n, H), device="cuda")
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, _i32(table), _i32(ctx), first=_i32(first), lse=lse, status=status)
    assert int(status) == pkg.SARA_EINVAL
    right = np.ones(n, dtype=bool)
    right[[3, 500, 77, 899, 200, 640]] = False
    keep = torch.from_numpy(right).cuda()
    assert torch.isnan(out[~keep]).all() and torch.isnan(lse[~keep]).all()
    c.table = c.table[right]
    _check_attention(c, q[keep], ctx[right], out[keep], "bf16", lse=lse[keep], chains=1)


# scores that rise along the row (a maximum that moves), fall, or are large and far apart; values whose scales differ by 2^60
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", ["rising", "falling", "large", "scales"])
def test_attention_moving_maximum_and_scales(pkg, kind, fmt):
    import torch
    rng = np.random.default_rng(11)
    c = Cache(pkg, rng, 2, 8, 1, 128, fmt)
    q = _q(rng, 2, 6, 128, "bf16")
    if kind in ("rising", "falling"):
        e = torch.arange(32).float()
        e = torch.exp2((e if kind == "rising" else 31 - e) / 4 - 13).view(8, 4).cuda()
        for i in range(2):
            c.scales[c.table[i], 0, 0] = torch.exp2(torch.round(torch.log2(e)))
        q = q.abs()
        c.codes[:, 0] = c.codes[:, 0].float().abs().to(c.codes.dtype)
    elif kind == "large":
        q = q * 30
    else:
        c.scales[:, 1] = torch.exp2(torch.randint(-60, 1, c.scales[:, 1].shape, generator=torch.Generator().manual_seed(1)).float()).cuda()
    c.want_codes, c.want_scales = c.values(), c.scales.double().cpu().numpy()
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32([1000, 1024]))
    _check_attention(c, q, [1000, 1024], out, "bf16")


# Blocks of values with a large scale and next to no weight, first or in the middle of what a warp sees, among blocks that hold the weight
# with scales 2^24 to 2^100 smaller (or 2^200, where the others' weight of 2^-392 is nothing beside it); shares of a CTA and of a warp.
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("n,blocks", [(160, 8), (1700, 4), (3, 30)])
@pytest.mark.parametrize("part", [0, 2])
@pytest.mark.parametrize("apart", [24, 40, 60, 100, 200])
def test_attention_values_of_large_scales_without_weight(pkg, apart, part, n, blocks, fmt):
    import torch
    rng = np.random.default_rng(apart + part)
    H, hd = 4, 128
    c = Cache(pkg, rng, 24, 1, 1, hd, fmt, spare=0)
    _shared_pages(c, rng, n, blocks)
    q = _q(rng, n, H, hd, "bf16", 0.1) + 1.0
    c.scales[:, 0] = 2.0 ** -5                                    # keys: scores of a few units
    c.codes[:, 0, :, 32 * part:32 * part + 32] = torch.tensor(-96.0, device="cuda").to(c.codes.dtype)
    far = apart == 200
    c.scales[:, 0, :, part] = 2.0 ** (-2 if far else -4)          # ... and of -96 2^-4 sqrt(128) = -68, or -272
    c.scales[:, 1] = 2.0 ** (-100 if far else -apart)
    c.scales[:, 1, :, part] = 2.0 ** 100 if far else 1.0
    c.want_codes, c.want_scales = c.values(), c.scales.double().cpu().numpy()
    ctx = rng.integers(1, 128 * blocks + 1, n)
    ctx[: n // 2] = 128 * blocks
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx))
    got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    for i in rng.permutation(n)[:40]:
        k, v = oracle.read(c.want_codes, c.want_scales, c.table[i], 0, ctx[i])
        want, _, mag, pv = oracle.attention(qn[i], k, v)
        # probabilities: 21 bits or more, or multiples of 2^-31 of the largest probability times its scale, for which pv has at least
        # p scale / 2^9 of each value that is not 0; below 2^-126 of the largest nothing
        p = np.exp((k[:, 0] @ qn[i].T) / np.sqrt(hd))
        p /= p.sum(0)
        scale = c.want_scales[c.table[i][np.arange(ctx[i]) // 128], 1, 0, np.arange(ctx[i]) % 128 // 32]
        top = (p * scale[:, None]).max(0)
        ds = (hd + 8) * 2.0 ** -24 * mag[:, None]
        tol = HALF_STEP["bf16"] * np.abs(want) + (2 * ds + 2.0 ** -20 + (ctx[i] + 32) * 2.0 ** -24) * pv \
            + 2.0 ** -31 * top[:, None] * np.abs(v[:, 0] / scale[:, None]).sum(0) + (not far) * 2.0 ** -126 * np.abs(v[:, 0]).sum(0)
        assert (np.abs(got[i] - want) <= tol).all(), (i, ctx[i], np.max(np.abs(got[i] - want) - tol))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attention_reads_nothing_behind_or_before(pkg, fmt):
    # NaN codes and scales outside [first, ctx): in pages of nobody, behind the row's end, before its window
    import torch
    rng = np.random.default_rng(12)
    c = Cache(pkg, rng, 3, 3, 2, 64, fmt)
    ctx, first = [200, 257, 90], [0, 160, 64]
    q = _q(rng, 3, 8, 64, "bf16")
    keep = np.zeros((c.codes.shape[0], 128), bool)
    for i in range(3):
        for p in range(first[i], ctx[i]):
            keep[c.table[i, p // 128], p % 128] = True
    raw = c.codes.view(torch.uint8)
    drop = torch.from_numpy(~keep).cuda()[:, None, None, :, None]
    raw.copy_(torch.where(drop, torch.full_like(raw, 0x7f), raw))
    blocks = torch.from_numpy(keep.reshape(-1, 4, 32).any(-1)).cuda()[:, None, None, :]
    c.scales.copy_(torch.where(blocks, c.scales, torch.full_like(c.scales, float("nan"))))
    tab = c.table.copy()
    tab[0, 2:], tab[2, 1:], tab[1, 0] = -1, 2 ** 31 - 1, -7  # (unused entries may hold anything)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, _i32(tab), _i32(ctx), first=_i32(first), status=status)
    assert int(status) == 0
    _check_attention(c, q, ctx, out, "bf16", first)


def test_attention_nan_reaches_its_rows_alone(pkg):
    import torch
    rng = np.random.default_rng(13)
    c = Cache(pkg, rng, 3, 2, 2, 32, "e4m3")
    c.scales[c.table[0, 1], 0, 1, 2] = float("nan")    # keys of row 0, KV head 1
    c.scales[c.table[1, 0], 1, 0, 0] = float("nan")    # values of row 1, KV head 0
    c.codes.view(torch.uint8)[c.table[2, 0], 0, 0, 5, 3] = 0x7f  # one NaN code of row 2, KV head 0
    q = _q(rng, 3, 4, 32, "bf16")
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32([250, 250, 250]))
    nan = out.isnan().all(-1).cpu().numpy()
    assert np.array_equal(nan, [[False, False, True, True], [True, True, False, False], [True, True, False, False]])
    assert np.array_equal(out.isnan().any(-1).cpu().numpy(), nan)


def test_attention_wrong_rows_give_nan_and_are_reported(pkg):
    import torch
    rng = np.random.default_rng(14)
    c = Cache(pkg, rng, 4, 3, 2, 128, "int8")
    q = _q(rng, 4, 4, 128, "fp16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = pkg.attention_kv8_workspace(4, 4, 2, 128)
    good = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32([300, 384, 5, 0]), workspace=ws)

    def rows(ctx=(300, 384, 5, 0), first=(0, 0, 0, 0), table=None):
        status.zero_()
        lse = torch.zeros((4, 4), device="cuda")
        out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab if table is None else _i32(table), _i32(ctx), first=_i32(first),
                                       workspace=ws, lse=lse, status=status)
        nan = out.isnan().flatten(1).any(1).cpu().numpy()
        assert np.array_equal(nan, out.isnan().flatten(1).all(1).cpu().numpy())
        assert np.array_equal(nan, lse.isnan().all(1).cpu().numpy())
        assert torch.equal(out[torch.from_numpy(~nan)], good[torch.from_numpy(~nan)])
        return int(status), nan.tolist()

    assert rows() == (0, [False] * 4)
    for bad in (-1, 385, 2 ** 31 - 1, -2 ** 31):
        assert rows(ctx=(300, bad, 5, 0)) == (pkg.SARA_EINVAL, [False, True, False, False])
    assert rows(first=(0, 0, -1, 0)) == (pkg.SARA_EINVAL, [False, False, True, False])
    for bad in (-1, c.codes.shape[0], 2 ** 31 - 1):
        t = c.table.copy()
        t[0, 2], t[2, 1] = bad, bad  # row 2 does not reach its second entry
        assert rows(table=t) == (pkg.SARA_EINVAL, [True, False, False, False])
    assert rows() == (0, [False] * 4)


def test_cache_past_32_bits(pkg):
    # pages that begin beyond 2^32 bytes
    import torch
    kvh, hd, nb = 8, 128, 18000
    codes = torch.empty((nb, 2, kvh, 128, hd), dtype=torch.int8, device="cuda")
    scales = torch.ones((nb, 2, kvh, 4), device="cuda")
    rng = np.random.default_rng(15)
    table = np.array([[17999, 3], [17000, 17998]])
    k, v = _tokens(rng, 400, kvh, hd, "fp16")
    pkg.kv8_write(codes, scales, _i32(table), k, v, _i32([0, 0]), _i32([0, 200, 400]))
    a, b = pkg.kv8_read(codes, scales, _i32(table), _i32([0, 0]), _i32([0, 200, 400]), 400, dtype=torch.float32)
    c = type("C", (), {"hd": hd, "table": np.array([[0, 1], [2, 3]])})()
    c.want_codes, c.want_scales = np.zeros((4, 2, kvh, 128, hd)), np.ones((4, 2, kvh, 4))
    for i in range(2):
        oracle.write(c.want_codes, c.want_scales, "int8", c.table[i], 0, k[200 * i:200 * i + 200].double().cpu().numpy(),
                     v[200 * i:200 * i + 200].double().cpu().numpy())
        for got, want in zip((a, b), oracle.read(c.want_codes, c.want_scales, c.table[i], 0, 200)):
            assert np.array_equal(got[200 * i:200 * i + 200].double().cpu().numpy(), want)
    q = _q(rng, 2, 32, hd, "bf16")
    _check_attention(c, q, [200, 199], pkg.attention_decode_kv8(q, codes, scales, _i32(table), _i32([200, 199])), "bf16")


def test_long_row(pkg):
    # 150,000 positions of one row, in a page order of its own
    rng = np.random.default_rng(16)
    c = Cache(pkg, rng, 1, 1172, 1, 32, "int8")
    q = _q(rng, 1, 4, 32, "fp16")
    _check_attention(c, q, [150000], pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32([150000])), "fp16")


def test_wider_tables_rows_before_the_first_sequence_and_strided_queries(pkg):
    # the table is a part of a wider one; the first sequence's tokens do not begin at row 0; q is a part of a projection's rows
    import torch
    rng = np.random.default_rng(20)
    n, kvh, hd, H = 3, 2, 64, 8
    c = Cache(pkg, rng, n, 2, kvh, hd, "e4m3")
    wide = torch.full((n, 7), -5, dtype=torch.int32, device="cuda")
    wide[:, 2:4] = c.tab
    c.tab = wide[:, 2:4]
    k, v = _tokens(rng, 200, kvh, hd, "bf16")
    k[:9], v[:9] = float("nan"), float("nan")
    c.write(k, v, [0, 0, 0], [9, 110, 110, 200])
    c.check()
    qkv = _q(rng, n, 2 * H, hd, "bf16")
    q = qkv[:, H // 2:H // 2 + H]
    ctx = [101, 0, 90]
    _check_attention(c, q, ctx, pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx)), "bf16")
    out = tuple(torch.full((200, kvh, hd), 7.0, device="cuda") for _ in range(2))
    pkg.kv8_read(c.codes, c.scales, c.tab, _i32([0, 0, 0]), _i32([9, 110, 110, 200]), 200, out=out)
    assert (out[0][:9] == 7).all() and torch.isfinite(out[0]).all()
    want, _ = oracle.read(c.want_codes, c.want_scales, c.table[2], 0, 90)
    assert np.array_equal(out[0][110:].double().cpu().numpy(), want)


def test_rollouts_share_their_prompts_pages(pkg):
    # the same full pages at the head of several rows, a page of its own behind them for each
    rng = np.random.default_rng(21)
    n, kvh, hd = 6, 2, 128
    c = Cache(pkg, rng, n, 3, kvh, hd, "int8")
    c.table[1:, :2] = c.table[0, :2]
    c.tab = _i32(c.table)
    k, v = _tokens(rng, 256, kvh, hd, "bf16")
    one = c.tab
    c.tab = _i32(c.table[:1])
    c.write(k, v, [0], [0, 256])
    c.tab = one
    for t in range(3):
        k, v = _tokens(rng, n, kvh, hd, "bf16")
        c.write(k, v, [256 + t] * n, np.arange(n + 1))
    c.check()
    q = _q(rng, n, 12, hd, "bf16")
    _check_attention(c, q, [259] * n, pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32([259] * n)), "bf16")


@pytest.mark.parametrize("n", [1, 5, 700, 2000])
def test_batches_without_a_position(pkg, n):
    import torch
    codes, scales = pkg.kv8_cache(4, 2, 64)
    table, zero = _i32(np.zeros((n, 2))), _i32(np.zeros(n))
    q, lse = torch.ones((n, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros((n, 4), device="cuda")
    out = pkg.attention_decode_kv8(q, codes, scales, table, zero, lse=lse)
    assert (out == 0).all() and (lse == -np.inf).all()
    none = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    pkg.kv8_write(codes, scales, table, none, none, zero, _i32(np.zeros(n + 1)))
    k, v = pkg.kv8_read(codes, scales, table, zero, _i32(np.zeros(n + 1)), 0)
    assert k.shape == v.shape == (0, 2, 64)


def test_batches_of_no_sequence(pkg):
    import torch
    codes, scales = pkg.kv8_cache(4, 2, 64)
    table, none = torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    pkg.kv8_write(codes, scales, table, x, x, none, _i32([0]))
    pkg.kv8_read(codes, scales, table, none, _i32([0]), 0)
    assert pkg.attention_decode_kv8(torch.empty((0, 4, 64), dtype=torch.float16, device="cuda"), codes, scales, table, none).shape == (0, 4, 64)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
def test_queries_of_every_size(pkg, typ):
    # a NaN or an infinity in one head leaves the others; queries of zero, near the type's ends, far apart within a row
    import torch
    rng = np.random.default_rng(22)
    c = Cache(pkg, rng, 5, 4, 2, 128, "e4m3")
    q = _q(rng, 5, 8, 128, typ)
    top = float(torch.finfo(q.dtype).max)
    ctx = [500] * 5
    q[0, 1, 3], q[1, 6, 100] = float("nan"), float("inf")
    q[2] = 0
    q[3, 0] *= 2.0 ** -20 if typ == "fp16" else 2.0 ** -120
    q[3, 1, 5] = 0.01 * top if typ == "fp16" else 300.0
    q[4, :, 1:] *= 2.0 ** -10
    out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx))
    bad = out.isnan().any(-1).cpu().numpy()
    assert bad[0].tolist() == [i == 1 for i in range(8)] and bad[1].tolist() == [i == 6 for i in range(8)] and not bad[2:].any()
    q[0, 1, 3], q[1, 6, 100] = 0.5, 0.25
    good = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx))
    keep = torch.from_numpy(~bad).cuda()
    assert torch.equal(out[keep], good[keep])
    _check_attention(c, q, ctx, good, typ)


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_prompts_then_decode_steps(pkg, fmt):
    """Prompts are written, then each step appends one token per row and attends over what the cache holds; a finished row
    leaves the batch (ctx 0); at the end the whole history is read back."""
    import torch
    rng = np.random.default_rng(17)
    n, H, kvh, hd, steps = 5, 12, 2, 128, 40
    c = Cache(pkg, rng, n, 3, kvh, hd, fmt)
    lens = np.array([30, 1, 127, 250, 64])
    start = np.concatenate([[0], np.cumsum(lens)])
    k, v = _tokens(rng, start[-1], kvh, hd, "bf16")
    c.write(k, v, np.zeros(n, int), start)
    ws = pkg.attention_kv8_workspace(n, H, kvh, hd)
    pos = lens.copy()
    for t in range(steps):
        k, v = _tokens(rng, n, kvh, hd, "bf16", 1.0 + t / 4)
        c.write(k, v, pos, np.arange(n + 1))
        pos += 1
        ctx = pos.copy()
        if t > 20:
            ctx[1] = 0
        q = _q(rng, n, H, hd, "bf16")
        out = pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx), workspace=ws)
        if t % 13 == 0 or t == steps - 1:
            c.check()
            _check_attention(c, q, ctx, out, "bf16")
    start = np.concatenate([[0], np.cumsum(pos)])
    a, b = pkg.kv8_read(c.codes, c.scales, c.tab, _i32(np.zeros(n)), _i32(start), int(start[-1]), dtype=torch.float32)
    for i in range(n):
        for got, want in zip((a, b), oracle.read(c.want_codes, c.want_scales, c.table[i], 0, pos[i])):
            assert np.array_equal(got[start[i]:start[i + 1]].double().cpu().numpy(), want)


def test_step_captured_and_replayed_on_another_stream(pkg):
    """One decode step (append, attention) as a CUDA graph; its lengths advance on the device between replays."""
    import torch
    rng = np.random.default_rng(18)
    n, H, kvh, hd = 3, 8, 2, 64
    c = Cache(pkg, rng, n, 3, kvh, hd, "e4m3")
    k, v = _tokens(rng, n, kvh, hd, "fp16")
    q = _q(rng, n, H, hd, "fp16")
    pos, ctx, start = _i32([0, 100, 250]), _i32([1, 101, 251]), _i32(np.arange(n + 1))
    ws, out = pkg.attention_kv8_workspace(n, H, kvh, hd), torch.empty_like(q)

    def step():
        pkg.kv8_write(c.codes, c.scales, c.tab, k, v, pos, start)
        pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, ctx, workspace=ws, out=out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for t in range(6):
        kt, vt = _tokens(rng, n, kvh, hd, "fp16", 1.0 + t)
        k.copy_(kt)
        v.copy_(vt)
        at = pos.cpu().numpy()
        graph.replay()
        for i in range(n):
            oracle.write(c.want_codes, c.want_scales, "e4m3", c.table[i], int(at[i]), kt[i:i + 1].double().cpu().numpy(),
                         vt[i:i + 1].double().cpu().numpy())
        c.check()
        _check_attention(c, q, at + 1, out, "fp16")
        pos += 1
        ctx += 1


def test_two_calls_at_once(pkg):
    # two streams, each with its own workspace
    import torch
    rng = np.random.default_rng(19)
    c = Cache(pkg, rng, 8, 40, 2, 128, "int8")
    ctx = [5000] * 8
    qs = [_q(rng, 8, 12, 128, "bf16") for _ in range(2)]
    want = [pkg.attention_decode_kv8(q, c.codes, c.scales, c.tab, _i32(ctx)) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [pkg.attention_kv8_workspace(8, 12, 2, 128) for _ in range(2)]
    dctx = _i32(ctx)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                got[j].append(pkg.attention_decode_kv8(qs[j], c.codes, c.scales, c.tab, dctx, workspace=ws[j]))
    torch.cuda.synchronize()
    for j in range(2):
        assert all(torch.equal(x, want[j]) for x in got[j])
