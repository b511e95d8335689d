"""The paged key-value cache and the attention over it against 64-bit references.

Bounds of the attention, u = 2^-24: a score sums head_dim <= 256 exact products
in FP32 (at most 64 of them one after another, whatever the order inside an
instruction, which may cut off instead of rounding: 2 u each) and is scaled by a
product of three factors, so that it is off by 136 u of the largest sum of |q k|
scale; 2^x by the hardware is within 2^-22 (relative), the weight's two words
within 2^-17.  A position's weight is off by that twice (it is divided by the sum
of all), and the sums over n positions add at most n / 64 + 32 terms one after
another (64 positions a step, four warps and the join), cut off: 2 u each.  All
that is relative to the weighted sum of |v|; the output's rounding is half its
eps.  Eight bits: the stored entries are exact inputs, times their FP32 scales
(one rounding more, in what is counted)."""
import math

import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


def randn(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def f64(t):
    return t.detach().float().double().cpu().numpy()


def half_eps(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def close(got, want, bound):
    got, want, bound = np.broadcast_arrays(got, want, bound)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - want) <= bound)
    bad &= ~((got == want) & np.isinf(want))
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], bound[bad][:5])


def cache_of(pmpe, pages, page, heads, dim, dtype, seed):
    """A cache with something in every entry."""
    c = pmpe.KvCache.empty(pages, page, heads, dim, dtype)
    for n, t in enumerate((c.k, c.v)):
        t.copy_(randn(tuple(t.shape), seed + n).to(dtype))
    if dtype == E4M3:
        for n, t in enumerate((c.k_scale, c.v_scale)):
            t.copy_(torch.exp(randn(tuple(t.shape), seed + 2 + n)) / 8)
    return c


def plan(lengths, page, seed, width=None, pages=None):
    """A table over shuffled pages; entries that are not needed are out of range."""
    need = [-(-max(n, 0) // page) for n in lengths]
    width = width or max(1, *need)
    pages = pages or sum(need) + 3
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), width), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        n = min(n, width)
        table[b, :n] = order[at:at + n]
        at += n
    return table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), pages


def state(c):
    return [t.clone() for t in c._held if t is not None]


def bits(t):
    return t.contiguous().view(torch.uint8)


def check_append(pmpe, c, k, v, table, lengths, cu=None):
    before = state(c)
    c.append(k, v, table, lengths, cu_seqlens=cu)
    torch.cuda.synchronize()
    pages, heads, page, dim = c.k.shape
    cun = None if cu is None else cu.cpu().numpy()
    entries = ref.kv_entries(table.cpu().numpy(), lengths.cpu().numpy(), cun, k.shape[0], pages, page)
    for n, (x, was) in enumerate(((k, before[0]), (v, before[1]))):
        pool = (c.k, c.v)[n]
        x64 = f64(x)
        rest = torch.ones((pages, page), dtype=torch.bool)
        for r, at in enumerate(entries):
            if at is not None:
                rest[at] = False
        live = [r for r, at in enumerate(entries) if at is not None]
        pg, pl = [entries[r][0] for r in live], [entries[r][1] for r in live]
        got = f64(pool)[pg, :, pl]
        if c.k.dtype != E4M3:
            dt = c.k.dtype
            big = np.abs(x64[live]) > torch.finfo(dt).max
            close(got[~big], x64[live][~big], half_eps(dt) * np.abs(x64[live][~big]) + smallest(dt))
        else:
            s = f64((c.k_scale, c.v_scale)[n])[pg, :, pl]
            exact = np.maximum(np.abs(x64[live]).max(2) / 448.0, 2.0 ** -126)
            close(s, exact, 2 * U * exact)
            q = x64[live] / exact[..., None]
            # half a step of e4m3 (and what a value next to the middle of two takes)
            close(got, q, (2.0 ** -4 + 2.0 ** -20) * np.abs(q) + 2.0 ** -10)
            assert (np.abs(got - ref.e4m3(q)) > 1e-9).mean() < 1e-3
            rest_s = rest[:, None].expand(pages, heads, page).cuda()
            assert torch.equal(bits((c.k_scale, c.v_scale)[n][rest_s]), bits(before[2 + n][rest_s]))
        keep = rest[:, None].expand(pages, heads, page).cuda()
        assert torch.equal(bits(pool)[keep.unsqueeze(-1).expand(-1, -1, -1, bits(pool).shape[-1])], bits(was)[keep.unsqueeze(-1).expand(-1, -1, -1, bits(was).shape[-1])])
    return entries


def check_read(pmpe, c, table, lengths, cu, rows, dtype):
    k, v = c.read(table, lengths, cu_seqlens=cu, rows=rows, dtype=dtype)
    torch.cuda.synchronize()
    pages, heads, page, dim = c.k.shape
    n = rows if rows is not None else table.shape[0]
    entries = ref.kv_entries(table.cpu().numpy(), lengths.cpu().numpy(), None if cu is None else cu.cpu().numpy(), n, pages, page)
    for i, got in enumerate((k, v)):
        assert got.dtype == dtype and got.shape == (n, heads, dim)
        pool = f64((c.k, c.v)[i])
        if c.k.dtype == E4M3:
            pool = pool * f64((c.k_scale, c.v_scale)[i])[..., None]
        want = np.zeros((n, heads, dim))
        for r, at in enumerate(entries):
            if at is not None:
                want[r] = pool[at[0], :, at[1]]
        ok = np.abs(want) < torch.finfo(dtype).max
        close(f64(got)[ok], want[ok], (half_eps(dtype) + U) * np.abs(want[ok]) + smallest(dtype))


def cu_of(news):
    return torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()


CACHES = [BF16, F16, E4M3]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("src", [BF16, F16, F32])
@pytest.mark.parametrize("dim,heads,page", [(16, 1, 1), (64, 3, 16), (80, 2, 24), (128, 4, 64), (256, 2, 7), (192, 5, 100)])
def test_append_and_read(pmpe, cache, src, dim, heads, page):
    news, before = [3, 0, 1, 40, 7], [0, 9, 130, 5, 63]
    table, lengths, pages = plan([a + b for a, b in zip(news, before)], page, dim)
    c = cache_of(pmpe, pages, page, heads, dim, cache, 1)
    T, pad = sum(news), 3
    scale = torch.exp(randn((T + pad, 1, 1), 8))
    # keys and values inside wider rows
    wide = (randn((T + pad, 5 * heads, dim), 9) * scale).to(src)
    k, v = wide[:, heads:2 * heads], wide[:, 3 * heads:4 * heads]
    check_append(pmpe, c, k, v, table, lengths, cu_of(news))
    check_read(pmpe, c, table, lengths, cu_of(news), T + pad, src)
    check_read(pmpe, c, table, lengths, cu_of([a + b for a, b in zip(news, before)]), sum(news) + sum(before), BF16)
    # one token each
    news1 = randn((5, heads, dim), 10, src)
    check_append(pmpe, c, news1, news1 * 2, table, lengths)
    check_read(pmpe, c, table, lengths, None, None, F32)


@pytest.mark.parametrize("cache", CACHES)
def test_append_of_any_order_and_alignment(pmpe, cache):
    """Heads before rows, rows and heads of odd pitches, one head for all."""
    heads, dim, page, T = 3, 48, 16, 21
    table, lengths, pages = plan([T], page, 3)
    c = cache_of(pmpe, pages, page, heads, dim, cache, 5)
    cu = cu_of([T])
    for k in (randn((heads, T, dim), 1, F16).transpose(0, 1), randn((T, heads, dim + 1), 2, BF16)[:, :, :dim], randn((T, heads * dim + 3), 3)[:, 1:heads * dim + 1].view(T, heads, dim),
              randn((T, 1, dim), 4, BF16).expand(T, heads, dim), randn((1, heads, dim), 5, BF16).expand(T, heads, dim)):
        v = (2 * k.float()).to(k.dtype)
        check_append(pmpe, c, k, v, table, lengths, cu)


@pytest.mark.parametrize("cache", CACHES)
def test_pages_that_are_none(pmpe, cache):
    """Entries out of range, lengths past the table and below zero, more rows
    than positions, offsets that do not start at zero."""
    heads, dim, page, pages = 2, 32, 4, 11
    c = cache_of(pmpe, pages, page, heads, dim, cache, 2)
    table = torch.tensor([[1, 99, 2], [-1, 3, 4], [5, 6, 7], [8, 9, 2 ** 31 - 1], [10, -2 ** 31, 0]], dtype=torch.int32).cuda()
    lengths = torch.tensor([12, 9, 400, -3, 5], dtype=torch.int32).cuda()
    x = randn((40, heads, dim), 3, BF16)
    for cu in ([0, 12, 21, 33, 36, 40], [2, 12, 21, 33, 33, 39], [0, 0, 0, 0, 0, 40]):
        cu = torch.tensor(cu, dtype=torch.int32).cuda()
        check_append(pmpe, c, x, -x, table, lengths, cu)
        check_read(pmpe, c, table, lengths, cu, 40, F32)
    check_append(pmpe, c, x[:5], -x[:5], table, lengths)
    check_read(pmpe, c, table, lengths, None, None, BF16)
    # offsets that decrease: whose a row is is not defined, but pages of no sequence stay as they are
    was = state(c)
    for cu in ([0, 20, 10, 33, 36, 40], [50, 40, 30, 20, 10, 0], [-9, 2 ** 31 - 1, -2 ** 31, 5, 60, 40]):
        c.append(x, x, table[:, :2].contiguous(), lengths, cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda())
        c.read(table, lengths, cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), rows=40)
    for t, w in zip(state(c), was):
        for page in (0, 2, 4, 7):
            assert torch.equal(bits(t[page]), bits(w[page]))
    q = randn((5, 4, dim), 4, BF16 if cache == BF16 else F16)
    check_attend(pmpe, c, q, table, lengths)
    check_attend(pmpe, c, q, table, lengths, window=6)


def test_append_of_what_is_not_finite(pmpe):
    """A NaN or an infinity stays in its position and head; sums of zeros and of
    the smallest numbers keep a finite scale."""
    heads, dim, page, T = 2, 64, 16, 8
    table, lengths, pages = plan([T], page, 3)
    x = randn((T, heads, dim), 1)
    x[0, 0, 3], x[1, 1, 5], x[2], x[3], x[4] = math.nan, math.inf, 0.0, 1e-40, 3e38 * torch.sign(x[4])
    for cache in CACHES:
        c = cache_of(pmpe, pages, page, heads, dim, cache, 5)
        c.append(x, x, table, lengths, cu_seqlens=cu_of([T]))
        k, _ = c.read(table, lengths, cu_seqlens=cu_of([T]), rows=T, dtype=F32)
        ok = torch.ones((T, heads), dtype=torch.bool)
        ok[0, 0] = ok[1, 1] = False
        if cache == F16:
            ok[4] = False  # past its range
        assert torch.isfinite(k[ok.cuda()]).all()
        assert torch.isnan(k[0, 0, 3]) and not torch.isfinite(k[1, 1, 5])
        tol = 0.07 if cache == E4M3 else 2.0 ** -7
        for r in (5, 6, 7) + ((4,) if cache != F16 else ()):
            assert (k[r] - x[r]).abs().max() <= tol * x[r].abs().max()
        assert not k[2].any() and (k[3] - x[3]).abs().max() <= 2.0 ** -126
        assert (cache == E4M3) == (c.k_scale is not None)


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_caches_of_more_than_2_31_elements(pmpe, cache):
    heads, dim, page = 2, 128, 64
    pages = 2 ** 31 // (heads * dim * page) + 9
    c = pmpe.KvCache.empty(pages, page, heads, dim, cache)
    T = 200
    need = -(-T // page)
    table = torch.arange(pages - need, pages, dtype=torch.int32).view(1, need).cuda()
    lengths, cu = torch.tensor([T], dtype=torch.int32).cuda(), cu_of([T])
    k, v = randn((T, heads, dim), 1, BF16), randn((T, heads, dim), 2, BF16)
    c.append(k, v, table, lengths, cu_seqlens=cu)
    assert not c.k.view(torch.uint8)[:pages - need].any()
    gk, gv = c.read(table, lengths, cu_seqlens=cu, rows=T)
    tol = 2.0 ** -4 + 2.0 ** -8 if cache == E4M3 else 0.0
    amax = k.float().abs().amax(2, keepdim=True), v.float().abs().amax(2, keepdim=True)
    assert ((gk.float() - k.float()).abs() <= tol * k.float().abs() + (tol > 0) * 2.0 ** -10 / 448 * amax[0]).all()
    assert ((gv.float() - v.float()).abs() <= tol * v.float().abs() + (tol > 0) * 2.0 ** -10 / 448 * amax[1]).all()
    check_attend(pmpe, c, randn((1, 4, dim), 3, BF16), table, lengths, only=(pages - need, pages))


# ------------------------------------------------------------- attention

def check_attend(pmpe, c, q, table, lengths, scale=None, window=0, only=None):
    a = c.attend(q, table, lengths, scale=scale, window=window)
    torch.cuda.synchronize()
    B, H, D = q.shape
    assert a.out.dtype == q.dtype and a.out.shape == q.shape and a.lse.shape == (B, H) and a.lse.dtype == F32
    pages, heads, page, _ = c.k.shape
    first, last = only or (0, pages)  # of the pages, those that the table names
    pools = [f64(t[first:last]) for t in (c.k, c.v)]
    if c.k.dtype == E4M3:
        pools = [x * f64(s[first:last])[..., None] for x, s in zip(pools, (c.k_scale, c.v_scale))]
    out, lse, q64 = f64(a.out), f64(a.lse), f64(q)
    sc = 1 / math.sqrt(D) if scale is None else float(np.float32(scale))
    for b in range(B):
        pg, pl = ref.kv_seen(table[b].cpu().numpy(), int(lengths[b]), window, pages, page)
        k, v = (x[pg - first, :, pl] for x in pools)
        want, want_lse, size, scores = ref.attend(q64[b], k, v, sc)
        n = len(pg)
        err = 136 * U * scores + 2.0 ** -22  # of a score, and its power
        close(lse[b], want_lse, err + (n / 64 + 32) * 2 * U + 2 * U * np.abs(want_lse) if n else 0.0)
        bound = (2 * (err[:, None] + 2.0 ** -17) + (n / 64 + 32) * 2 * 2 * U) * size
        # what rounds past the type's largest value (half a step above it) is an infinity of its sign
        most = torch.finfo(q.dtype).max
        want = np.where((np.abs(want) > most) & (out[b] == np.copysign(np.inf, want)), out[b], want)
        close(out[b], want, bound + half_eps(q.dtype) * (np.abs(want) + bound) + smallest(q.dtype))
    return a


def attend_case(pmpe, lengths, heads, kv_heads, dim, page, cache, dtype, seed=1, window=0, scale=None, q_scale=1.5):
    table, n, pages = plan(lengths, page, seed)
    c = cache_of(pmpe, pages, page, kv_heads, dim, cache, seed)
    q = randn((len(lengths), heads, dim), seed + 7, dtype, q_scale)
    return check_attend(pmpe, c, q, table, n, window=window, scale=scale)


KINDS = [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)]


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 100, 129])
def test_attend_one_sequence(pmpe, cache, dtype, n):
    attend_case(pmpe, [n], 4, 2, 64, 16, cache, dtype, seed=n)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 208, 256])
def test_attend_widths(pmpe, cache, dtype, dim):
    attend_case(pmpe, [70, 0, 301], 6, 2, dim, 24, cache, dtype, seed=dim)


@pytest.mark.parametrize("cache,dtype", KINDS[:2])
@pytest.mark.parametrize("dim", [8, 24, 72, 120, 136, 200, 248])
def test_attend_widths_of_eight(pmpe, cache, dtype, dim):
    attend_case(pmpe, [70, 0, 301], 6, 2, dim, 24, cache, dtype, seed=dim)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (6, 2), (7, 1), (8, 1), (9, 1), (32, 4), (16, 1), (17, 1), (48, 2), (33, 1), (64, 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_head_layouts(pmpe, cache, dtype, heads, kv_heads, dim):
    attend_case(pmpe, [200, 33, 1], heads, kv_heads, dim, 16, cache, dtype, seed=heads)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("page", [1, 2, 3, 8, 24, 64, 100, 128, 1000])
def test_attend_pages(pmpe, cache, dtype, page):
    attend_case(pmpe, [257, 0, 1000, 3], 8, 2, 128, page, cache, dtype, seed=page)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("window", [1, 15, 16, 64, 65, 300, 5000])
def test_attend_window(pmpe, cache, dtype, window):
    attend_case(pmpe, [257, 0, 64, 1000, 3, 65], 8, 2, 64, 24, cache, dtype, seed=window, window=window)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("B,n", [(127, 90), (128, 65), (129, 64), (300, 40), (700, 3), (40, 1500)])
def test_attend_batches(pmpe, cache, dtype, B, n):
    """Lengths that differ, empty ones among them; more sequences than threads."""
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, n + 1, B)
    lengths[rng.random(B) < 0.1] = 0
    attend_case(pmpe, lengths.tolist(), 4, 2, 64, 16, cache, dtype, seed=B)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("lengths", [[20000], [70001, 1], [1, 0, 33333, 5, 7777]])
def test_attend_long(pmpe, cache, dtype, lengths):
    """One pair of sequence and head over many CTAs."""
    attend_case(pmpe, lengths, 16, 2, 128, 64, cache, dtype, seed=3)
    attend_case(pmpe, lengths, 5, 1, 64, 16, cache, dtype, seed=4, window=9000)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("scale,q_scale", [(0.0, 1.0), (-0.3, 1.0), (0.125, 60.0), (1e-6, 1e4), (1.0, 1e-6)])
def test_attend_scales(pmpe, cache, dtype, scale, q_scale):
    if dtype == F16 and q_scale == 1e4:
        q_scale = 3e3
    attend_case(pmpe, [300, 17], 8, 2, 64, 16, cache, dtype, seed=9, scale=scale, q_scale=q_scale)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_scales_of_eight_bits(pmpe, dtype):
    """Scales from token to token far apart, zero among them, queries of any size."""
    table, n, pages = plan([500, 40], 16, 1)
    c = cache_of(pmpe, pages, 16, 2, 64, E4M3, 1)
    for spread, base in ((8.0, 1.0), (1.0, 2.0 ** -60), (1.0, 2.0 ** 40)):
        c.v_scale.copy_(torch.exp2(torch.round(randn(tuple(c.v_scale.shape), 5) * spread)) * base)
        check_attend(pmpe, c, randn((2, 8, 64), 3, dtype, 2.0), table, n)
    c.v_scale.zero_()
    a = check_attend(pmpe, c, randn((2, 8, 64), 3, dtype, 2.0), table, n)
    assert not a.out.any()
    c.v_scale.fill_(1.0)
    for size in (1e-30, 1e30) if dtype == BF16 else (1e-4, 1e3):
        c.k_scale.copy_(torch.exp(randn(tuple(c.k_scale.shape), 6)) / size / 64)
        check_attend(pmpe, c, randn((2, 8, 64), 3, dtype, size), table, n)
    c.k_scale.fill_(1.0)
    q = randn((2, 8, 64), 3, dtype)
    q[0, 3] = 0.0
    check_attend(pmpe, c, q, table, n)


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_what_is_not_seen_does_not_matter(pmpe, cache, dtype):
    """NaN and infinities in the pages' rest, in other pages, before the window."""
    lengths = [70, 3, 0, 161]
    table, n, pages = plan(lengths, 32, 1)
    clean = cache_of(pmpe, pages, 32, 2, 64, cache, 1)
    seen = torch.zeros((pages, 32), dtype=torch.bool)
    for b, length in enumerate(lengths):
        pg, pl = ref.kv_seen(table[b].cpu().numpy(), length, 50, pages, 32)
        seen[pg, pl] = True
    q = randn((4, 8, 64), 5, dtype)
    want = clean.attend(q, table, n, window=50)
    for poison in (math.nan, math.inf, -math.inf):
        held = [t.clone() for t in clean._held if t is not None]
        for i, t in enumerate(held):
            rest = (~seen)[:, None].expand(pages, 2, 32).cuda()
            if t.dim() == 4 and cache == E4M3:
                t.view(torch.uint8)[rest] = 0x7F  # NaN, its only one
            else:
                t[rest] = poison
        got = pmpe.KvCache(*held).attend(q, table, n, window=50)
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_a_nan_that_is_seen_shows(pmpe, cache, dtype):
    table, n, pages = plan([40, 40], 16, 1)
    c = cache_of(pmpe, pages, 16, 2, 64, cache, 1)
    q = randn((2, 4, 64), 5, dtype)
    want = c.attend(q, table, n)
    if cache == E4M3:
        c.k.view(torch.uint8)[int(table[0, 1]), 1, 3, 7] = 0x7F
    else:
        c.k[int(table[0, 1]), 1, 3, 7] = math.nan
    got = c.attend(q, table, n)
    assert torch.isnan(got.out[0, 2:]).all() and torch.isnan(got.lse[0, 2:]).all()
    assert torch.equal(got.out[0, :2], want.out[0, :2]) and torch.equal(got.out[1], want.out[1])


def test_queries_and_tables_of_any_pitch(pmpe):
    table, n, pages = plan([70, 3, 161], 16, 1)
    c = cache_of(pmpe, pages, 16, 2, 64, BF16, 1)
    q = randn((3, 8, 64), 5, BF16)
    want = c.attend(q, table, n)
    wide = torch.zeros((3, 9, 67), dtype=BF16, device="cuda")
    wide[:, 1:, 2:66] = q
    tables = torch.full((3, table.shape[1] + 5), 3, dtype=torch.int32, device="cuda")
    tables[:, 2:2 + table.shape[1]] = table
    views = [(wide[:, 1:, 2:66], tables[:, 2:2 + table.shape[1]]), (q.transpose(0, 1).contiguous().transpose(0, 1), tables[:, 2:2 + table.shape[1]])]
    for qq, tt in views:
        got = c.attend(qq, tt, n)
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
    one = randn((1, 1, 64), 6, BF16).expand(3, 8, 64)
    check_attend(pmpe, c, one, table, n)


def test_the_same_call_gives_the_same_bits(pmpe):
    lengths = np.random.default_rng(0).integers(0, 3000, 50).tolist()
    table, n, pages = plan(lengths, 16, 1)
    c = cache_of(pmpe, pages, 16, 2, 128, BF16, 1)
    q = randn((50, 16, 128), 5, BF16)
    want = c.attend(q, table, n)
    for _ in range(5):
        got = c.attend(q, table, n)
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


def test_pages_may_be_shared(pmpe):
    """Two sequences with the same prefix, and one page twice in a sequence."""
    c = cache_of(pmpe, 9, 16, 2, 64, F16, 1)
    table = torch.tensor([[4, 2, 7], [4, 2, 1], [5, 5, 5]], dtype=torch.int32).cuda()
    n = torch.tensor([40, 37, 48], dtype=torch.int32).cuda()
    check_attend(pmpe, c, randn((3, 4, 64), 5, F16), table, n)
    check_read(pmpe, c, table, n, cu_of([40, 37, 48]), 125, F16)


def test_parts_join_by_their_lse(pmpe):
    """What lse is for: attention over two halves, joined, is that over both."""
    c = cache_of(pmpe, 12, 16, 2, 64, BF16, 1)
    table = torch.arange(12, dtype=torch.int32).view(1, 12).cuda()
    q = randn((1, 8, 64), 5, BF16)
    n = lambda v: torch.tensor([v], dtype=torch.int32).cuda()  # noqa: E731
    whole = c.attend(q, table, n(192))
    a, b = c.attend(q, table[:, :6].contiguous(), n(96)), c.attend(q, table[:, 6:].contiguous(), n(96))
    m = torch.maximum(a.lse, b.lse)
    wa, wb = torch.exp(a.lse - m)[..., None], torch.exp(b.lse - m)[..., None]
    out = (a.out.float() * wa + b.out.float() * wb) / (wa + wb)
    # each half's output is rounded once to BF16
    assert ((out - whole.out.float()).abs() <= 2.0 ** -8 * (a.out.float().abs() + b.out.float().abs() + whole.out.float().abs()) + 1e-5).all()
    assert (m + torch.log(wa + wb)[..., 0] - whole.lse).abs().max() < 1e-5


def test_another_stream_and_graphs(pmpe):
    lengths = [70, 3, 0, 161, 1000]
    table, n, pages = plan(lengths, 32, 1, width=40)
    c = cache_of(pmpe, pages, 32, 2, 64, BF16, 1)
    q, k = randn((5, 8, 64), 5, BF16), randn((5, 2, 64), 6, BF16)
    c.append(k, -k, table, n)
    want = c.attend(q, table, n)
    back = c.read(table, n)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.append(k, -k, table, n, stream=s)
    got = c.attend(q, table, n, stream=s)
    rk, rv = c.read(table, n, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got.out, want.out) and torch.equal(rk, back[0]) and torch.equal(rv, back[1])
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        c.append(k, -k, table, n)
        o1 = c.attend(q, table, n)
    with torch.cuda.graph(g2, pool=g1.pool()):
        o2 = c.attend(q, table, n, window=40)
    # the lengths are read when the graph runs
    for new in ([70, 3, 0, 161, 1000], [1, 0, 64, 65, 900], [0, 0, 0, 0, 0]):
        n.copy_(torch.tensor(new, dtype=torch.int32))
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        w1, w2 = c.attend(q, table, n), c.attend(q, table, n, window=40)
        assert torch.equal(o2.out, w2.out) and torch.equal(o2.lse, w2.lse)
        if new[0] != 0:
            g1.replay()
            torch.cuda.synchronize()
            assert torch.equal(o1.out, w1.out)


def test_refusals_on_the_gpu(pmpe):
    table, n, pages = plan([70, 3], 16, 1)
    c = cache_of(pmpe, pages, 16, 2, 64, BF16, 1)
    q, k = randn((2, 4, 64), 5, BF16), randn((2, 2, 64), 6, BF16)
    cu = cu_of([1, 1])
    bad = [lambda: c.append(k, k, table, n[:1]), lambda: c.append(k[:1], k[:1], table, n), lambda: c.append(k, k[:1], table, n), lambda: c.append(k, k.float(), table, n),
           lambda: c.append(k.double(), k.double(), table, n), lambda: c.append(k.transpose(1, 2), k, table, n), lambda: c.append(k, k, table.long(), n),
           lambda: c.append(k, k, table.cpu(), n), lambda: c.append(k, k, table, n, cu_seqlens=cu[:2]), lambda: c.append(k, k, table[0], n),
           lambda: c.append(c.k[0, :, :2].transpose(0, 1), k, table, n), lambda: c.append(k, k, table.t().contiguous().t(), n),
           lambda: c.read(table, n, cu_seqlens=cu), lambda: c.read(table, n, cu_seqlens=cu, rows=-1), lambda: c.read(table, n, rows=3),
           lambda: c.read(table, n, dtype=E4M3), lambda: c.attend(q.half(), table, n), lambda: c.attend(q[:1], table, n), lambda: c.attend(q[:, :3], table, n),
           lambda: c.attend(q[:, :, :32], table, n), lambda: c.attend(q, table, n, window=-1), lambda: c.attend(q, table, n, scale=math.nan),
           lambda: c.attend(q.float(), table, n), lambda: c.attend(q[:, :0], table, n)]
    for i, call in enumerate(bad):
        with pytest.raises(pmpe.PmpeError):
            call()
            print("not refused:", i)
    with pytest.raises(TypeError):
        c.attend(q, table, n, scale="x")
    rows = c.read(table[:0], n[:0], cu_seqlens=cu[:1], rows=3)  # rows of no sequence
    assert rows[0].shape == (3, 2, 64) and not rows[0].any() and not rows[1].any()
    c.append(k, k, table[:0], n[:0], cu_seqlens=cu[:1])
    empty = c.attend(q[:0], table[:0], n[:0])
    assert empty.out.shape == (0, 4, 64) and empty.lse.shape == (0, 4)
    v = c.k._version
    c.append(k, k, table, n)
    assert c.k._version > v and c.v._version > v
