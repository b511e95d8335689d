"""What the attention's weights hold to.

u = 2^-24.  Scores here are one product q k and its factors: off by 2 u of
themselves in 16 bits (log2 e, and one product), 6 u in 8 bits (the scale, the key's
scale and their products besides).  2^x by the hardware is within 2^-22; a weight
in BF16 words is exact, in FP16 words within 2^-22, or 2^-39 of the largest weight
where it is below 2^-22 of it (a step of 2^-24 halved, the largest at 2^14 or above; over
8 bits at 2^12).  A matrix instruction's sums may be cut off instead of rounded: 2 u
of the largest term each."""
import math

import numpy as np
import pytest
import torch

import operators_ref as ref
from test_gpu_kv import BF16, E4M3, F16, KINDS, U, cache_of, close, f64, half_eps, smallest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_weights_have_the_bits_of_fp32(pmpe, dtype):
    """Three positions whose values cancel the first two words of a weight: keys
    0, x, 0 and values -c1, 1, -c2 with c1 + c2 = e^x to two words of the type."""
    B, D = 96, 16
    x = (-torch.linspace(0.02, 0.68, B)).to(dtype)
    w = torch.exp(x.double())
    c1 = w.to(dtype)
    c2 = (w - c1.double()).to(dtype)
    c = pmpe.KvCache.empty(B, 16, 1, D, dtype)
    c.k[:, 0, 1, 0] = x.cuda()
    c.v[:, 0, 0] = -c1.cuda()[:, None]
    c.v[:, 0, 1] = 1.0
    c.v[:, 0, 2] = -c2.cuda()[:, None]
    q = torch.zeros((B, 1, D), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    a = c.attend(q, table, torch.full((B,), 3, dtype=torch.int32, device="cuda"), scale=1.0)
    w, x, rest = w.numpy(), np.abs(f64(x)), (w - c1.double() - c2.double()).numpy()
    want = rest / (2 + w)
    # the score's and the power's errors; three instructions' sums of terms up to 1, the four warps', the quotient's
    bound = (w * (2 * U * x + 2.0 ** -22) + (0 if dtype == BF16 else 2.0 ** -22) + 2 * 3 * U + 6 * U * np.abs(rest)) / (2 + w)
    close(f64(a.out[:, 0]), want[:, None], (bound + half_eps(dtype) * (np.abs(want) + bound) + smallest(dtype))[:, None])


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("others", ["equal", "random"])
@pytest.mark.parametrize("page", [16, 24])
def test_what_is_far_below_a_position_without_value(pmpe, cache, dtype, others, page):
    """Positions of large scores and zero values (one for each warp of a tile),
    and thousands of others up to 2^-29 of their weight: the output is theirs alone."""
    n, D, H, G = 4000, 32, 4, 12
    g = torch.Generator().manual_seed(3)
    k, v = torch.zeros((n, 1, D)), (torch.rand((n, 1, D), generator=g) + 0.5) * 1000
    if others == "random":
        k[:, 0, 0] = torch.randn(n, generator=g)
    first = [0, 16, 32, 48, 64, 80, 96, 112]
    k[first, 0, 0], v[first] = 16.0, 0.0
    need = -(-n // page)
    c = pmpe.KvCache.empty(need, page, 1, D, cache)
    one = torch.arange(need, dtype=torch.int32, device="cuda").view(1, need)
    rows = BF16 if cache == E4M3 else cache
    c.append(k.to(rows).cuda(), v.to(rows).cuda(), one, torch.tensor([n], dtype=torch.int32, device="cuda"), cu_seqlens=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    # enough sequences that a CTA has whole ones; G of them differ
    B = 57 * G
    q1 = torch.zeros((G, H, D))
    q1[..., 0] = torch.linspace(4.0, 20.0, G * H).view(G, H) / 16
    q = q1.to(dtype).cuda().repeat(B // G, 1, 1)
    a = c.attend(q, one.expand(B, need).contiguous(), torch.full((B,), n, dtype=torch.int32, device="cuda"), scale=1.0)
    pos = np.arange(n)
    pools = [f64(t) if s is None else f64(t) * f64(s)[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]
    kk, vv = (x[pos // page, 0, pos % page] for x in pools)
    s = np.einsum("ghd,nd->ghn", f64(q[:G]), kk)
    top = s.max(2, keepdims=True)
    e = np.exp(s - top)
    p = e / e.sum(2, keepdims=True)
    want = np.einsum("ghn,nd->ghd", p, vv)  # (values are not negative: also what errors are relative to)
    # a score and its scale's rounding in 8 bits, the power, the words, the sums of 64 positions a step; each twice, the total has them too
    rel = 2 * (6 * U * np.abs(s).max(2) + 2.0 ** -22 + 2.0 ** -22 + (n / 64 + 32) * 2 * U)
    bound = rel[..., None] * want
    if cache != BF16:
        # each below 2^-22 of the largest (in 8 bits 2^-19, with the values' scales, relative to a power of two up to twice the largest)
        bound = bound + n * p.max(2)[..., None] * vv.max() * (2.0 ** -39 if cache == F16 else 2.0 ** -36)
    bound = bound + half_eps(dtype) * (want + bound) + smallest(dtype)
    close(f64(a.out).reshape(B // G, G, H, D), want[None], bound[None])
    lse = (top + np.log(e.sum(2, keepdims=True)))[..., 0]
    close(f64(a.lse).reshape(B // G, G, H), lse[None], (rel / 2 + 2 * U * np.abs(lse) + 2.0 ** -22)[None])
    assert math.isfinite(float(a.out.float().sum()))


@pytest.mark.parametrize("n", [1, 2, 3, 70])
@pytest.mark.parametrize("base", [2.0 ** -126, 2.0 ** -125, 2.0 ** -123, 2.0 ** -110, 2.0 ** 118])
def test_values_of_the_smallest_scales(pmpe, base, n):
    """Eight bits: scales down to 2^-126, the least that an append writes, and near FP32's end."""
    D, page = 32, 16
    need = -(-n // page)
    g = torch.Generator().manual_seed(4)
    c = pmpe.KvCache.empty(need, page, 1, D, E4M3)
    c.k.copy_(torch.randn(c.k.shape, generator=g).to(E4M3))
    c.v.copy_((1 + 255 * torch.rand(c.v.shape, generator=g)).to(E4M3))
    c.k_scale.fill_(0.25)
    c.v_scale.copy_(base * (1 + torch.rand(c.v_scale.shape, generator=g)))
    q = torch.randn((1, 4, D), generator=g).to(BF16).cuda()
    table = torch.arange(need, dtype=torch.int32, device="cuda").view(1, need)
    a = c.attend(q, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    pos = np.arange(n)
    k, v = (x[pos // page, :, pos % page] for x in (f64(c.k) * f64(c.k_scale)[..., None], f64(c.v) * f64(c.v_scale)[..., None]))
    want, _, size, scores = ref.attend(f64(q[0]), k, v, 1 / math.sqrt(D))
    # as in the other file's, FP16's words in place of 2^-17
    bound = (2 * (136 * U * scores[:, None] + 2.0 ** -22 + 2.0 ** -22) + (n / 64 + 32) * 4 * U) * size
    bound = bound + n * 2.0 ** -36 * v.max() + half_eps(BF16) * (np.abs(want) + bound) + smallest(BF16)
    # the sum over the values before it is divided, up to 2^3 n of the largest value, is FP32's: 2^128 ends it
    ok = np.full(want.shape, 8 * n * v.max() < 2.0 ** 128) | (n == 1)
    close(f64(a.out[0])[ok], want[ok], bound[ok])


@pytest.mark.parametrize("cache,dtype,n", [(BF16, BF16, 1 << 22), (F16, F16, 1 << 20), (E4M3, F16, 1 << 20), (E4M3, BF16, 1 << 22)])
def test_long_sums_are_not_cut_off(pmpe, cache, dtype, n):
    """Enough long sequences that a CTA has whole ones, all values 1: the weights'
    sum over the weights' sum.  A warp adds a quarter of them, 16 at a time: roundings
    of half a step each, in any direction, ten standard deviations of which are
    10 sqrt(n / 64) u, for both sums."""
    B, H, D, page, pages = 480, 8, 32, 1024, 8
    c = cache_of(pmpe, pages, page, 1, D, cache, 1)
    c.v.copy_(torch.ones(c.v.shape).to(cache))
    if cache == E4M3:
        c.v_scale.fill_(1.0)
    g = torch.Generator().manual_seed(2)
    table = torch.randint(0, pages, (1, n // page), generator=g, dtype=torch.int32).cuda().expand(B, -1).contiguous()
    q = torch.randn((B, H, D), generator=g).to(dtype).cuda()
    a = c.attend(q, table, torch.full((B,), n, dtype=torch.int32, device="cuda"))
    close(f64(a.out), 1.0, 2 * 10 * math.sqrt(n / 64) * U + half_eps(dtype))


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_an_infinite_value_shows_in_its_column_alone(pmpe, dtype):
    c = cache_of(pmpe, 8, 16, 2, 64, dtype, 1)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    n = torch.tensor([64, 50], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(3)
    q = torch.randn((2, 8, 64), generator=g).to(dtype).cuda()
    want = c.attend(q, table, n)
    c.v[5, 1, 3, 7] = math.inf
    got = c.attend(q, table, n)
    at = torch.zeros((2, 8, 64), dtype=torch.bool, device="cuda")
    at[1, 4:, 7] = True
    assert not torch.isfinite(got.out[at]).any()
    assert torch.equal(got.out[~at], want.out[~at]) and torch.equal(got.lse, want.lse)
