"""Sampling against a 64-bit reference.  Tokens are equal: r is within 2^-31, its
sums of multiples of 2^-46 or finer, so that a border would have to lie that near
to a draw (the seeds are fixed).  prob: r and the sum are rounded to FP32, and their quotient:
three half steps, and a tenth of one for r."""
import math

import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


def randn(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def rand(T, seed):
    return torch.rand(T, generator=torch.Generator().manual_seed(seed))


def check(pmpe, z, u, **kw):
    T = z.shape[0]
    s = pmpe.sample(z, u.cuda(), **{n: v.cuda() if torch.is_tensor(v) else v for n, v in kw.items()})
    torch.cuda.synchronize()
    assert s.token.dtype == torch.int32 and s.token.shape == (T,) and s.prob.dtype == F32 and s.prob.shape == (T,)
    rows, token, prob = z.detach().float().double().cpu().numpy(), s.token.tolist(), s.prob.tolist()
    for t in range(T):
        args = {n: (int(v[t]) if n == "top_k" else float(v[t])) if torch.is_tensor(v) else int(v) if n == "top_k" else float(np.float32(v))
                for n, v in kw.items()}
        want, p, kept = ref.sample_row(rows[t], float(u[t]), **args)
        assert token[t] == want, (t, args, float(u[t]), len(kept))
        assert abs(prob[t] - p) <= 3.1 * 2.0 ** -24 * p, (t, prob[t], p)
    return s


SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=1.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=50), dict(top_k=2000), dict(top_p=0.9),
            dict(top_p=0.3), dict(top_p=0.0), dict(min_p=0.05), dict(min_p=1.0), dict(top_k=40, top_p=0.95), dict(top_k=700, top_p=0.5, temperature=0.8, min_p=0.01)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 100, 1000, 4097, 32003])
def test_vocabularies(pmpe, V, dtype):
    z, u = randn((6, V), V, dtype, 2.0), rand(6, V + 1)
    for kw in SETTINGS:
        check(pmpe, z, u, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,V", [(1, 131072), (1, 50001), (3, 200003), (20, 65536), (40, 20011), (300, 5000), (2, 2 ** 21)])
@pytest.mark.parametrize("spread", [0.3, 3.0])
def test_rows(pmpe, T, V, dtype, spread):
    z, u = randn((T, V), T + V, dtype, spread), rand(T, V + 1)
    for kw in SETTINGS[-2:] + [dict(), dict(top_p=0.9), dict(top_k=5000)]:
        check(pmpe, z, u, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_with_settings_of_their_own(pmpe, dtype):
    T, V = 64, 30000
    rng = np.random.default_rng(0)
    z, u = randn((T, V), 1, dtype, 2.5), rand(T, 2)
    kw = dict(temperature=torch.tensor(rng.choice([0.0, -1.0, 0.5, 1.0, 2.0], T), dtype=F32), top_k=torch.tensor(rng.choice([0, -3, 1, 20, 1000, V, 2 ** 31 - 1], T), dtype=torch.int32),
              top_p=torch.tensor(rng.choice([0.0, 0.5, 0.9, 1.0, 2.0, -1.0], T), dtype=F32), min_p=torch.tensor(rng.choice([0.0, -1.0, 0.1, 1.0, 3.0], T), dtype=F32))
    check(pmpe, z, u, **kw)
    for n in kw:
        check(pmpe, z, u, **{n: kw[n]})


def test_settings_that_are_not_numbers(pmpe):
    """NaN: of a temperature the largest logit, of top_p the first alone, of min_p no limit, of u 0."""
    T, V = 4, 5000
    z, nan = randn((T, V), 1, F32, 2.0), torch.full((T,), math.nan)
    u = rand(T, 2)
    best = z.argmax(1).to(torch.int32)
    s = pmpe.sample(z, u.cuda(), temperature=nan.cuda())
    assert torch.equal(s.token, best) and (s.prob == 1).all()
    s = pmpe.sample(z, u.cuda(), top_p=nan.cuda())
    assert torch.equal(s.token, best) and (s.prob == 1).all()
    s, w = pmpe.sample(z, u.cuda(), min_p=nan.cuda()), pmpe.sample(z, u.cuda())
    assert torch.equal(s.token, w.token) and torch.equal(s.prob, w.prob)
    s, w = pmpe.sample(z, nan.cuda()), pmpe.sample(z, torch.zeros(T).cuda())
    assert torch.equal(s.token, w.token)
    for bad, good in ((-0.5, 0.0), (-math.inf, 0.0), (1.0, 1 - 2.0 ** -24), (7.0, 1 - 2.0 ** -24), (math.inf, 1 - 2.0 ** -24)):
        for kw in SETTINGS[:2]:
            assert torch.equal(pmpe.sample(z, torch.full((T,), bad).cuda(), **kw).token, pmpe.sample(z, torch.full((T,), good).cuda(), **kw).token)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_the_ends_of_u(pmpe, dtype):
    z = randn((8, 9000), 3, dtype, 4.0)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 2.0 ** -24, 1e-30, 1e-45, 0.5, 0.25, 2.0 ** -100])
    for kw in SETTINGS:
        check(pmpe, z, u, **kw)


@pytest.mark.parametrize("T,V", [(3, 131072), (200, 2048), (200, 2049), (200, 9000)])
def test_large_top_k(pmpe, T, V):
    """As many as there are runs of loads, more, and less; rows of which a mask leaves about as many."""
    g = torch.Generator().manual_seed(V)
    z, u = randn((T, V), V, BF16, 2.0), rand(T, V + 1)
    top_k = torch.tensor(np.random.default_rng(V).choice([400, 511, 512, 513, 800, 1000, 1023, 1024, 1025, 2047, 2048], T), dtype=torch.int32)
    check(pmpe, z, u, top_k=top_k, top_p=0.98)
    left = torch.tensor([1, 10, 300, 1000, 1024, 1500, 2500])[torch.arange(T) % 7]
    z = z.masked_fill(torch.rand((T, V), generator=g).argsort(1).argsort(1).ge(left[:, None]).cuda(), -math.inf)
    check(pmpe, z, u, top_k=top_k)
    check(pmpe, z.sort(1).values, u, top_k=top_k, top_p=0.9)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("descending", [True, False])
def test_sorted_logits(pmpe, dtype, descending):
    """The draw lies among the smallest tokens, whose sum R is 2^-24 of all, S, and of which one is about
    2^-31.  Of 16491 tokens r is rounded to a multiple of 2^-48: up to 2^-49 each, n of them below the
    border, and 2^-31 of r.  The border itself, 2^-24 S, is off by 2^-24 (2^-31 S + V 2^-49)."""
    T, V, low = 48, 16491, 2.0 ** -24
    z = torch.sort(randn((T, V), 6, F32, 5.0), dim=1, descending=descending).values.to(dtype)
    u = torch.full((T,), 1 - low if descending else low)
    rows = np.sort(z.double().cpu().numpy(), axis=1)  # the smallest first
    for kw in SETTINGS[:2]:
        s = pmpe.sample(z, u.cuda(), **kw)
        for t, token in enumerate(s.token.tolist()):
            r = np.exp((rows[t] - rows[t, -1]) / np.float64(np.float32(kw.get("temperature", 1.0))))
            r[r < 2.0 ** -40] = 0
            upto = np.cumsum(r)
            at = V - 1 - token if descending else token
            n, border = int((r[:at + 1] > 0).sum()), low * upto[-1]
            off = n * 2.0 ** -49 + 2.0 ** -31 * upto[at] + low * (2.0 ** -31 * upto[-1] + V * 2.0 ** -49)
            assert r[at] > 0 and off < r[at], (t, off, r[at])
            assert upto[at] - r[at] - off <= border <= upto[at] + off, (t, token, border, upto[at], off)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_equal_logits(pmpe, dtype):
    """The lowest ids of equal ones stay, where all are equal and where few values are."""
    u = rand(7, 1)
    flat = torch.full((7, 10007), -1.25, dtype=dtype).cuda()
    few = torch.round(randn((7, 10007), 2)).to(dtype)
    zeros = torch.where(randn((7, 10007), 3) > 0, 0.0, -0.0).to(dtype)
    for z in (flat, few, zeros):
        for kw in SETTINGS + [dict(top_k=9999), dict(top_k=10007), dict(top_k=3, top_p=0.5), dict(top_p=0.99)]:
            check(pmpe, z, u, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masked_logits(pmpe, dtype):
    """-inf, NaN and the type's lowest value; rows with one token, with none; +inf."""
    V = 5000
    z = randn((9, V), 1, dtype, 2.0)
    z[0] = -math.inf
    z[1] = math.nan
    z[2] = -math.inf
    z[2, 4321] = -3.0
    z[3, ::2] = -math.inf
    z[4, 5:] = torch.finfo(dtype).min
    z[5, 77], z[5, 99] = math.inf, math.inf
    z[6] = torch.finfo(dtype).min
    z[7, ::3] = math.nan
    z[8] = torch.where(torch.arange(V).cuda() % 2 == 0, math.inf, -math.inf)
    z = torch.where(z.float() == math.inf, torch.tensor(torch.finfo(F32).max).cuda(), z.float()) if dtype == F32 else z
    for kw in SETTINGS:
        s = check(pmpe, z, rand(9, 2), **kw)
        assert s.token[0] == -1 and s.prob[0] == 0 and s.token[1] == -1 and s.token[2] == 4321 and s.prob[2] == 1


def test_infinite_logits_count_as_the_largest(pmpe):
    z = randn((3, 300), 1)
    z[0, 7], z[1, 8], z[1, 9], z[2, 5], z[2, 6] = math.inf, math.inf, torch.finfo(F32).max, math.inf, math.inf
    s = pmpe.sample(z, torch.tensor([0.9, 0.9, 0.1]).cuda())
    assert s.token.tolist() == [7, 9, 5] and s.prob.tolist() == [1.0, 0.5, 0.5]


def test_temperatures_of_any_size(pmpe):
    z, u = randn((5, 3000), 1, F32, 2.0), rand(5, 2)
    for T in (1e-45, 1e-38, 1e-30, 1e-3, 0.1, 30.0, 1e10, 1e30, 3e38):
        check(pmpe, z, u, temperature=T)
        check(pmpe, z, u, temperature=T, top_k=100, top_p=0.7)
    big = randn((5, 3000), 1, F32, 1e37)
    for T in (1.0, 1e36, 1e37, 3e38):
        check(pmpe, big, u, temperature=T, top_p=0.9)
    small = randn((5, 3000), 1, F32, 1e-38)
    for T in (1e-40, 1e-38, 1e-37, 1.0):
        check(pmpe, small, u, temperature=T, top_p=0.9, min_p=0.01)


def test_values_next_to_one_another(pmpe):
    """Logits a few ulps apart, about zero, and on both sides of powers of two."""
    u = rand(6, 3)
    for base, step in ((1.0, 2.0 ** -23), (-8.0, 2.0 ** -21), (0.0, 2.0 ** -149), (1024.0, 2.0 ** -14), (0.0, 1e-20)):
        k = torch.randint(-40, 41, (6, 20000), generator=torch.Generator().manual_seed(4)).double()
        z = (base + k * step).float().cuda()
        for kw in SETTINGS:
            check(pmpe, z, u, **kw)


def test_rows_of_any_pitch(pmpe):
    u = rand(5, 1)
    for dtype in (F32, BF16):
        wide = randn((5, 3011), 2, dtype, 2.0)
        for z in (wide[:, 1:3002], wide[:, :3000], wide[:, 3:4]):
            for kw in SETTINGS[-2:]:
                s = check(pmpe, z, u, **kw)
                w = pmpe.sample(z.contiguous(), u.cuda(), **kw)
                assert torch.equal(s.token, w.token) and torch.equal(s.prob, w.prob)
    row = randn((1, 3000), 3)
    check(pmpe, row.expand(5, 3000), u, top_p=0.9)


def test_a_row_does_not_depend_on_the_others(pmpe):
    """The same row in batches that are split over other numbers of CTAs."""
    z, u = randn((200, 70000), 1, BF16, 2.0), rand(200, 2).cuda()
    for kw in SETTINGS:
        want = pmpe.sample(z, u, **kw)
        for n in (1, 2, 10, 60):
            s = pmpe.sample(z[:n], u[:n], **kw)
            assert torch.equal(s.token, want.token[:n]) and torch.equal(s.prob, want.prob[:n])


def test_more_than_2_31_logits(pmpe):
    V = 2 ** 20
    z = torch.zeros((2 ** 11 + 3, V), dtype=BF16, device="cuda")
    z[2 ** 11 + 1, 12345] = 30.0
    z[2 ** 11 + 2, 0], z[2 ** 11 + 2, V - 1] = 9.0, 9.5
    u = torch.full((z.shape[0],), 0.5, device="cuda")
    s = pmpe.sample(z, u)
    assert s.token[0] == V // 2 and s.token[-2] == 12345
    check(pmpe, z[-3:], u[-3:].cpu(), top_p=0.9)
    assert torch.equal(s.token[-3:], pmpe.sample(z[-3:], u[-3:]).token)


def test_frequencies(pmpe):
    """Even steps of u give each token its share."""
    z = torch.log(torch.tensor([0.1, 0.4, 0.05, 0.25, 0.2]))
    T = 4000
    s = pmpe.sample(z.cuda().expand(T, 5), ((torch.arange(T) + 0.5) / T).cuda())
    assert torch.bincount(s.token.long(), minlength=5).tolist() == [400, 1600, 200, 1000, 800]


def test_another_stream_and_a_graph(pmpe):
    z, u = randn((7, 40000), 1, F32, 2.0), rand(7, 2).cuda()
    k = torch.tensor([0, 1, 5, 50, 500, 5000, 50000], dtype=torch.int32).cuda()
    want = pmpe.sample(z, u, top_k=k, top_p=0.9)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s = pmpe.sample(z, u, top_k=k, top_p=0.9, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(s.token, want.token) and torch.equal(s.prob, want.prob)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = pmpe.sample(z, u, top_k=k, top_p=0.9)
    for seed in (5, 6):
        z.copy_(randn((7, 40000), seed, F32, 2.0))
        u.copy_(rand(7, seed + 1))
        g.replay()
        torch.cuda.synchronize()
        want = pmpe.sample(z, u, top_k=k, top_p=0.9)
        assert torch.equal(out.token, want.token) and torch.equal(out.prob, want.prob)


def test_refusals_on_the_gpu(pmpe):
    z, u = randn((4, 100), 1), rand(4, 2).cuda()
    for call in (lambda: pmpe.sample(z[0], u), lambda: pmpe.sample(z, u[:3]), lambda: pmpe.sample(z, u.cpu()), lambda: pmpe.sample(z, u.double()),
                 lambda: pmpe.sample(z.double(), u), lambda: pmpe.sample(z.t(), u), lambda: pmpe.sample(z, u, temperature=u.cpu()), lambda: pmpe.sample(z, u, top_k=u),
                 lambda: pmpe.sample(z, u, top_p=u.half()), lambda: pmpe.sample(z, u, min_p=u[:2]), lambda: pmpe.sample(z, u, temperature=-1.0),
                 lambda: pmpe.sample(z, u, temperature=math.inf), lambda: pmpe.sample(z, u, top_p=1.5), lambda: pmpe.sample(z, u, min_p=-0.5), lambda: pmpe.sample(z, u, top_k=-1),
                 lambda: pmpe.sample(z[:, :0], u)):
        with pytest.raises(pmpe.PmpeError):
            call()
    with pytest.raises(TypeError):
        pmpe.sample(z, u, temperature="hot")
    with pytest.raises(TypeError):
        pmpe.sample(z, u, top_k=0.5)
    s = pmpe.sample(z[:0], u[:0])
    assert s.token.shape == (0,) and s.prob.shape == (0,)
