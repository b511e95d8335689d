"""clip_grad_norm against 64-bit references.

Bounds: the square sum of a vector of 8 and four of them in FP32, 12 x 2^-24,
halved by the root, the rest 48 bits or more, FP32's rounding of the result: below
2^-20 for the norm and the factor; an output adds one rounding of its type."""
import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2.0 ** -20


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


def randn(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def check(pmpe, grads, max_norm, out=None, **kw):
    before = [f64(g) for g in grads]
    norm = pmpe.clip_grad_norm(grads, max_norm, out=out, **kw)
    torch.cuda.synchronize()
    want = ref.global_norm(before)
    assert norm.shape == () and norm.dtype == F32
    assert abs(float(norm) - want) <= REL * want, (float(norm), want)
    f = min(1.0, max_norm / (want + 1e-6))
    for g, o, b in zip(grads, out if out is not None else grads, before):
        r = torch.finfo(o.dtype)
        tiny = r.smallest_normal * r.eps / 2
        assert (np.abs(f64(o) - b * f) <= (r.eps / 2 + REL) * np.abs(b * f) + tiny).all()
        if out is not None:
            assert np.array_equal(f64(g), b)


SHAPES = [[(1,)], [(3,), (5, 7)], [(1000,)], [(4096,), (4097,), (1,)], [(8192,)], [(33, 129), (2, 2), (17,), (4, 300, 5)],
          [(0,), (5,), (0, 3)], [(300000,)], [(64, 256), (4, 128, 256), (4, 128, 256), (4, 256, 128)]]


@pytest.mark.parametrize("shapes", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_shapes(pmpe, shapes, dtype):
    grads = [randn(s, i, dtype) for i, s in enumerate(shapes)]
    n = sum(g.numel() for g in grads)
    check(pmpe, [g.clone() for g in grads], 0.3 * n ** 0.5)           # clips
    check(pmpe, [g.clone() for g in grads], 3.0 * n ** 0.5)           # does not
    check(pmpe, [g.clone() for g in grads], float("inf"))
    check(pmpe, [g.clone() for g in grads], 0.0)
    check(pmpe, grads, 0.3 * n ** 0.5, out=[torch.empty_like(g) for g in grads])
    check(pmpe, grads, 3.0 * n ** 0.5, out=[torch.empty_like(g) for g in grads])


@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_unaligned_views_of_one_buffer(pmpe, offset, dtype):
    flat, flat_out = randn((20000,), 1, dtype), torch.zeros(20000, dtype=dtype, device="cuda")
    cuts = [offset, offset + 1, offset + 4100, offset + 4101 + 4096, 19990]
    grads = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
    out = [flat_out[a - offset:b - offset] for a, b in zip(cuts, cuts[1:])]  # another alignment than the gradients'
    before = flat.clone()
    check(pmpe, grads, 20.0, out=out)
    assert (flat_out[cuts[-1] - offset:] == 0).all()
    check(pmpe, grads, 20.0)
    assert torch.equal(flat[:offset], before[:offset]) and torch.equal(flat[cuts[-1]:], before[cuts[-1]:])


@pytest.mark.parametrize("count", [2, 64, 65, 1024, 1025, 2500])
def test_many_tensors(pmpe, count):
    """The table of a launch holds 64 or 1024 tensors; more take more launches."""
    flat = randn((count * 40,), count)
    grads = [flat[40 * i:40 * i + 1 + i % 37] for i in range(count)]
    check(pmpe, grads, 10.0)


def test_mixed_types_orders_and_a_dict(pmpe):
    grads = [randn((40, 30), 1, F32), randn((50,), 2, BF16), randn((6, 7, 8), 3, F16), randn((20, 30), 4, F32).t()]
    check(pmpe, grads, 5.0)
    d = {"a": randn((40, 30), 5), "b": randn((70,), 6, BF16)}
    want = {n: g.clone() for n, g in d.items()}
    a = pmpe.clip_grad_norm(d, 2.0)
    b = pmpe.clip_grad_norm(list(want.values()), 2.0)
    assert torch.equal(a, b) and all(torch.equal(d[n], want[n]) for n in d)


@pytest.mark.parametrize("scale", [1e30, 1e19, 1e-22, 1e-30, 1e-41])
def test_squares_outside_fp32(pmpe, scale):
    grads = [randn((5000,), 1, F32, scale), randn((33,), 2, F32, scale)]
    check(pmpe, [g.clone() for g in grads], 10 * scale)
    mixed = [torch.cat([grads[0], torch.zeros(4096, device="cuda")]), randn((33,), 2, F32, 1.0)]
    check(pmpe, mixed, 1.0)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_clips_nothing(pmpe, bad):
    grads = [randn((5000,), 1), randn((77,), 2, BF16)]
    grads[1][3] = bad
    before = [g.clone() for g in grads]
    out = [torch.zeros_like(g) for g in grads]
    norm = pmpe.clip_grad_norm(grads, 1.0)
    n2 = pmpe.clip_grad_norm(grads, 1.0, out=out)
    torch.cuda.synchronize()
    for v in (norm, n2):
        assert (torch.isnan(v) if bad != bad else torch.isinf(v)).item()
    for g, o, b in zip(grads, out, before):
        assert torch.equal(torch.nan_to_num(g.float(), 7.0), torch.nan_to_num(b.float(), 7.0))
        assert torch.equal(torch.nan_to_num(o.float(), 7.0), torch.nan_to_num(b.float(), 7.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_norm_past_fp32_clips_nothing(pmpe, dtype):
    """Finite gradients whose norm FP32 does not hold: it is reported as
    infinity, and what is reported decides."""
    high = torch.finfo(dtype).max
    for values in ((3e38, 3e38), (high, high, high, 1.0), (high, 2.0 ** 127) * 3000):
        g = torch.tensor(values).to(dtype).cuda()
        more, out = randn((500,), 2), [torch.zeros_like(g), torch.zeros(500, device="cuda")]
        before = [g.clone(), more.clone()]
        n = [pmpe.clip_grad_norm([g, more], 1.0, out=out), pmpe.clip_grad_norm([g, more], 1.0)]
        assert all(float(v) == float("inf") for v in n)
        for a, b, o in zip(before, (g, more), out):
            assert torch.equal(a, b) and torch.equal(a, o)
    for values in ((2e38, 2e38), (3.4e38,)):  # within FP32: clipped
        check(pmpe, [torch.tensor(values).cuda(), torch.tensor([7.0], device="cuda")], 1e30)


@pytest.mark.parametrize("dtype,scale", [(F32, 1e35), (F32, 1e30), (BF16, 1e35), (F32, 1e-3)])
@pytest.mark.parametrize("max_norm", [1e-4, 1e-10, 1e-34])
def test_factors_below_the_normal_range(pmpe, dtype, scale, max_norm):
    """Large gradients and a small limit: the factor is below 2^-126, the
    clipped gradients (of the size max_norm / 70) are not."""
    grads = [randn((5000,), 1, dtype, scale), randn((33,), 2, dtype, scale)]
    check(pmpe, grads, max_norm, out=[torch.empty_like(g) for g in grads])
    check(pmpe, grads, max_norm)


def test_zero_gradients(pmpe):
    grads = [torch.zeros(5000, device="cuda"), torch.zeros(3, device="cuda")]
    grads += [torch.full((5001,), -0.0, dtype=t, device="cuda") for t in (F32, BF16, F16)]
    assert float(pmpe.clip_grad_norm(grads, 1.0)) == 0.0
    assert all((g == 0).all() for g in grads)
    masked = randn((9000,), 3, BF16)
    masked[:8000] *= -0.0
    check(pmpe, [masked], 1.0)


def test_what_is_written_in_place_counts_up_its_version(pmpe):
    """So that autograd does not go on with a tensor that it saved before."""
    def version(call, t):
        v = t._version
        call()
        return t._version - v

    a, out = randn((300,), 1), [torch.empty(300, device="cuda")]
    assert version(lambda: pmpe.clip_grad_norm([a], 1.0), a) == 1
    assert version(lambda: pmpe.clip_grad_norm([a], float("inf")), a) == 0  # the norm alone
    assert version(lambda: pmpe.clip_grad_norm([a], 1.0, out=out), a) == 0 and out[0]._version == 1
    assert version(lambda: pmpe.clip_grad_norm([a], float("inf"), out=out), out[0]) == 1
    x, res, w = randn((4, 64), 2), randn((4, 64), 3), randn((64,), 4)
    assert version(lambda: pmpe.rms_norm(x, w, residual=res), res) == 0
    assert version(lambda: pmpe.rms_norm(x, w, residual=res, h_out=res), res) == 1
    load = torch.zeros(8, dtype=torch.int32, device="cuda")
    assert version(lambda: pmpe.Router(8, 0, 2).route(randn((4, 8), 5), load=load), load) == 1
    leaf = randn((4, 64), 6).requires_grad_()
    saved = leaf * 2
    loss = saved.square().sum()
    pmpe.rms_norm(x, w, residual=saved.detach(), h_out=saved.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():  # tensors without versions
        b = randn((300,), 7)
        pmpe.clip_grad_norm([b], 1.0)
        pmpe.rms_norm(x, w, residual=b[:256].view(4, 64), h_out=b[:256].view(4, 64))
    pmpe.clip_grad_norm([b], 0.5)


def test_refusals(pmpe):
    a, b = randn((64, 64), 1), randn((64,), 2)
    for bad in (dict(grads=[a, a]), dict(grads=[a, a[3]]), dict(grads=[a, a.view(-1)[4090:]]), dict(grads=[a[:, :30]]),
                dict(grads=[a.double()]), dict(grads=[a.cpu()]), dict(grads=[a, b.cpu()]), dict(grads=[a], out=[b]),
                dict(grads=[a], out=[]), dict(grads=[a], out=[a.half()]), dict(grads=[a], max_norm=-1.0),
                dict(grads=[a], max_norm=float("nan")), dict(grads=[a], out=[torch.empty_like(a.t())]),
                dict(grads=[a, b], out=[torch.empty_like(a), a[0]]),
                # as many elements and the same strides, but not one run of memory
                dict(grads=[a[:2, :3].contiguous().t().as_strided((2, 3), (1, 2))], out=[b.as_strided((3, 2), (1, 2))])):
        with pytest.raises(pmpe.PmpeError):
            pmpe.clip_grad_norm(**dict(dict(max_norm=1.0), **bad))


def test_other_stream_and_two_graphs(pmpe):
    grads = [randn((3000,), 1), randn((500, 33), 2, BF16)]
    other = [randn((700,), 3)]
    want, want2 = [g.clone() for g in grads], [g.clone() for g in other]
    na, nb = pmpe.clip_grad_norm(want, 5.0), pmpe.clip_grad_norm(want2, 5.0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    mine = [g.clone() for g in grads]
    torch.cuda.synchronize()
    n = pmpe.clip_grad_norm(mine, 5.0, stream=s)
    s.synchronize()
    assert torch.equal(n, na) and all(torch.equal(a, b) for a, b in zip(mine, want))
    outs = [torch.empty_like(g) for g in grads], [torch.empty_like(g) for g in other]
    ga, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(ga):
        n1 = pmpe.clip_grad_norm(grads, 5.0, out=outs[0])
    with torch.cuda.graph(gb):
        n2 = pmpe.clip_grad_norm(other, 5.0, out=outs[1])
    for _ in range(3):
        with torch.cuda.stream(s):
            ga.replay()
        gb.replay()
        torch.cuda.synchronize()
        assert torch.equal(n1, na) and torch.equal(n2, nb)
        assert all(torch.equal(a, b) for a, b in zip(outs[0] + outs[1], want + want2))


def test_more_than_2_to_31_elements(pmpe):
    """Offsets past 32 bits, in a tensor that is not aligned to a vector."""
    n = 2 ** 31 + 1001
    g = torch.empty(n + 3, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))[3:]
    edges = [g[:1000].clone(), g[-3000:].clone()]
    want = sum(float(g[i:i + 2 ** 28].double().square().sum()) for i in range(0, n, 2 ** 28)) ** 0.5
    norm = pmpe.clip_grad_norm([g], 0.5 * want)
    assert abs(float(norm) - want) <= REL * want
    for got, was in zip((g[:1000], g[-3000:]), edges):
        r = was.double() * 0.5
        assert ((got.double() - r).abs() <= (2.0 ** -8 + REL) * r.abs()).all()
