"""rms_norm and its backward against 64-bit references.

Bounds: a row's sum of squares adds at most 64 terms a thread in sequence and
ten in the trees, 74 x 2^-24, halved by the root; rsqrt (2 ulp) and three
products are below 2^-21 together: 2^-18 relative, plus the rounding of the
output's type (half its eps)."""
import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2.0 ** -18


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


def randn(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def half_eps(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, rel, floor=0.0):
    """|got - want| <= rel |want| + floor, element by element."""
    got, want = np.asarray(got), np.asarray(want)
    bad = ~(np.abs(got - want) <= rel * np.abs(want) + floor)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5])


def smallest(dtype):
    """Half the spacing of the type's subnormals."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def check(pmpe, x, w, res, eps=1e-6, quant=None, **kw):
    n = pmpe.rms_norm(x, w, residual=res, eps=eps, quant=quant, **kw)
    torch.cuda.synchronize()
    h = f64(x) if res is None else f64(x) + f64(res)
    dt = x.dtype
    if res is None:
        assert n.h is x
    else:
        close(f64(n.h), h, half_eps(dt) + 2.0 ** -24, smallest(dt))
        h = f64(n.h)  # the norm is that of the rounded rows
    y, rstd = ref.rms_norm(h, f64(w), eps)
    close(f64(n.rstd), rstd, REL)
    if quant is None:
        assert n.scale is None and n.y.dtype == dt
        close(f64(n.y), y, half_eps(dt) + REL, smallest(dt))
        return n
    T, H = y.shape
    width = 128 if quant == "block" else H
    assert n.y.dtype == torch.float8_e4m3fn and n.scale.shape == (T, -(-H // width))
    s, q = f64(n.scale), f64(n.y)
    for b in range(s.shape[1]):
        part = y[:, b * width:(b + 1) * width]
        close(s[:, b], np.maximum(np.abs(part).max(1) / 448.0, 2.0 ** -126), 2 * REL)
        back = q[:, b * width:(b + 1) * width] * s[:, b:b + 1]
        # half a step of e4m3: 2^-4 of a normal value, 2^-10 of the scale below
        close(back, part, 2.0 ** -4 + 4 * REL, 2.0 ** -10 * s[:, b:b + 1] * (1 + 4 * REL))
    return n


WIDTHS = [1, 7, 8, 31, 128, 129, 256, 257, 1000, 1001, 1024, 2048, 2056, 4096, 8192, 8200, 16384, 16383]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("H", WIDTHS)
def test_widths(pmpe, H, dtype):
    x, res, w = randn((5, H), H, dtype), randn((5, H), H + 1, dtype, 2.0), randn((H,), H + 2, dtype) + 1
    check(pmpe, x, w, res)
    check(pmpe, x, w.float() if H % 2 else w, None)
    check(pmpe, x, w, res, quant="block")
    check(pmpe, x, w, None, quant="row")


@pytest.mark.parametrize("T,H,dtype", [(1, 2048, BF16), (2, 256, BF16), (1023, 256, BF16), (1024, 256, BF16), (1025, 2048, BF16),
                                       (1100, 512, F16), (1100, 1024, F32), (1030, 2048, F32), (1027, 2040, BF16),
                                       (1027, 2041, BF16), (3000, 136, F16)])
@pytest.mark.parametrize("quant", [None, "block", "row"])
def test_rows(pmpe, T, H, dtype, quant):
    check(pmpe, randn((T, H), T, dtype), randn((H,), 5, dtype) + 1, randn((T, H), T + 1, dtype), quant=quant)


@pytest.mark.parametrize("offset,pitch", [(0, 260), (0, 264), (1, 300), (8, 272), (3, 259)])
def test_pitches_and_alignments(pmpe, offset, pitch):
    buf = randn((9 * pitch + 16,), 3, BF16)
    x = buf[offset:offset + 9 * pitch].view(9, pitch)[:, :256]
    res = randn((9, 256), 4, BF16)
    check(pmpe, x, randn((256,), 5, BF16), res)
    check(pmpe, res, randn((257,), 5, BF16)[1:], x, quant="block")
    check(pmpe, x, randn((256,), 5, F32), None)


@pytest.mark.parametrize("T", [3, 1500])
@pytest.mark.parametrize("where", ["residual", "x"])
def test_h_in_place(pmpe, where, T):
    x, res, w = randn((T, 2048), 1, BF16), randn((T, 2048), 2, BF16), randn((2048,), 3, BF16)
    want = pmpe.rms_norm(x, w, residual=res)
    a, b = x.clone(), res.clone()
    got = pmpe.rms_norm(a, w, residual=b, h_out=b if where == "residual" else a)
    assert torch.equal(got.h, want.h) and torch.equal(got.y, want.y) and torch.equal(got.rstd, want.rstd)
    assert got.h.data_ptr() == (b if where == "residual" else a).data_ptr()


def test_h_beside_its_inputs(pmpe):
    """h_out in the same buffer: refused where it shares memory in another
    order, taken where it lies between rows or after them."""
    w = randn((64,), 1, F32)
    flat = randn((4096,), 2, F32)
    x = flat.as_strided((3, 64), (1000, 1))
    res = randn((3, 64), 3, F32)
    want = pmpe.rms_norm(x, w, residual=res)
    for at in (64, 500, 1000 - 192, 2064, 3000):
        got = pmpe.rms_norm(x, w, residual=res, h_out=flat[at:at + 192].view(3, 64))
        assert torch.equal(got.h, want.h) and torch.equal(got.y, want.y)
    for at in (0, 63, 1000 - 191, 1000, 1063, 2063):
        with pytest.raises(pmpe.PmpeError):
            pmpe.rms_norm(x, w, residual=res, h_out=flat[at:at + 192].view(3, 64))
    rows = randn((4, 64), 4, F32)
    for a, b in ((rows[:3], rows[1:]), (rows[1:], rows[:3])):
        with pytest.raises(pmpe.PmpeError):
            pmpe.rms_norm(res, w, residual=a, h_out=b)
    one = flat.as_strided((1, 64), (1, 1))
    n = pmpe.rms_norm(one, w, residual=res[:1], h_out=flat[64:128].view(1, 64))
    assert torch.equal(n.h, one + res[:1])


@pytest.mark.parametrize("quant", [None, "block", "row"])
@pytest.mark.parametrize("T,H", [(6, 384), (1200, 256)])
def test_rows_of_zeros_infinities_and_nans_stay_in_their_rows(pmpe, T, H, quant):
    x, w = randn((T, H), 1, BF16), randn((H,), 2, BF16) + 2
    clean = pmpe.rms_norm(x, w, quant=quant)
    y = x.clone()
    y[1] = 0
    y[2, 5] = float("inf")
    y[3, 7] = float("nan")
    n = pmpe.rms_norm(y, w, quant=quant)
    keep = [i for i in range(T) if i not in (1, 2, 3)]
    got, want = n.y.float(), clean.y.float()
    assert torch.equal(got[keep], want[keep])
    assert (got[1] == 0).all() and not torch.isnan(n.rstd[1])
    if quant:
        assert torch.equal(n.scale[keep], clean.scale[keep]) and (n.scale[1] == 2.0 ** -126).all()
        assert torch.isnan(n.scale[3]).all() and torch.isnan(got[3]).all()
    else:
        assert torch.isnan(got[2, 5]) and (got[2, :5] == 0).all() and torch.isnan(got[3]).all()


@pytest.mark.parametrize("T", [4, 1300])
@pytest.mark.parametrize("scale", [1e30, 3e18, 1e-18, 1e-30])
def test_values_whose_squares_leave_fp32(pmpe, scale, T):
    check(pmpe, randn((T, 512), 1, F32, scale), randn((512,), 2), None, eps=1e-12)


@pytest.mark.parametrize("dtype,scale", [(BF16, 2.0 ** -128), (F16, 2.0 ** -18)])
def test_sums_below_the_types_normal_values(pmpe, dtype, scale):
    """x + residual is rounded to the type, subnormals included."""
    x, res = randn((4, 256), 1, dtype, scale), randn((4, 256), 2, dtype, scale)
    n = pmpe.rms_norm(x, randn((256,), 3, dtype), residual=res, eps=1e-20)
    torch.cuda.synchronize()
    assert torch.equal(n.h.cpu().double(), (x.cpu().double() + res.cpu().double()).to(dtype).double())


def test_no_rows_and_refusals(pmpe):
    w = randn((64,), 1, BF16)
    n = pmpe.rms_norm(torch.empty((0, 64), dtype=BF16, device="cuda"), w, quant="block")
    assert n.y.shape == (0, 64) and n.scale.shape == (0, 1) and n.rstd.shape == (0,)
    x = randn((4, 64), 2, BF16)
    for bad in (dict(x=x.t().contiguous().t()), dict(x=x.double()), dict(x=x[0]), dict(weight=w[:63]), dict(weight=w.half()),
                dict(weight=w.cpu()), dict(residual=x.half()), dict(residual=x[:3]), dict(quant="int8"), dict(h_out=x),
                dict(eps=0.0), dict(x=x[:1].expand(4, 64)), dict(residual=x, h_out=x.t().contiguous().t())):
        with pytest.raises(pmpe.PmpeError):
            pmpe.rms_norm(**dict(dict(x=x, weight=w), **bad))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_weights_that_are_not_the_rows_are_refused(pmpe, dtype):
    x, w, rstd = randn((4, 64), 2, dtype), randn((64,), 1, dtype), torch.ones(4, device="cuda")
    other = F16 if dtype is BF16 else BF16
    for bad in (w.to(other), w.double(), w[:63], w.float()[:63], w.cpu(), w.float().cpu(), w[None], w[:1].expand(64), torch.ones(65, device="cuda"),
                torch.ones(128, device="cuda")[::2], torch.ones(0, device="cuda")):
        with pytest.raises(pmpe.PmpeError, match="weight is"):
            pmpe.rms_norm(x, bad)
        with pytest.raises(pmpe.PmpeError, match="weight is"):
            pmpe.rms_norm_backward(x, x, bad, rstd)


# ------------------------------------------------------------- backward

def check_backward(pmpe, T, H, dtype, gtype=None, xtype=None, d_h=True, wtype=None, seed=0):
    gtype, xtype, wtype = gtype or dtype, xtype or dtype, wtype or dtype
    h, w = randn((T, H), seed + 1, dtype), randn((H,), seed + 2, wtype) + 1
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-6).float()
    dy, dh = randn((T, H), seed + 3, gtype), randn((T, H), seed + 4, xtype) if d_h else None
    dx, dw = pmpe.rms_norm_backward(dy, h, w, rstd, d_h=dh, dx_dtype=xtype)
    torch.cuda.synchronize()
    rx, rw, sx, sw = ref.rms_norm_backward(f64(dy), f64(h), f64(w), f64(rstd), None if dh is None else f64(dh))
    # dx: a handful of FP32 roundings of each term, 26 in the mean's tree;
    # dw: at most 33 rows in sequence (T = 4900 over 152 CTAs), 29 partials (of
    # 1824) a strand, 64 strands in seven steps: 69 x 2^-24 < 2^-17
    assert dx.dtype == xtype and dw.dtype == F32
    close(f64(dx), rx, half_eps(xtype), sx * REL + smallest(xtype))
    close(f64(dw), rw, 0.0, sw * 2.0 ** -16 + 1e-30)
    only, none = pmpe.rms_norm_backward(dy, h, w, rstd, d_h=dh, dx_dtype=xtype, need_dw=False)
    assert none is None and torch.equal(only, dx)
    again, dw2 = pmpe.rms_norm_backward(dy, h, w, rstd, d_h=dh, dx_dtype=xtype)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)  # the same sums in the same order


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("H", WIDTHS)
def test_backward_widths(pmpe, H, dtype):
    check_backward(pmpe, 5, H, dtype)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 607, 608, 609, 2000, 4900])
@pytest.mark.parametrize("H", [256, 320, 2048, 1001, 8200])
def test_backward_rows(pmpe, T, H):
    check_backward(pmpe, T, H, BF16, gtype=F32, d_h=T % 2 == 0)


@pytest.mark.parametrize("gtype,xtype,wtype", [(F32, F32, BF16), (BF16, F32, F32), (F32, BF16, F32), (BF16, BF16, F32)])
def test_backward_types(pmpe, gtype, xtype, wtype):
    check_backward(pmpe, 33, 512, BF16, gtype, xtype, True, wtype)
    check_backward(pmpe, 700, 320, BF16, gtype, xtype, False, wtype)


def test_backward_against_differences(pmpe):
    """The forward's own change along a direction, in FP32: with steps of 2^-6
    of the rows, the difference quotient is off by step^2 (the third
    derivative, of the size of the gradient here) and by y's rounding over the
    step, 2^-18 x sqrt(T H) |dy| / 2^-6 in the worst case."""
    T, H, step = 6, 320, 2.0 ** -6
    h, w, dy, v = (randn(s, i, F32) for i, s in ((1, (T, H)), (2, (H,)), (3, (T, H)), (4, (T, H))))
    n = pmpe.rms_norm(h, w)
    dx, _ = pmpe.rms_norm_backward(dy, h, w, n.rstd)
    up, down = pmpe.rms_norm(h + step * v, w).y, pmpe.rms_norm(h - step * v, w).y
    quotient = ((up.double() - down.double()) * dy.double()).sum().item() / (2 * step)
    along = (dx.double() * v.double()).sum().item()
    bound = (dy.double() * n.y.double()).norm().item() * (2.0 ** -18 / step * 2 + 16 * step ** 2)
    assert abs(quotient - along) <= bound, (quotient, along, bound)


@pytest.mark.parametrize("T,H", [(300, 2048), (40, 256), (33, 1001), (500, 8192)])
def test_backward_does_not_go_by_the_workspaces_address(pmpe, T, H):
    """Any 16-byte aligned workspace of the size asked for gives the same bits,
    and so does none where there is no weight's gradient; nothing is written
    past its end or before it."""
    from test_operators_abi import RmsNormBackwardDesc, desc
    h, dy, w = randn((T, H), 1, BF16), randn((T, H), 2, BF16), randn((H,), 3, BF16)
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-6).float()
    need = pmpe._lib.pmpe_rms_norm_backward_workspace_size(T, H)
    got = []
    for at in (0, 16, 32, 48, None):
        ws = torch.full((need + 128,), 77, dtype=torch.uint8, device="cuda")
        dx, dw = torch.empty_like(h), torch.empty(H, device="cuda")
        base = dict(T=T, H=H, type=1, weight_type=1, dy_type=1, dx_type=1, dy=dy.data_ptr(), h=h.data_ptr(), weight=w.data_ptr(),
                    rstd=rstd.data_ptr(), d_h=None, dx=dx.data_ptr(), dw=dw.data_ptr(), workspace=ws.data_ptr() + (at or 0), workspace_bytes=need)
        if at is None:
            base.update(dw=None, workspace=ws.data_ptr() + 16, workspace_bytes=0)
        torch.cuda.synchronize()
        assert pmpe._lib.pmpe_rms_norm_backward(desc(RmsNormBackwardDesc, base), None) == pmpe.OK
        torch.cuda.synchronize()
        assert (ws[:at or 0] == 77).all() and (ws[(at or 0) + need:] == 77).all()
        assert at is not None or (ws == 77).all()
        got.append((dx, dw))
    for dx, dw in got[1:]:
        assert torch.equal(dx, got[0][0])
        assert dw is got[-1][1] or torch.equal(dw, got[0][1])


@pytest.mark.parametrize("T,H", [(400_000, 4104), (2 * 38_912 + 77, 8200), (466_945, 300), (2 * 933_888 + 5, 8), (933_888, 8), (38_912, 4104)])
def test_backward_weights_sum_over_many_rows(pmpe, T, H):
    """The weight gradient's error does not grow with the rows: 256 of a thread
    in sequence, eight warps, 29 partials a strand, seven steps of their tree,
    four of the pairs, two roundings of a term: 306 x 2^-24 of the terms'
    magnitudes.  Terms of one size and sign are the worst case for a sequence."""
    g = torch.Generator("cuda").manual_seed(T)
    h = torch.ones((T, H), dtype=BF16, device="cuda")
    rstd = torch.full((T,), 0.7, device="cuda")
    w = torch.ones(H, dtype=BF16, device="cuda")
    for dy in (torch.full((T, H), 1.1, dtype=BF16, device="cuda"), torch.rand((T, H), generator=g, device="cuda", dtype=BF16) - 0.25):
        dx, dw = pmpe.rms_norm_backward(dy, h, w, rstd)
        want, size = (sum(f(p.double()).sum(0) for p in dy.split(20000)) * float(rstd[0]) for f in (lambda v: v, torch.abs))
        assert ((dw.double() - want).abs() <= 306 * 2.0 ** -24 * size).all(), float(((dw.double() - want).abs() / size).max() * 2 ** 24)
        tail, _ = pmpe.rms_norm_backward(dy[-9:].contiguous(), h[-9:].contiguous(), w, rstd[-9:].contiguous())
        assert torch.equal(dx[-9:], tail)
        only, none = pmpe.rms_norm_backward(dy, h, w, rstd, need_dw=False)
        assert none is None and torch.equal(only, dx)


def test_backward_no_rows(pmpe):
    e = torch.empty((0, 64), dtype=BF16, device="cuda")
    dx, dw = pmpe.rms_norm_backward(e, e, randn((64,), 1, BF16), torch.empty(0, device="cuda"))
    torch.cuda.synchronize()
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_other_stream_and_graph(pmpe):
    T, H = 1300, 2048
    x, res, w = randn((T, H), 1, BF16), randn((T, H), 2, BF16), randn((H,), 3, BF16)
    dy = randn((T, H), 4, F32)
    want = pmpe.rms_norm(x, w, residual=res)
    wx, ww = pmpe.rms_norm_backward(dy, want.h, w, want.rstd, d_h=res)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    n = pmpe.rms_norm(x, w, residual=res, stream=s)
    gx, gw = pmpe.rms_norm_backward(dy, n.h, w, n.rstd, d_h=res, stream=s)
    s.synchronize()
    assert torch.equal(n.y, want.y) and torch.equal(gx, wx) and torch.equal(gw, ww)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        n = pmpe.rms_norm(x, w, residual=res)
        gx, gw = pmpe.rms_norm_backward(dy, n.h, w, n.rstd, d_h=res)
    for seed in (7, 8):
        x.copy_(randn((T, H), seed, BF16))
        g.replay()
        torch.cuda.synchronize()
        e = pmpe.rms_norm(x, w, residual=res)
        ex, ew = pmpe.rms_norm_backward(dy, e.h, w, e.rstd, d_h=res)
        assert torch.equal(n.y, e.y) and torch.equal(gx, ex) and torch.equal(gw, ew)


def test_arguments_freed_while_the_other_stream_has_yet_to_run(pmpe):
    """The memory of a call's arguments is not handed out again before the
    stream that it was given is done with them."""
    w = randn((2048,), 1, BF16)
    x, res = randn((300, 2048), 2, BF16), randn((300, 2048), 3, BF16)
    want = pmpe.rms_norm(x, w, residual=res).y.clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)  # some 10 ms
    got = pmpe.rms_norm(x, w, residual=res, stream=s)
    del x, res
    other = [torch.full((300, 2048), 7.0, dtype=BF16, device="cuda") for _ in range(4)]
    y = got.y
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and all((o == 7).all() for o in other)


def test_two_threads_at_once(pmpe):
    """Calls of two threads, a stream each, do not disturb one another."""
    import threading
    x = [randn((64, 2048), i, BF16) for i in range(2)]
    w = randn((2048,), 3, BF16)
    want = [pmpe.rms_norm(v, w, residual=v).y for v in x]
    torch.cuda.synchronize()
    same = [False, False]

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got = [pmpe.rms_norm(x[i], w, residual=x[i]).y for _ in range(300)]
        s.synchronize()
        same[i] = all(torch.equal(g, want[i]) for g in got)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert same == [True, True]


def test_more_than_2_to_31_elements(pmpe):
    """Offsets past 32 bits: the last rows are those of a call on them alone."""
    T, H = 140000, 16384
    x = torch.empty((T, H), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    w = randn((H,), 2, F32)
    few = x[-5:].clone()
    n, m = pmpe.rms_norm(x, w, residual=x), pmpe.rms_norm(few, w, residual=few)
    q, r = pmpe.rms_norm(x, w, quant="block"), pmpe.rms_norm(few, w, quant="block")
    for a, b in ((n.y, m.y), (n.h, m.h), (n.rstd, m.rstd), (q.y.view(torch.uint8), r.y.view(torch.uint8)), (q.scale, r.scale)):
        assert torch.equal(a[-5:], b)
    del q
    dx, dw = pmpe.rms_norm_backward(x, n.h, w, n.rstd, d_h=x)
    small, _ = pmpe.rms_norm_backward(few, m.h, w, m.rstd, d_h=few)
    assert torch.equal(dx[-5:], small)
    want, size = torch.zeros(H, dtype=torch.float64, device="cuda"), torch.zeros(H, dtype=torch.float64, device="cuda")
    for t in range(0, T, 10000):
        part = x[t:t + 10000].double() * n.h[t:t + 10000].double() * n.rstd[t:t + 10000, None].double()
        want += part.sum(0)
        size += part.abs().sum(0)
    # a CTA's rows in sequence (140000 / 152), five sums of the CTAs' and the strands' tree
    assert ((dw.double() - want).abs() <= (140000 / 152 + 20) * 2.0 ** -24 * size).all()
