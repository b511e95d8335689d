"""Router.route and Router.backward against 64-bit references.

The selection has to be the reference's exactly.  Weights: an FP32 exponential
of a difference of logits is off by 2^-24 times that difference (below 40 in
these inputs' chosen experts) and 2 ulp, a sum of 256 terms by 13 x 2^-24:
2^-17 relative covers them."""
import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2.0 ** -17


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import pmpe as m
    return m


def make(T, E_pub, E_priv, seed, dtype=F32, bias=False, pitch=None):
    g = torch.Generator().manual_seed(seed)
    E = E_pub + E_priv
    wide = (1.5 * torch.randn((T, pitch or E), generator=g)).to(dtype).cuda()
    policy = torch.randint(0, 3, (T,), generator=g).to(torch.uint8).cuda() if E_priv else None
    b = (0.05 * torch.randn((E,), generator=g)).cuda() if bias else None
    return wide[:, :E], policy, b


def n64(t):
    return None if t is None else t.double().cpu().numpy()


def host(t):
    return None if t is None else t.cpu().numpy()


def check(pmpe, logits, policy, bias, E_pub, E_priv, k, score="softmax", renorm=True, scale=1.0, groups=(1, 1), groups_priv=(1, 1),
          group_score="max", backward=True, stream=None):
    r = pmpe.Router(E_pub, E_priv, k, score=score, renormalize=renorm, scale=scale, groups=groups, groups_priv=groups_priv,
                    group_score=group_score)
    load = torch.full((E_pub + E_priv,), 3, dtype=torch.int32, device="cuda")
    idx, w = r.route(logits, policy, bias=bias, load=load)
    torch.cuda.synchronize()
    ri, rw = ref.route(n64(logits), host(policy), E_pub, E_priv, k, score == "sigmoid", renorm, scale, n64(bias), groups, groups_priv,
                       group_score == "top2")
    got = host(idx)
    assert np.array_equal(got, ri), (np.argwhere((got != ri).any(1))[:3], got[(got != ri).any(1)][:3], ri[(got != ri).any(1)][:3])
    gw = n64(w)
    assert (np.abs(gw - rw) <= REL * np.abs(rw) + 2.0 ** -126).all(), np.abs(gw - rw).max()
    assert (gw[ri < 0] == 0).all()
    count = np.bincount(ri[ri >= 0], minlength=E_pub + E_priv)
    assert np.array_equal(host(load), count + 3)  # added to what was there
    if not backward:
        return
    g = torch.Generator().manual_seed(99)
    dw = torch.randn(idx.shape, generator=g).cuda()
    d = r.backward(logits, policy, idx, dw)
    torch.cuda.synchronize()
    assert d.dtype == logits.dtype and d.shape == logits.shape
    rd, size = ref.route_backward(n64(logits), host(policy), ri, n64(dw), E_pub, E_priv, score == "sigmoid", renorm, scale)
    eps = torch.finfo(logits.dtype)
    bad = ~(np.abs(n64(d) - rd) <= eps.eps / 2 * np.abs(rd) + 2 * REL * size + eps.smallest_normal * eps.eps / 2)
    assert not bad.any(), (np.argwhere(bad)[:4], n64(d)[bad][:4], rd[bad][:4])


POOLS = [(4, 0, 1), (8, 0, 8), (16, 4, 2), (33, 31, 5), (64, 16, 6), (128, 32, 8), (128, 128, 12), (160, 0, 6), (255, 17, 7),
         (256, 0, 8), (256, 256, 32), (40, 32, 32)]


@pytest.mark.parametrize("E_pub,E_priv,k", POOLS)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_pools(pmpe, E_pub, E_priv, k, score, dtype):
    for renorm, bias in ((True, False), (False, True)):
        z, policy, b = make(37, E_pub, E_priv, E_pub + k, dtype, bias)
        check(pmpe, z, policy, b, E_pub, E_priv, k, score, renorm, 2.5 if bias else 1.0)


@pytest.mark.parametrize("E_pub,groups,k", [(16, (4, 2), 4), (64, (8, 3), 6), (256, (8, 4), 8), (256, (32, 5), 8), (160, (8, 3), 6),
                                            (96, (3, 1), 5), (30, (10, 7), 3), (7, (7, 3), 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_groups(pmpe, E_pub, groups, k, score, group_score):
    for bias, dtype in ((False, F32), (True, BF16)):
        z, policy, b = make(41, E_pub, 32, 7, dtype, bias)
        check(pmpe, z, policy, b, E_pub, 32, k, score, True, 2.5, groups, (4, 2), group_score)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 130, 4875])
def test_tokens(pmpe, T):
    z, policy, b = make(T, 128, 32, T, F32, True)
    check(pmpe, z, policy, b, 128, 32, 8, "sigmoid", True, 2.5, (8, 4), (1, 1), "top2")


@pytest.mark.parametrize("pitch", [160, 161, 164, 168, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pitches(pmpe, pitch, dtype):
    z, policy, _ = make(19, 128, 32, 3, dtype, pitch=pitch)
    check(pmpe, z, policy, None, 128, 32, 8, renorm=False)
    check(pmpe, z[1:], policy[1:].clone(), None, 128, 32, 8)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masked_experts(pmpe, score, renorm):
    """Rows with fewer eligible experts than k, none, infinities, NaN, the
    type's lowest value: what is left is chosen and nothing spreads."""
    z, policy, b = make(12, 16, 8, 5, F32, True)
    policy[:] = 0
    policy[6:] = 1
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, 3] = 0.5
    z[2, 1:] = float("nan")
    z[3, 5] = np.inf
    z[4, :16] = torch.finfo(F32).min
    z[5, ::2] = -np.inf
    z[6] = float("nan")
    z[7, 16:20] = -np.inf
    z[8, :16] = float("nan")  # the other pool of an ALLOW token
    for bias in (None, b):
        check(pmpe, z, policy, bias, 16, 8, 4, score, renorm)
        check(pmpe, z, policy, bias, 16, 8, 4, score, renorm, 1.0, (4, 2), (2, 1), "top2")
    b[2] = -np.inf  # an expert taken out by its bias
    check(pmpe, z, policy, b, 16, 8, 4, score, renorm)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [64, 60])  # groups of whole lanes, and others
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_extreme_biases(pmpe, score, E, group_score):
    """Experts forced by a bias of +inf, masked by the type's lowest value or
    by -inf, and the largest finite bias: sums of two that pass FP32's range."""
    z, _, _ = make(9, E, 0, 21)
    size = E // 4
    low, high = torch.finfo(F32).min, torch.finfo(F32).max
    z[1, :size] = -np.inf  # a group without a candidate before those of the lowest value
    for kind in range(6):
        b = 0.05 * torch.randn(E, generator=torch.Generator().manual_seed(kind))
        if kind == 0:  # fewer, as many and more than k
            b[[3, 17, 40]] = np.inf
        elif kind == 1:
            b[[3, 5, 17, 40, 41]] = np.inf
        elif kind == 2:
            b[::2] = np.inf
        elif kind == 3:
            b[:] = low
        elif kind == 4:
            b[size:] = low
            b[:size:3] = -np.inf
        else:
            b[2 * size:] = high
            b[0] = low
        b = b.cuda()
        check(pmpe, z, None, b, E, 0, 5, score, True, backward=False)
        check(pmpe, z, None, b, E, 0, 5, score, False, 2.5, (4, 2), (1, 1), group_score, backward=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_near_ties(pmpe, score):
    """Logits and biases that FP32 scores cannot tell apart: the selection is
    that of 64 bits, equal values by the lower id."""
    g = torch.Generator().manual_seed(11)
    T, E = 64, 64
    z = torch.randn((T, 1), generator=g).expand(T, E).clone()
    z += torch.randint(-3, 4, (T, E), generator=g) * 2.0 ** -23  # a few ulps apart
    z = z.cuda()
    check(pmpe, z, None, None, E, 0, 8, score)
    b = (torch.randint(-2, 3, (E,), generator=g) * 2.0 ** -26).cuda()
    check(pmpe, z, None, b, E, 0, 8, score)
    check(pmpe, z, None, b, E, 0, 32, score)
    check(pmpe, z, None, b, E, 0, 8, score, True, 1.0, (8, 3), (1, 1), "top2")
    check(pmpe, z, None, None, E, 0, 8, score, True, 1.0, (8, 3), (1, 1), "top2")
    check(pmpe, z, None, b, E, 0, 8, score, True, 1.0, (8, 3), (1, 1), "max")
    same = torch.zeros((5, E), device="cuda")
    check(pmpe, same, None, torch.zeros(E, device="cuda"), E, 0, 8, score)
    z16 = torch.randn((200, E), generator=g).to(BF16).cuda()  # many true ties
    check(pmpe, z16, None, torch.zeros(E, device="cuda"), E, 0, 8, score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("top2", [False, True])
def test_near_ties_of_many_tokens(pmpe, score, top2):
    """Most tokens of a long batch in doubt at once, several of each CTA: the
    selection against a sort of 64-bit choices, with the loads."""
    T, E, k = 12001, 32, 5
    g = torch.Generator().manual_seed(17)
    z = (torch.randn((T, 1), generator=g).expand(T, E) + torch.randint(-3, 4, (T, E), generator=g) * 2.0 ** -22).float().cuda()
    b = (torch.randint(-2, 3, (E,), generator=g) * 2.0 ** -25).cuda()
    load = torch.zeros(E, dtype=torch.int32, device="cuda")
    idx, w = pmpe.Router(E, 0, k, score=score, groups=(4, 2), group_score="top2" if top2 else "max").route(z, bias=b, load=load)
    torch.cuda.synchronize()
    s = 1 / (1 + torch.exp(-z.double())) if score == "sigmoid" else torch.softmax(z.double(), 1)
    c = s + b.double()
    v = torch.sort(c.view(T, 4, 8), dim=2, descending=True).values
    v = v[:, :, 0] + v[:, :, 1] if top2 else v[:, :, 0]
    kept = torch.zeros((T, 4), dtype=torch.bool, device="cuda")
    kept.scatter_(1, torch.sort(v, dim=1, descending=True, stable=True).indices[:, :2], True)
    c = torch.where(kept.repeat_interleave(8, 1), c, -1.0)
    want = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    # torch's own softmax and this reference may round a sum differently: 64-bit
    # choices within 2^-50 of one another have no order to hold to
    a, d = torch.gather(c, 1, idx.long()), torch.gather(c, 1, want)
    assert ((a - d).abs() <= 2.0 ** -50).all()
    assert (idx == want).double().mean() > 0.999
    assert torch.equal(load, torch.bincount(idx.flatten().long(), minlength=E).int())
    weights = torch.gather(s, 1, idx.long())
    assert (w.double() - weights / weights.sum(1, keepdim=True)).abs().max() <= REL


def choices64(z, bias, score, groups=None, top2=False):
    """64-bit choices of one pool; the experts of the groups left out at -inf."""
    s = 1 / (1 + torch.exp(-z.double())) if score == "sigmoid" else torch.softmax(z.double(), 1)
    c = s + bias.double()
    if groups:
        v = torch.sort(c.unflatten(1, (groups[0], -1)), dim=2, descending=True).values
        v = v[:, :, 0] + v[:, :, 1] if top2 else v[:, :, 0]
        kept = torch.zeros(v.shape, dtype=torch.bool, device="cuda")
        kept.scatter_(1, torch.sort(v, dim=1, descending=True, stable=True).indices[:, :groups[1]], True)
        c = torch.where(kept.repeat_interleave(z.shape[1] // groups[0], 1), c, -torch.inf)
    return c


def same_choices(idx, c, k):
    """The k largest in order, equal ones by the lower id; choices that 64 bits
    hardly tell apart (torch's own sums may round them another way) as they come."""
    want = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    a, d = torch.gather(c, 1, idx.long()), torch.gather(c, 1, want)
    off = idx.long() != want
    assert ((a - d).abs() <= 2.0 ** -50)[off].all(), (int(off.any(1).sum()), float((a - d).abs().max()))
    assert off.any(1).double().mean() < 1e-3


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("std,mean", [(3.0, 0.0), (5.0, 0.0), (8.0, 0.0), (1.5, -15.0)])
@pytest.mark.parametrize("bias", [0.0, 0.3])
def test_wide_logits_with_equal_biases(pmpe, score, std, mean, bias):
    """Where most scores are small, or saturated, most tokens are settled in 64 bits."""
    T, E, k = 3001, 256, 8
    z = (std * torch.randn((T, E), generator=torch.Generator().manual_seed(int(std * 10))) + mean).cuda()
    b = torch.full((E,), bias, device="cuda")
    idx, _ = pmpe.Router(E, 0, k, score=score).route(z, bias=b)
    same_choices(idx, choices64(z, b, score), k)


@pytest.mark.parametrize("mask", [-100.0, -1e4, -1e9, torch.finfo(F32).min, -np.inf])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_with_masked_biases(pmpe, score, mask):
    """One expert in sixteen masked by its bias, at a prompt's size: the bound on
    the groups' sums goes by the largest choice, the result does not."""
    T, E, k = 8192, 256, 8
    g = torch.Generator().manual_seed(5)
    z, b = (1.5 * torch.randn((T, E), generator=g)).to(BF16).cuda(), (0.05 * torch.randn(E, generator=g)).cuda()
    b[::16] = mask
    idx, _ = pmpe.Router(E, 0, k, score=score, groups=(8, 4), group_score="top2").route(z, bias=b)
    c = choices64(z, b, score, (8, 4), True)
    same_choices(idx, torch.where(c > mask / 2, c, -torch.inf), k)  # no masked one is among them
    assert (idx % 16 != 0).all()


@pytest.mark.parametrize("edge", [0.75, 0.5 + 2.0 ** -9, 0.6875])
def test_choices_at_the_edge_of_a_packed_word(pmpe, edge):
    """The best two choices within a few ulps on either side of a value where
    the packed words change, a third one below that shares the second's word:
    the order is that of 64 bits."""
    g = torch.Generator().manual_seed(23)
    T = 100000
    at = float(np.log(edge / (1 - edge)))
    close = at + torch.randint(-12, 13, (T, 2), generator=g, dtype=torch.float64) * 2.0 ** -23
    third = edge - 2.0 ** -16 * torch.rand((T, 1), generator=g, dtype=torch.float64)
    z = torch.cat([torch.log(third / (1 - third)), close], 1).float().cuda()
    for order in ([0, 1, 2], [1, 0, 2], [1, 2, 0]):
        zo = z[:, order].contiguous()
        want = torch.sort(1 / (1 + torch.exp(-zo.double())), dim=1, descending=True, stable=True).indices
        for k in (1, 2):
            idx, _ = pmpe.Router(3, 0, k, score="sigmoid").route(zo, bias=torch.zeros(3, device="cuda"))
            assert torch.equal(idx.long(), want[:, :k]), (order, k, int((idx.long() != want[:, :k]).any(1).sum()))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_rows_of_equal_logits(pmpe, score, group_score):
    """Padding: every choice of a row is the same, or all but one."""
    z, policy, b = make(24, 64, 30, 31, F32, True)
    z[::2] = 0.0
    z[1::4] = -1.5
    z[2, 5] = 2.0 ** -24
    z[4, 63] = -np.inf
    z[6, 64:] = float("nan")
    z[8] = np.inf
    for bias in (None, torch.zeros_like(b), torch.full_like(b, 0.3), b):
        check(pmpe, z, policy, bias, 64, 30, 6, score, True, 1.0, (8, 3), (10, 4), group_score)


def test_saturated_sigmoids(pmpe):
    """Sigmoids that round to 1 in 64 bits too are equal: the lower id."""
    g = torch.Generator().manual_seed(13)
    z = (60 * torch.randn((40, 32), generator=g)).cuda()
    check(pmpe, z, None, torch.zeros(32, device="cuda"), 32, 0, 6, "sigmoid", backward=False)


def test_backward_ignores_foreign_ids_and_adds_repeated_ones(pmpe):
    z, policy, _ = make(6, 16, 8, 2)
    policy[:] = 0
    r = pmpe.Router(16, 8, 3, renormalize=False)
    idx = torch.tensor([[1, 1, 2], [-1, 5, 20], [3, 99, 4], [16, 17, 18], [0, 1, 2], [-7, -2 ** 31, 15]], dtype=torch.int32).cuda()
    dw = torch.randn((6, 3), generator=torch.Generator().manual_seed(1)).cuda()
    d = r.backward(z, policy, idx, dw)
    torch.cuda.synchronize()
    rd, size = ref.route_backward(n64(z), host(policy), host(idx), n64(dw), 16, 8, False, False, 1.0)
    assert (np.abs(n64(d) - rd) <= 2 * REL * size + 1e-30).all()


def test_no_tokens_and_refusals(pmpe):
    r = pmpe.Router(16, 4, 2)
    z, policy, b = make(3, 16, 4, 1, F32, True)
    idx, w = r.route(z[:0], policy[:0])
    assert idx.shape == (0, 2) and w.shape == (0, 2) and r.backward(z[:0], policy[:0], idx, w).shape == (0, 20)
    good = dict(logits=z, policy=policy, bias=b)
    for bad in (dict(logits=z[:, :19]), dict(logits=z.double()), dict(logits=z.t().contiguous().t()), dict(policy=policy[:2]),
                dict(policy=policy.int()), dict(policy=policy.cpu()), dict(bias=b[:19]), dict(bias=b.half()),
                dict(load=torch.zeros(20, device="cuda")), dict(load=torch.zeros(19, dtype=torch.int32, device="cuda")),
                dict(logits=z[:1].expand(3, 20))):
        with pytest.raises(pmpe.PmpeError):
            r.route(**dict(good, **bad))
    idx, w = r.route(**good)
    with pytest.raises(pmpe.PmpeError):
        r.backward(z, policy, idx.long(), w)
    with pytest.raises(pmpe.PmpeError):
        r.backward(z, policy, idx, w[:2])
    with pytest.raises(pmpe.PmpeError):
        pmpe.Router(20, 0, 2).route(z, policy)  # a policy without a private pool


def test_other_stream_and_graph(pmpe):
    z, policy, b = make(700, 128, 32, 4, F32, True)
    r = pmpe.Router(128, 32, 8, score="sigmoid")
    idx, w = r.route(z, policy, bias=b)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    i2, w2 = r.route(z, policy, bias=b, stream=s)
    d2 = r.backward(z, policy, i2, w2, stream=s)
    s.synchronize()
    assert torch.equal(idx, i2) and torch.equal(w, w2) and torch.equal(d2, r.backward(z, policy, idx, w))
    load = torch.zeros(160, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        i3, w3 = r.route(z, policy, bias=b, load=load)
        d3 = r.backward(z, policy, i3, w3)
    z.copy_(make(700, 128, 32, 5)[0])
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    i4, w4 = r.route(z, policy, bias=b)
    assert torch.equal(i3, i4) and torch.equal(w3, w4) and torch.equal(d3, r.backward(z, policy, i4, w4))
    assert int(load.sum()) == 2 * 700 * 8


def test_more_than_2_to_31_logits(pmpe):
    """Offsets past 32 bits: the last tokens are those of a call on them alone."""
    T, E = 8_400_000, 256
    z = torch.empty((T, E), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    b = 0.05 * torch.randn(E, generator=torch.Generator().manual_seed(2)).cuda()
    r = pmpe.Router(E, 0, 4, score="sigmoid", groups=(8, 4), group_score="top2")
    load = torch.zeros(E, dtype=torch.int32, device="cuda")
    idx, w = r.route(z, bias=b, load=load)
    few = z[-500:].clone()
    i2, w2 = r.route(few, bias=b)
    assert torch.equal(idx[-500:], i2) and torch.equal(w[-500:], w2) and int(load.sum(dtype=torch.int64)) == 4 * T
    assert torch.equal(r.backward(z, None, idx, w)[-500:], r.backward(few, None, i2, w2))
