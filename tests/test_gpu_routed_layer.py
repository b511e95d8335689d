"""The layer with a given route, and the operators around it run together as
a wrapped model's block runs them: norm, routing, experts, and the way back to
the clipped gradients."""
import numpy as np
import pytest
import torch

from paper_2608_06690_gb300 import pmpe
from paper_2608_06690_gb300.inputs import LayerShape
from pmpe_testlib import make_layer, to_device

pytestmark = pytest.mark.gpu

SHAPES = {
    "renorm": (LayerShape(T=300, H=384, I=256, E_pub=24, E_priv=8, E_sh=0, k=4, renormalize=True), 11, "iid"),
    "pool_softmax_shared": (LayerShape(T=200, H=256, I=256, E_pub=16, E_priv=8, E_sh=2, k=3, renormalize=False), 12, "iid"),
    "one_token": (LayerShape(T=1, H=256, I=128, E_pub=8, E_priv=4, E_sh=1, k=2, renormalize=True), 13, "allow"),
    "tile_edges": (LayerShape(T=129, H=256, I=128, E_pub=40, E_priv=16, E_sh=0, k=12, renormalize=True), 14, "iid"),
    "no_policy": (LayerShape(T=256, H=256, I=128, E_pub=8, E_priv=4, E_sh=0, k=4, renormalize=True), 15, "none"),
    "large_experts_decode": (LayerShape(T=70, H=2048, I=768, E_pub=32, E_priv=16, E_sh=1, k=8, renormalize=True), 17, "iid"),
    "large_experts": (LayerShape(T=700, H=2048, I=768, E_pub=128, E_priv=32, E_sh=0, k=8, renormalize=True), 16, "iid"),
}


def build(name):
    shape, seed, policy = SHAPES[name]
    wd, hd, pd = to_device(*make_layer(shape, seed, policy=policy))
    return shape, pmpe.MoeLayer(shape, wd), hd, pd, seed


def own_route(shape, layer, h, pol, audit=None):
    idx = torch.empty((shape.T, shape.k), dtype=torch.int32, device="cuda")
    w = torch.empty((shape.T, shape.k), dtype=torch.float32, device="cuda")
    out = layer.forward(h, pol, topk_idx=idx, topk_w=w, audit=audit)
    return out, idx, w


def new_audit(shape):
    return torch.zeros(pmpe.audit_words(shape.T, shape.E), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("name", list(SHAPES))
def test_the_layers_own_route_given_back(name, saved):
    """Same rows in the same order: the output, the private experts' gradients
    and the audit are the layer's own, bit by bit."""
    shape, layer, h, pol, seed = build(name)
    dout = torch.randn((shape.T, shape.H), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
    a, b = new_audit(shape), new_audit(shape)
    want, idx, w = own_route(shape, layer, h, pol, a)
    grads, d_hidden = layer.backward(h, pol, dout)
    want, grads, d_hidden = want.clone(), {n: g.clone() for n, g in grads.items()}, d_hidden.clone()
    got = layer.forward(h, pol, route=(idx, w), audit=b, save_for_backward=saved)
    g, dh, dw = layer.backward_routed(h, pol, dout)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert torch.equal(a, b)
    for n in ("d_gate", "d_up", "d_down"):
        assert torch.equal(g[n], grads[n]), n
    assert set(g) == {"d_gate", "d_up", "d_down"}
    # the router's part, from d_w on, gives what the layer's own backward has
    # besides: the same FP32 sums in another order, over H and T terms
    allow = torch.zeros(shape.T, dtype=torch.bool, device="cuda") if pol is None else pol == 1
    wr = [layer.weights["router_pub"].double(), layer.weights["router_priv"].double()]
    logits = torch.cat([h.double() @ r.T for r in wr], 1)
    d = pmpe.Router(shape.E_pub, shape.E_priv, shape.k, renormalize=shape.renormalize).backward(logits.float(), pol, idx, dw)
    total = dh.double() + d.double() @ torch.cat(wr)
    # an FP32 dot product of up to 256 experts and k picks, and w's own error
    bound = 2.0 ** -14 * (dh.double().abs() + d.double().abs() @ torch.cat(wr).abs() + d_hidden.double().abs()) + 1e-7 * float(dw.abs().max())
    assert ((total - d_hidden.double()).abs() <= bound).all()
    dr = d.double()[:, shape.E_pub:].T @ h.double()
    size = d.double()[:, shape.E_pub:].abs().T @ h.double().abs()
    slack = 1e-6 * float(dw.abs().max()) * h.double().abs().sum(0)[None, :]  # a gradient's own rounding, 2^-20 of d_w, on every token
    assert ((dr - grads["d_router"].double()).abs() <= 2.0 ** -14 * size + slack).all()
    assert (d[allow][:, :shape.E_pub] == 0).all() and (d[~allow][:, shape.E_pub:] == 0).all()


LARGE = {
    "prefill": LayerShape(T=4096, H=2048, I=768, E_pub=128, E_priv=32, E_sh=0, k=8, renormalize=True),
    "largest_prefill": LayerShape(T=16384, H=2048, I=768, E_pub=128, E_priv=32, E_sh=0, k=8, renormalize=True),
    "shared_pool_softmax": LayerShape(T=8191, H=2048, I=1408, E_pub=64, E_priv=16, E_sh=2, k=6, renormalize=False),
    "small_experts": LayerShape(T=5001, H=256, I=128, E_pub=40, E_priv=16, E_sh=1, k=6, renormalize=True),
}


@pytest.mark.parametrize("name", list(LARGE) + ["large_experts_decode", "one_token"])
def test_a_given_route_after_another_batch(name):
    """Prompt batches of up to 129 router tiles, and small ones: with the
    workspace as another batch left it, the own route given back gives the
    layer's output, audit and private gradients bit by bit."""
    from paper_2608_06690_gb300 import inputs as inp
    shape = LARGE[name] if name in LARGE else SHAPES[name][0]
    layer = pmpe.MoeLayer(shape, inp.make_weights(shape, 21, device="cuda"))
    h, other = (inp.make_hidden(shape, seed, device="cuda") for seed in (21, 22))
    pol = inp.policy_iid_mixed(shape.T, 23).cuda()
    dout = torch.randn((shape.T, shape.H), generator=torch.Generator().manual_seed(24)).to(torch.bfloat16).cuda()
    a, b = new_audit(shape), new_audit(shape)
    want, idx, w = own_route(shape, layer, h, pol, a)
    grads, _ = layer.backward(h, pol, dout)
    _, idx2, w2 = own_route(shape, layer, other, (pol != 1).to(torch.uint8))  # the other pool of most tokens
    assert not torch.equal(idx, idx2)
    got = layer.forward(h, pol, route=(idx, w), audit=b)
    g, dh, dw = layer.backward_routed(h, pol, dout)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(a, b)
    for n in ("d_gate", "d_up", "d_down"):
        assert torch.equal(g[n], grads[n]), n
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()
    # d_w: the picks' outputs along dout, from what the forward kept of them
    y = (got.double() * dout.double()).sum(1)
    if shape.E_sh == 0:  # out = sum_j w_j y_j: BF16 rows and output, 2^-8 each of the terms
        total, size = (dw.double() * w.double()).sum(1), (dw.double() * w.double()).abs().sum(1)
        scale = (got.double().abs() * dout.double().abs()).sum(1)
        assert ((total - y).abs() <= 2.0 ** -7 * (size + scale)).all()


def test_picks_that_cannot_be_taken():
    shape, layer, h, pol, _ = build("renorm")
    _, idx, w = own_route(shape, layer, h, pol)
    allow = (pol == 1).cpu()
    t_deny, t_allow = int(torch.nonzero(~allow)[0]), int(torch.nonzero(allow)[0])
    bad, clean, wc = idx.clone(), idx.clone(), w.clone()

    def lowest_free(row, base, n, used):
        return next(e for e in range(base, base + n) if e not in row and e not in used)

    edits = {t_deny: [(0, shape.E_pub), (2, 10 ** 9), (3, -2 ** 31)],   # a private expert for a DENY token, and no expert at all
             t_allow: [(1, 0), (3, -5)]}                 # a public one for an ALLOW token
    twice = int(torch.nonzero(~allow)[1])
    edits[twice] = [(1, int(idx[twice, 0]))]             # the same expert twice
    none = int(torch.nonzero(allow)[1])
    edits[none] = [(j, -1) for j in range(shape.k)]      # no expert: not an error by itself
    for t, row in edits.items():
        for j, e in row:
            bad[t, j] = e
        base, n = (shape.E_pub, shape.E_priv) if allow[t] else (0, shape.E_pub)
        kept = [int(v) for j, v in enumerate(idx[t]) if j not in [x for x, _ in row]]
        used = []
        for j, _ in row:
            used.append(lowest_free(kept, base, n, used))
            clean[t, j] = used[-1]
            wc[t, j] = 0.0
    a, b = new_audit(shape), new_audit(shape)
    got = layer.forward(h, pol, route=(bad, w), audit=a).clone()
    dout = torch.randn((shape.T, shape.H), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    g, dh, dw = layer.backward_routed(h, pol, dout)
    g = {n: v.clone() for n, v in g.items()}
    want = layer.forward(h, pol, route=(clean, wc), audit=b).clone()
    g2, dh2, dw2 = layer.backward_routed(h, pol, dout)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(dh, dh2)
    for n in g:
        assert torch.equal(g[n], g2[n]), n
    keep = (bad == clean)
    assert torch.equal(dw[keep], dw2[keep]) and (dw[~keep] == 0).all()
    x = pmpe.audit_read(a, shape.T, shape.E, check_status=False)
    y = pmpe.audit_read(b, shape.T, shape.E)
    assert x["status"] == pmpe.STATUS_BAD_EXPERT_ID and y["status"] == 0
    assert np.array_equal(x["exec_rows"], x["route_count"]) and np.array_equal(x["exec_rows"], y["exec_rows"])
    assert (x["exec_priv_rows"][~allow.numpy()] == 0).all()  # no private row ran for a DENY token
    only_none = idx.clone()
    only_none[none] = -1
    c = new_audit(shape)
    layer.forward(h, pol, route=(only_none, w), audit=c)
    assert pmpe.audit_read(c, shape.T, shape.E)["status"] == 0


def test_refusals_and_the_empty_batch():
    shape, layer, h, pol, _ = build("tile_edges")
    _, idx, w = own_route(shape, layer, h, pol)
    for bad in (dict(route=(idx.long(), w)), dict(route=(idx, w.half())), dict(route=(idx[:5], w)), dict(route=(idx.t(), w)),
                dict(route=(idx, w), topk_idx=idx), dict(route=(idx, w), unmasked_control=True),
                dict(route=(idx, w), stages=pmpe.STAGE_ROUTE)):
        with pytest.raises(pmpe.PmpeError):
            layer.forward(h, pol, **bad)
    dout = torch.zeros_like(h)
    with pytest.raises(pmpe.PmpeError):
        layer.backward_routed(h, pol, dout)  # the last forward ran the layer's own router
    layer.forward(h, pol, route=(idx, w))
    with pytest.raises(pmpe.PmpeError):
        layer.backward_routed(h[:5], pol[:5], dout[:5])  # another number of tokens than the forward's
    for back in (layer.backward, layer.backward_private, layer.backward_input):
        with pytest.raises(pmpe.PmpeError):
            back(h, pol, dout)
    e = torch.empty((0, shape.H), dtype=torch.bfloat16, device="cuda")
    out = layer.forward(e, pol[:0], route=(idx[:0].contiguous(), w[:0].contiguous()))
    g, dh, dw = layer.backward_routed(e, pol[:0], e)
    torch.cuda.synchronize()
    assert out.shape == (0, shape.H) and dh.shape == (0, shape.H) and dw.shape == (0, shape.k)
    assert all((v == 0).all() for v in g.values())


def test_tensors_that_are_not_the_layers_rows_are_refused():
    shape, layer, h, pol, _ = build("tile_edges")
    _, idx, w = own_route(shape, layer, h, pol)
    for bad in (dict(policy=pol.cpu()), dict(out=torch.empty_like(h, device="cpu")), dict(topk_idx=idx.cpu()), dict(audit=new_audit(shape).cpu()),
                dict(route=(idx.cpu(), w)), dict(route=(idx, w.cpu())), dict(hidden=h.cpu())):
        with pytest.raises(pmpe.PmpeError):
            layer.forward(**dict(dict(hidden=h, policy=pol), **bad))
    dout = torch.zeros_like(h)
    wide = torch.zeros((shape.T, 2 * shape.H), dtype=torch.bfloat16, device="cuda")
    bad = (h.float(), h[:, :128].contiguous(), wide[:, ::2], wide[:, :shape.H], h.cpu(), h[:5])
    layer.forward(h, pol)
    for back in (layer.backward, layer.backward_private, layer.backward_input):
        for x in bad[:-1]:
            with pytest.raises(pmpe.PmpeError):
                back(x, pol, dout)
    layer.forward(h, pol, route=(idx, w))
    for x in bad:
        with pytest.raises(pmpe.PmpeError):
            layer.backward_routed(x, pol, dout)


@pytest.mark.parametrize("given", [False, True])
def test_memory_freed_while_the_other_stream_has_yet_to_run(given):
    """Neither a call's arguments nor its results are handed out again before
    the stream that it was given is done with them, nor scratch that a larger
    call replaced."""
    shape, layer, h, pol, seed = build("large_experts_decode")
    want, idx, w = own_route(shape, layer, h, pol)
    dout = torch.randn((shape.T, shape.H), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
    route = dict(route=(idx, w)) if given else {}
    back = layer.backward_routed if given else layer.backward
    layer.forward(h, pol, **route)
    grads, dh = back(h, pol, dout)[:2]
    layer._bws = None  # a scratch of this call's own
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(40_000_000)  # some 20 ms
    a, b, c = h.clone(), pol.clone(), dout.clone()
    kept = torch.empty_like(a)
    torch.cuda.current_stream().synchronize()
    layer.forward(a, b, stream=s, **route)                # the result is dropped at once
    layer.forward(a, b, out=kept, stream=s, **route)
    got = back(a, b, c, stream=s)
    g, d = got[0]["d_gate"], got[1]
    layer._bws = None
    del a, b, c, got
    other = [torch.full_like(h, 7.0) for _ in range(6)] + [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(64)]
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(kept, want) and torch.equal(g, grads["d_gate"]) and torch.equal(d, dh)
    assert all((o == 7).all() for o in other)


# ------------------------------------------------------- the block together

def block(layer, router, x, res, wn, wr, bias, policy, dout, max_norm, load):
    """A training step of a wrapped model's block: forward, then back."""
    n = pmpe.rms_norm(x, wn, residual=res)
    logits = n.y.float() @ wr.T
    route = router.route(logits, policy, bias=bias, load=load)
    out = layer.forward(n.y, policy, route=route, save_for_backward=True)
    grads, dy, dw = layer.backward_routed(n.y, policy, dout)
    dz = router.backward(logits, policy, route[0], dw)
    grads["d_wr"] = dz.T @ n.y.float()
    dx, grads["d_norm"] = pmpe.rms_norm_backward(dy + dz @ wr, n.h, wn, n.rstd, d_h=dout.float(), dx_dtype=torch.float32)
    norm = pmpe.clip_grad_norm(grads, max_norm)
    return dict(out=out, h=n.h, y=n.y, logits=logits, idx=route[0], w=route[1], dx=dx, norm=norm, grads=grads)


def make_block(name, score, seed=3):
    shape, s, policy = SHAPES[name]
    wd, h, pol = to_device(*make_layer(shape, s, policy=policy))
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *size: torch.randn(size, generator=g).cuda()  # noqa: E731
    x, res = rnd(shape.T, shape.H).bfloat16(), rnd(shape.T, shape.H).bfloat16()
    wn, wr, bias = (1 + 0.1 * rnd(shape.H)).bfloat16(), 0.05 * rnd(shape.E, shape.H), 0.05 * rnd(shape.E)
    dout = rnd(shape.T, shape.H).bfloat16()
    router = pmpe.Router(shape.E_pub, shape.E_priv, shape.k, score=score, scale=1.5, groups=(4, 2) if shape.E_pub % 4 == 0 else (1, 1),
                         group_score="top2")
    layer = pmpe.MoeLayer(shape, wd)
    return shape, (layer, router, x, res, wn, wr, bias, pol, dout, 0.5, torch.zeros(shape.E, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("name", ["renorm", "pool_softmax_shared", "one_token"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_block_against_autograd_in_64_bits(name, score):
    """The whole block against torch.autograd in FP64 on the same selection.
    The layer's own bounds (outputs 1e-2 of the largest value and 5e-3 on
    average, gradients 2e-2 and 1e-2: BF16 activations) hold for what comes out
    of it; the other operators' errors are of the order 2^-17."""
    shape, args = make_block(name, score)
    layer, router, x, res, wn, wr, bias, pol, dout, max_norm, load = args
    r = block(*args)
    torch.cuda.synchronize()
    W = {n: (None if v is None else v.double()) for n, v in layer.weights.items()}
    leaves = {n: W[n].clone().requires_grad_() for n in ("gate_priv", "up_priv", "down_priv")}
    h = r["h"].double().requires_grad_()
    nw, rw = wn.double().requires_grad_(), wr.double().requires_grad_()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * nw
    y = y + (r["y"].double() - y).detach()  # the stored rows, with the exact ones' gradient
    z = y @ rw.T
    allow = torch.zeros(shape.T, dtype=torch.bool, device="cuda") if pol is None else pol == 1
    own = (torch.arange(shape.E, device="cuda") >= shape.E_pub)[None] == allow[:, None]
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(torch.where(own, z, -torch.inf), 1)
    idx = r["idx"].long()
    w = torch.gather(s, 1, idx)
    w = 1.5 * w / w.sum(1, keepdim=True)
    gate, up, down = (torch.cat([W[n + "_pub"], leaves[n + "_priv"]]) for n in ("gate", "up", "down"))
    silu = torch.nn.functional.silu
    out = torch.zeros_like(y)
    for e in range(shape.E):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        if t.numel():
            a = y[t]
            out = out.index_add(0, t, w[t, j][:, None] * ((silu(a @ gate[e].T) * (a @ up[e].T)) @ down[e].T))
    for e in range(shape.E_sh):
        out = out + (silu(y @ W["gate_sh"][e].T) * (y @ W["up_sh"][e].T)) @ W["down_sh"][e].T
    ((out + h) * dout.double()).sum().backward()

    def near(got, want, most, mean):
        err, size = (got.double() - want).abs(), want.abs()
        assert err.max() <= most * size.max() and err.sum() <= mean * size.sum(), (float(err.max() / size.max()), float(err.sum() / size.sum()))

    near(r["out"], out.detach(), 1e-2, 5e-3)
    near(r["w"], w.detach(), 1e-4, 1e-5)
    near(r["dx"], h.grad, 2e-2, 1e-2)
    want = {"d_gate": leaves["gate_priv"].grad, "d_up": leaves["up_priv"].grad, "d_down": leaves["down_priv"].grad, "d_wr": rw.grad,
            "d_norm": nw.grad}
    total = torch.stack([v.square().sum() for v in want.values()]).sum().sqrt()
    assert abs(float(r["norm"]) - float(total)) <= 1e-2 * float(total)
    f = min(1.0, max_norm / (float(total) + 1e-6))
    assert f < 1.0
    for n, v in want.items():
        if float(v.abs().max()) > 0:
            near(r["grads"][n], f * v, 3e-2, 2e-2)  # the norm's own 1e-2 on top
    assert int(load.sum()) == shape.T * shape.k


def test_block_captured_into_a_graph():
    """The block replayed with new inputs gives what the eager calls give,
    while eager results of the same tensors are alive."""
    shape, args = make_block("renorm", "sigmoid")
    eager = block(*args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):  # the library's workspaces are there before the capture
        block(*args)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = block(*args)
    g.replay()
    torch.cuda.synchronize()
    flat = lambda r: [r[n] for n in ("out", "h", "y", "idx", "w", "dx", "norm")] + [r["grads"][n] for n in sorted(r["grads"])]  # noqa: E731
    for a, b in zip(flat(held), flat(eager)):
        assert torch.equal(a, b)
    args[2].copy_(torch.randn(args[2].shape, generator=torch.Generator().manual_seed(9)).bfloat16())
    g.replay()
    torch.cuda.synchronize()
    again = block(*args)
    torch.cuda.synchronize()
    for a, b in zip(flat(held), flat(again)):
        assert torch.equal(a, b)
    assert not torch.equal(again["out"], eager["out"])
