"""The operators around the expert layer, as measurable cases: the norm of the
residual stream before it, the routing to its experts, and the clipping of the
gradients its backward gives.

Operators (``op``):
  norm       ``rms_norm``: the residual's addition, the root-mean-square norm,
             its output in the input's type or in 8 bits with scales
  norm_bwd   ``rms_norm_backward``: gradients of the input and of the weight
  route      ``Router.route``: scores, balance bias, groups, top-k, weights
  route_bwd  ``Router.backward``: gradient of the logits
  clip       ``clip_grad_norm``: the global norm of many gradients, and the
             clipped gradients

Sizes are those of the layers in ``configs`` (hidden sizes 256 and 2048, pools
of 128 + 32, 128 + 16, 64 + 16 and 16 + 4 experts, batches of 1 to 16384
tokens) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
BLOCK = 128          # columns that share a scale
E4M3_MAX = 448.0
FLT_MAX = 3.4028234663852886e38
FLT_MIN = 2.0 ** -126


def _norm(T, H, dtype, **more):
    return dict(dict(op="norm", T=T, H=H, dtype=dtype, wtype=dtype, ld=H, residual=True, quant="none"), **more)


def _norm_bwd(T, H, dtype, **more):
    return dict(dict(op="norm_bwd", T=T, H=H, dtype=dtype, wtype=dtype, gtype=dtype, xtype=dtype, d_res=True), **more)


def _route(T, E_pub, E_priv, k, **more):
    return dict(dict(op="route", T=T, E_pub=E_pub, E_priv=E_priv, k=k, dtype="fp32", score="softmax", bias=False,
                     renorm=True, scale=1.0, groups=1, top_groups=1, group_score="max", load=False, requests=min(T, 16),
                     allow=0.5 if E_priv else 0.0), **more)


def listed():
    return [
        # one user's decode step: the smallest call, all latency
        dict(_norm(1, 2048, "bf16"), name="norm_decode_t1"),
        # a prompt batch whose next projection takes 8-bit inputs, scales per 128 columns
        dict(_norm(4096, 2048, "bf16", quant="block"), name="norm_e4m3_t4096"),
        # ragged rows: an odd width inside a wider buffer, half precision, no residual
        dict(_norm(777, 1001, "fp16", residual=False, ld=1003), name="norm_odd_t777"),
        # the largest prompt batch of the 48-layer stack
        dict(_norm(16384, 2048, "bf16"), name="norm_prefill_t16384"),
        # training: the FP32 input gradient that the layer's backward gives, a residual gradient beside it
        dict(_norm_bwd(4096, 2048, "bf16", gtype="fp32"), name="norm_bwd_t4096"),
        # a decode batch of 64 users, alternating policies
        dict(_route(64, 128, 32, 8, requests=64), name="route_decode_t64"),
        # a large prompt batch of the same pools
        dict(_route(16384, 128, 32, 8, requests=64), name="route_prefill_t16384"),
        # sigmoid scores, a balance bias and group limits over 256 experts, loads counted for the bias's update
        dict(_route(8192, 256, 0, 8, dtype="bf16", score="sigmoid", bias=True, groups=8, top_groups=4,
                    group_score="top2", scale=2.5, load=True), name="route_groups_t8192"),
        # training: the logits' gradient of the pool softmax without renormalisation
        dict(_route(4096, 64, 16, 6, renorm=False, op="route_bwd", requests=11, allow=0.25), name="route_bwd_t4096"),
        # the tiny layer's private gradients: four small tensors
        dict(op="clip", kind="layer", layers=1, E_priv=4, H=256, I=128, dtype="fp32", name="clip_tiny"),
        # ten small layers' private gradients with ragged widths, in half precision
        dict(op="clip", kind="ragged", layers=10, E_priv=7, H=1000, I=333, dtype="bf16", name="clip_ragged_bf16"),
        # one wrapped layer's private gradients, 604 MB of FP32
        dict(op="clip", kind="layer", layers=1, E_priv=32, H=2048, I=768, dtype="fp32", name="clip_qwen3_layer"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm", "norm_bwd", "norm_bwd", "route", "route", "route", "route_bwd", "clip", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm", "norm_bwd"):
        H = rng.choice([256, 512, 1024, 2048, 2048, 4096, 5120, 7168, 8 * _log_int(rng, 4, 1024), _log_int(rng, 17, 8191)])
        T = _log_int(rng, 1, max(1, min(16384, 16384 * 2048 * 2 // (H * SIZE[dtype]))))
        wtype = rng.choice([dtype, dtype, "fp32"])
        if op == "norm":
            quant = rng.choice(["none", "none", "block", "row"])
            return _norm(T, H, dtype, wtype=wtype, residual=rng.random() < 0.7, quant=quant,
                         ld=H if rng.random() < 0.7 else H + rng.choice([1, 8, 64, 333]))
        T = max(1, T // 2)
        return _norm_bwd(T, H, dtype, wtype=wtype, gtype=rng.choice([dtype, "fp32"]), xtype=rng.choice([dtype, "fp32"]),
                         d_res=rng.random() < 0.7)
    if op in ("route", "route_bwd"):
        pools = rng.choice([(16, 4), (128, 32), (128, 16), (64, 16), (256, 0), (256, 32), (rng.randint(8, 256), 0),
                            (rng.randint(8, 256), rng.randint(8, 256))])
        k = rng.choice([1, 2, 4, 6, 8, 8, rng.randint(1, 12)])
        k = min([k, pools[0]] + ([pools[1]] if pools[1] else []))
        T = _log_int(rng, 1, 16384 * 160 // max(160, sum(pools)))
        groups = rng.choice([g for g in (1, 2, 4, 8, 16) if pools[0] % g == 0 and pools[0] // g >= 2])
        top_groups = rng.randint(1, groups)
        if top_groups * (pools[0] // groups) < k:
            groups = top_groups = 1
        # a single renormalised weight is constant: its gradient is nothing but rounding
        renorm = rng.random() < 0.6 and not (op == "route_bwd" and k == 1)
        return _route(T, pools[0], pools[1], k, op=op, dtype=dtype, score=rng.choice(["softmax", "sigmoid"]),
                      bias=rng.random() < 0.5, renorm=renorm, scale=rng.choice([1.0, 2.5]), groups=groups,
                      top_groups=top_groups, group_score=rng.choice(["max", "top2"]), load=rng.random() < 0.4,
                      requests=min(T, _log_int(rng, 1, 64)), allow=rng.choice([0.0, 0.25, 0.5, 1.0]) if pools[1] else 0.0)
    if rng.random() < 0.5:
        E, H, I = rng.randint(1, 16), 128 * rng.randint(1, 16), 128 * rng.randint(1, 6)
        return dict(op="clip", kind="layer", layers=min(rng.randint(1, 14), max(1, 140_000_000 // (3 * E * H * I))),
                    E_priv=E, H=H, I=I, dtype=dtype)
    return dict(op="clip", kind="ragged", layers=rng.randint(1, 14), E_priv=rng.randint(1, 9), H=_log_int(rng, 1, 1500),
                I=_log_int(rng, 1, 900), dtype=dtype)


# ------------------------------------------------------------------- inputs

def _gen(seed, n=0):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 131 + n)


def _randn(shape, seed, n, dtype="fp32"):
    return torch.randn(shape, generator=_gen(seed, n), device="cuda").to(DTYPES[dtype])


def _policy(case, seed):
    """Ragged contiguous requests, some of them ALLOW (byte 1)."""
    if not case["E_priv"]:
        return None
    g = torch.Generator().manual_seed(int(seed) + 71)
    T, n = case["T"], case["requests"]
    cuts = torch.sort(torch.randperm(T - 1, generator=g)[:n - 1] + 1).values if n > 1 else torch.zeros(0, dtype=torch.int64)
    edge = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([T])])
    byte = torch.zeros(n, dtype=torch.uint8)
    byte[torch.randperm(n, generator=g)[:int(round(case["allow"] * n))]] = 1
    return byte.repeat_interleave(edge[1:] - edge[:-1]).cuda()


def _grad_shapes(case):
    """The private gradients of each layer: router, gate, up, down; ragged: also
    a vector of each layer's width, and widths that differ from layer to layer."""
    E, H, I = case["E_priv"], case["H"], case["I"]
    shapes = []
    for l in range(case["layers"]):
        if case["kind"] == "layer":
            shapes += [(E, H), (E, I, H), (E, I, H), (E, H, I)]
        else:
            shapes += [(E, H + l), (E, I, H + l), (E, H + l, I), (H + l,)]
    return shapes


def _clip_inputs(case, seed):
    """Gradients whose scale differs from tensor to tensor, and a limit below their norm."""
    grads = [_randn(s, seed, i).mul_(1e-3 * (1 + i % 5)).to(DTYPES[case["dtype"]])
             for i, s in enumerate(_grad_shapes(case))]
    return grads, 0.25 * 1e-3 * math.sqrt(sum(g.numel() for g in grads))


def _inputs(case, seed):
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        T, H = case["T"], case["H"]
        st = {"weight": (1.0 + 0.1 * _randn((H,), seed, 1)).to(DTYPES[case["wtype"]])}
        if op == "norm":
            # a few columns of the residual stream are much larger than the others
            scale = torch.exp(0.5 * _randn((H,), seed, 2))
            wide = _randn((T, case["ld"]), seed, 3)
            wide[:, :H] *= scale
            st["x"] = wide.to(DTYPES[case["dtype"]])[:, :H]
            st["residual"] = (2 * scale * _randn((T, H), seed, 4)).to(DTYPES[case["dtype"]]) if case["residual"] else None
            return st
        st["h"] = (torch.exp(0.5 * _randn((H,), seed, 2)) * _randn((T, H), seed, 3)).to(DTYPES[case["dtype"]])
        st["rstd"] = torch.rsqrt(st["h"].double().square().mean(1) + EPS).float()
        st["dy"] = _randn((T, H), seed, 5, case["gtype"])
        st["d_res"] = _randn((T, H), seed, 6, case["xtype"]) if case["d_res"] else None
        return st
    if op in ("route", "route_bwd"):
        T, E = case["T"], case["E_pub"] + case["E_priv"]
        st = {"logits": (1.5 * _randn((T, E), seed, 1) + 0.5 * _randn((E,), seed, 2)).to(DTYPES[case["dtype"]]),
              "bias": 0.05 * _randn((E,), seed, 3) if case["bias"] else None, "policy": _policy(case, seed)}
        if op == "route_bwd":
            st["idx"] = _plain_route(case, st)["idx"]
            st["dw"] = _randn((T, case["k"]), seed, 4)
        return st
    grads, limit = _clip_inputs(case, seed)
    return {"grads": grads, "limit": limit}


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if case["op"] == "clip":
        st["out"] = [torch.empty_like(g) for g in st["grads"]]
    if own and case["op"] in ("route", "route_bwd"):
        from paper_2608_06690_gb300 import pmpe
        st["router"] = pmpe.Router(case["E_pub"], case["E_priv"], case["k"], score=case["score"], renormalize=case["renorm"],
                                   scale=case["scale"], groups=(case["groups"], case["top_groups"]),
                                   group_score=case["group_score"])
    return st


# -------------------------------------------------------------- plain forms

def _blocks(y, quant):
    """[T, blocks, columns of a block], the last block filled up with zeros."""
    T, H = y.shape
    width = BLOCK if quant == "block" else H
    n = -(-H // width)
    return torch.cat([y, y.new_zeros(T, n * width - H)], 1).view(T, n, width)


def _plain_norm(case, st):
    dt = st["x"].dtype
    h = st["x"].float()
    if st["residual"] is not None:
        h = (h + st["residual"].float()).to(dt)
    h64 = h.double()
    rstd = torch.rsqrt(h64.square().mean(1) + EPS)
    y = h64 * rstd[:, None] * st["weight"].double()
    out = {"h": h if st["residual"] is not None else None, "rstd": rstd.float()}
    if case["quant"] == "none":
        return dict(out, y=y.to(dt), scale=None)
    b = _blocks(y, case["quant"])
    scale = (b.abs().amax(2) / E4M3_MAX).clamp(min=FLT_MIN).float()
    q = (b / scale.double()[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).flatten(1)[:, :case["H"]]
    return dict(out, y=q.float().to(torch.float8_e4m3fn), scale=scale)


def _plain_norm_bwd(case, st):
    h, dy, r = st["h"].float(), st["dy"].float(), st["rstd"][:, None]
    g = dy * st["weight"].float()
    dx = r * g - h * (r * r * r * ((g * h).double().mean(1, keepdim=True)).float())
    if st["d_res"] is not None:
        dx = dx + st["d_res"].float()
    return {"dx": dx.to(DTYPES[case["xtype"]]), "dw": (dy * h * r).double().sum(0).float()}


def _keep_groups(case, choice, score):
    """Whether each public expert lies in one of its token's best groups."""
    T, E = choice.shape
    n, size = case["groups"], E // case["groups"]
    if case["top_groups"] == n:
        return torch.ones_like(choice, dtype=torch.bool)
    if case["group_score"] == "max":
        g = choice.view(T, n, size).amax(2)
    else:
        two = torch.sort(score.view(T, n, size), dim=2, descending=True).values[:, :, :2]
        g = torch.where(two[:, :, 0] > -math.inf, two[:, :, 0] + torch.where(two[:, :, 1] > -math.inf, two[:, :, 1], 0.0), -math.inf)
    place = torch.sort(torch.sort(g, dim=1, descending=True, stable=True).indices, dim=1).indices
    return (place < case["top_groups"]).repeat_interleave(size, 1)


def _plain_scores(case, st):
    z = st["logits"].double()
    T, E = z.shape
    allow = torch.zeros(T, dtype=torch.bool, device=z.device) if st["policy"] is None else st["policy"] == 1
    eligible = ((torch.arange(E, device=z.device) >= case["E_pub"])[None, :] == allow[:, None]) & (z > -math.inf)
    z = torch.where(eligible, z.clamp(max=FLT_MAX), -math.inf)
    if case["score"] == "sigmoid":
        return z, eligible, 1.0 / (1.0 + torch.exp(-z))
    top = z.amax(1, keepdim=True)
    e = torch.where(eligible, torch.exp(z - torch.where(top > -math.inf, top, 0.0)), 0.0)
    return z, eligible, e / e.sum(1, keepdim=True).clamp(min=1e-300)


def _plain_weights(case, score, idx):
    w = torch.where(idx >= 0, torch.gather(score, 1, idx.long().clamp(min=0)), 0.0)
    if case["renorm"]:
        w = w / (w.sum(1, keepdim=True) + 1e-20)
    return w * case["scale"]


def _plain_route(case, st):
    z, eligible, score = _plain_scores(case, st)
    value = torch.where(eligible, score + (st["bias"].double() if st["bias"] is not None else 0.0), -math.inf)
    choice = value if st["bias"] is not None else z
    keep = torch.ones_like(eligible)
    keep[:, :case["E_pub"]] = _keep_groups(case, choice[:, :case["E_pub"]], value[:, :case["E_pub"]])
    choice, sel = torch.sort(torch.where(keep, choice, -math.inf), dim=1, descending=True, stable=True)
    idx = torch.where(choice > -math.inf, sel, -1)[:, :case["k"]].to(torch.int32)
    out = {"idx": idx, "w": _plain_weights(case, score, idx).float()}
    if case["load"]:
        E = case["E_pub"] + case["E_priv"]
        out["load"] = torch.zeros(E + 1, dtype=torch.int32, device=idx.device).index_add_(
            0, idx.flatten().long() % (E + 1), torch.ones_like(idx).flatten())[:E].contiguous()
    return out


def _plain_route_bwd(case, st):
    z, _, score = _plain_scores(case, st)
    idx, live = st["idx"].long().clamp(min=0), st["idx"] >= 0
    dw = torch.where(live, st["dw"].double() * case["scale"], 0.0)
    s = torch.where(live, torch.gather(score, 1, idx), 0.0)
    if case["renorm"]:
        total = s.sum(1, keepdim=True) + 1e-20
        ds = (dw - (dw * s).sum(1, keepdim=True) / total) / total
    else:
        ds = dw
    d = torch.zeros_like(z).scatter_add_(1, idx, torch.where(live, ds, 0.0))
    if case["score"] == "sigmoid":
        dz = d * score * (1.0 - score)
    else:
        dz = score * (d - (d * score).sum(1, keepdim=True))
    return {"d_logits": dz.to(st["logits"].dtype)}


def _plain_clip(case, st):
    norm = torch.sqrt(torch.stack([g.double().square().sum() for g in st["grads"]]).sum())
    factor = torch.clamp(st["limit"] / (norm + 1e-6), max=1.0).float()
    return {"norm": norm.float(), "grads": [torch.mul(g.float(), factor).to(g.dtype) for g in st["grads"]]}


PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "route": _plain_route, "route_bwd": _plain_route_bwd,
         "clip": _plain_clip}


def run(st):
    case = st["case"]
    if not own:
        return PLAIN[case["op"]](case, st)
    from paper_2608_06690_gb300 import pmpe
    if case["op"] == "norm":
        n = pmpe.rms_norm(st["x"], st["weight"], residual=st["residual"], eps=EPS,
                          quant=None if case["quant"] == "none" else case["quant"])
        return {"y": n.y, "scale": n.scale, "h": n.h if case["residual"] else None, "rstd": n.rstd}
    if case["op"] == "norm_bwd":
        dx, dw = pmpe.rms_norm_backward(st["dy"], st["h"], st["weight"], st["rstd"], d_h=st["d_res"],
                                        dx_dtype=DTYPES[case["xtype"]])
        return {"dx": dx, "dw": dw}
    if case["op"] == "route":
        load = torch.zeros(case["E_pub"] + case["E_priv"], dtype=torch.int32, device="cuda") if case["load"] else None
        idx, w = st["router"].route(st["logits"], st["policy"], bias=st["bias"], load=load)
        return {"idx": idx, "w": w, "load": load} if case["load"] else {"idx": idx, "w": w}
    if case["op"] == "route_bwd":
        return {"d_logits": st["router"].backward(st["logits"], st["policy"], st["idx"], st["dw"])}
    norm = pmpe.clip_grad_norm(st["grads"], st["limit"], out=st["out"])
    return {"norm": norm, "grads": st["out"]}


# --------------------------------------------------------------------- work

def work(case):
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        n, e, T, H = case["T"] * case["H"], SIZE[case["dtype"]], case["T"], case["H"]
        if op == "norm":
            b = n * e * (3 if case["residual"] else 1) + H * SIZE[case["wtype"]] + 4 * T
            if case["quant"] == "none":
                b += n * e
            else:
                b += n + 4 * T * (-(-H // BLOCK) if case["quant"] == "block" else 1)
            return {"bytes": float(b), "flops": 5.0 * n}
        b = n * (e + SIZE[case["gtype"]] + SIZE[case["xtype"]] * (2 if case["d_res"] else 1)) + H * (SIZE[case["wtype"]] + 4) + 4 * T
        return {"bytes": float(b), "flops": 9.0 * n}
    if op in ("route", "route_bwd"):
        T, k, E = case["T"], case["k"], case["E_pub"] + case["E_priv"]
        allow = int(round(case["allow"] * case["requests"])) / case["requests"]
        seen = T * ((1 - allow) * case["E_pub"] + allow * case["E_priv"])  # logits of the tokens' own pools
        if op == "route":
            b = seen * SIZE[case["dtype"]] + 8 * T * k + (T if case["E_priv"] else 0) + (4 * E if case["bias"] else 0) + (4 * E if case["load"] else 0)
            return {"bytes": float(b), "flops": 4.0 * seen}
        if case["renorm"] or case["score"] == "sigmoid":
            seen = T * k  # only the chosen experts' logits have a gradient
        b = seen * SIZE[case["dtype"]] + 8 * T * k + T * E * SIZE[case["dtype"]] + (T if case["E_priv"] else 0)
        return {"bytes": float(b), "flops": 6.0 * seen}
    n = sum(math.prod(s) for s in _grad_shapes(case))
    return {"bytes": float(2 * n * SIZE[case["dtype"]] + 4), "flops": 3.0 * n}


# ------------------------------------------------------------ the same in 64 bits

def _e4m3(v):
    """v rounded to the nearest e4m3 value (ties to even mantissas), in 64 bits."""
    _, ex = torch.frexp(v)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def _exact_norm(case, st):
    dt, H = st["x"].dtype, case["H"]
    h = st["x"].double()
    if st["residual"] is not None:
        h = (h + st["residual"].double()).to(dt).double()
    ms = torch.einsum("th,th->t", h, h) / H
    y = torch.einsum("th,t,h->th", h, 1.0 / torch.sqrt(ms + EPS), st["weight"].double())
    out = {"h": h if st["residual"] is not None else None, "rstd": 1.0 / torch.sqrt(ms + EPS), "y": y, "scale": None}
    if case["quant"] != "none":
        parts = y.split(BLOCK if case["quant"] == "block" else H, dim=1)
        s = [torch.maximum(p.abs().max(1, keepdim=True).values / E4M3_MAX, torch.full((), FLT_MIN, dtype=torch.float64, device=p.device)) for p in parts]
        out["y"] = torch.cat([_e4m3((p / c).clamp(-E4M3_MAX, E4M3_MAX)) for p, c in zip(parts, s)], 1)
        out["scale"] = torch.cat(s, 1)
    return out


def _exact_norm_bwd(case, st):
    h, dy, w, r = st["h"].double(), st["dy"].double(), st["weight"].double(), st["rstd"].double()
    n = h * r[:, None]  # the normed rows
    g = dy * w
    dx = r[:, None] * (g - n * (torch.einsum("th,th->t", g, n) / case["H"])[:, None])
    if st["d_res"] is not None:
        dx = dx + st["d_res"].double()
    return {"dx": dx, "dw": torch.einsum("th,th->h", dy, n)}


def _exact_weights(case, z, idx):
    """Weights of the chosen experts from one pool's logits (rows of z), as a
    differentiable function of them."""
    if case["score"] == "sigmoid":
        s = torch.sigmoid(torch.gather(z, 1, idx))
        return case["scale"] * (s / s.sum(1, keepdim=True) if case["renorm"] else s)
    log_p = torch.log_softmax(z, 1)
    p = torch.gather(log_p, 1, idx)
    return case["scale"] * torch.exp(p - torch.logsumexp(p, 1, keepdim=True) if case["renorm"] else p)


def _exact_route(case, st):
    """Each pool's tokens by themselves: the experts in order of choice, one after another."""
    w = torch.empty((case["T"], case["k"]), dtype=torch.float64, device="cuda")
    for lo, hi, allow in ((0, case["E_pub"], 0), (case["E_pub"], case["E_pub"] + case["E_priv"], 1)):
        toks = torch.arange(case["T"], device="cuda") if st["policy"] is None else torch.nonzero(st["policy"] == allow).flatten()
        if hi == lo or toks.numel() == 0:
            continue
        z = st["logits"].double()[toks, lo:hi]
        v = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, 1)
        if st["bias"] is not None:
            v = v + st["bias"].double()[lo:hi]
        left = v if st["bias"] is not None else z
        if allow == 0 and case["top_groups"] < case["groups"]:
            per = (left if case["group_score"] == "max" else v).unflatten(1, (case["groups"], -1))
            first, at = per.max(2)
            second = per.scatter(2, at[:, :, None], -math.inf).amax(2)
            rest = first if case["group_score"] == "max" else first + second
            keep = torch.zeros_like(rest, dtype=torch.bool)
            for _ in range(case["top_groups"]):
                g = rest.argmax(1, keepdim=True)
                keep.scatter_(1, g, True)
                rest = rest.scatter(1, g, -math.inf)
            left = torch.where(keep.repeat_interleave(per.shape[2], 1), left, -math.inf)
        picks = []
        for _ in range(case["k"]):
            picks.append(left.argmax(1, keepdim=True))
            left = left.scatter(1, picks[-1], -math.inf)
        w[toks] = _exact_weights(case, z, torch.cat(picks, 1))
    return {"idx": None, "w": w, "load": None} if case["load"] else {"idx": None, "w": w}


def _exact_route_bwd(case, st):
    """By differentiating the weights themselves."""
    d = torch.zeros(st["logits"].shape, dtype=torch.float64, device="cuda")
    for lo, hi, allow in ((0, case["E_pub"], 0), (case["E_pub"], case["E_pub"] + case["E_priv"], 1)):
        toks = torch.arange(case["T"], device="cuda") if st["policy"] is None else torch.nonzero(st["policy"] == allow).flatten()
        if hi == lo or toks.numel() == 0:
            continue
        z = st["logits"].double()[toks, lo:hi].requires_grad_()
        w = _exact_weights(case, z, st["idx"][toks].long() - lo)
        d[toks, lo:hi] = torch.autograd.grad((w * st["dw"][toks].double()).sum(), z)[0]
    return {"d_logits": d}


def _exact_clip(case, st):
    total = sum(torch.linalg.vector_norm(g.double()).item() ** 2 for g in st["grads"])
    norm = math.sqrt(total)
    return {"norm": torch.tensor(norm, dtype=torch.float64),
            "grads": [g.double() * min(1.0, st["limit"] / (norm + 1e-6)) for g in st["grads"]]}


EXACT = {"norm": _exact_norm, "norm_bwd": _exact_norm_bwd, "route": _exact_route, "route_bwd": _exact_route_bwd,
         "clip": _exact_clip}


def exact(case, seed):
    return EXACT[case["op"]](case, _inputs(case, seed))
