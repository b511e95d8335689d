"""The operators of a decoding loop around the expert layer, as measurable
cases: the paged key-value cache, the attention that reads it, and the choice of
the next token.

Operators (``op``):
  append  ``KvCache.append``: new keys and values into the pages of their
          sequences, in the cache's type or in e4m3 with a scale per token and head
  read    ``KvCache.read``: cached positions back as rows in order
  attend  ``KvCache.attend``: one new token of each sequence over its cache
  sample  ``sample``: temperature, top-k, top-p and min-p from given random numbers

Sizes are generic (heads of 64 to 256 columns, pages of 1 to 256 positions, up
to 131072 positions and 131072 tokens of vocabulary) and those of the layers'
batches in ``configs`` (64 to 16384 tokens).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
E4M3_MAX = 448.0
FLT_MAX = 3.4028234663852886e38
FLT_MIN = 2.0 ** -126
LEAST = 2.0 ** -40      # of the best token's probability: what is below is not drawn


def _append(B, n_lo, n_hi, kv_heads, head_dim, page, cache, **more):
    """B sequences with n_lo to n_hi new tokens each; the longest has `before` positions already."""
    return dict(dict(op="append", B=B, n_lo=n_lo, n_hi=n_hi, before=100, kv_heads=kv_heads, head_dim=head_dim, page=page, cache=cache,
                     dtype="bf16" if cache == "e4m3" else cache, fused=True, pad=0), **more)


def _read(B, n_lo, n_hi, kv_heads, head_dim, page, cache, **more):
    return dict(dict(op="read", B=B, n_lo=n_lo, n_hi=n_hi, before=0, kv_heads=kv_heads, head_dim=head_dim, page=page, cache=cache,
                     dtype="bf16" if cache == "e4m3" else cache), **more)


def _attend(B, len_lo, len_hi, heads, kv_heads, head_dim, page, cache, **more):
    return dict(dict(op="attend", B=B, len_lo=len_lo, len_hi=len_hi, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                     cache=cache, dtype="bf16" if cache == "e4m3" else cache, window=0), **more)


def _sample(T, V, dtype, **more):
    return dict(dict(op="sample", T=T, V=V, dtype=dtype, ld=V, spread=2.5, rows="same", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **more)


def listed():
    return [
        # a decode batch of 64 users: one token each, all latency
        dict(_append(64, 1, 1, 4, 128, 16, "bf16", before=500), name="append_decode_b64"),
        # a large prompt batch of ragged prompts into an 8-bit cache, keys and values inside fused projection rows
        dict(_append(16, 60, 1988, 4, 128, 64, "e4m3"), name="append_prompt_e4m3"),
        # prefixes of eight sequences out of an 8-bit cache, for a prompt that continues them
        dict(_read(8, 1000, 15384, 4, 128, 64, "e4m3"), name="read_prefix_e4m3"),
        # a few short sequences with heads and pages of odd sizes
        dict(_read(5, 1, 399, 3, 80, 24, "fp16", before=77), name="read_odd_fp16"),
        # one user's decode step over a short conversation: the smallest attention, all latency
        dict(_attend(1, 1000, 1000, 32, 4, 128, 16, "bf16"), name="attend_b1"),
        # a decode batch of 64 users of very different lengths, one slot of the batch empty
        dict(_attend(64, 0, 8192, 32, 4, 128, 16, "bf16"), name="attend_ragged_b64"),
        # the same batch over an 8-bit cache
        dict(_attend(64, 0, 8192, 32, 4, 128, 64, "e4m3"), name="attend_ragged_e4m3_b64"),
        # one user's long document: few rows, a long axis
        dict(_attend(1, 131072, 131072, 32, 4, 128, 64, "bf16"), name="attend_long_b1"),
        # half precision, heads and pages of odd sizes, three queries a key, only the last 500 positions seen
        dict(_attend(19, 1, 2500, 15, 5, 80, 24, "fp16", window=500), name="attend_odd_window"),
        # one user's next token with the usual settings
        dict(_sample(1, 131072, "fp32", temperature=0.7, top_k=50, top_p=0.95), name="sample_b1"),
        # a decode batch of 64 users, each with settings of their own, some of them greedy
        dict(_sample(64, 131072, "fp32", rows="own"), name="sample_users_b64"),
        # rollouts for training: many rows of a small odd vocabulary in half precision, flat, hardly filtered
        dict(_sample(400, 32003, "bf16", spread=1.2, min_p=0.01), name="sample_rollout_t400"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "attend", "attend", "attend", "sample", "sample"])
    if op == "sample":
        V = rng.choice([32000, 65536, 131072, _log_int(rng, 50, 131072), _log_int(rng, 50, 131072)])
        T = _log_int(rng, 1, max(1, min(1024, 64 * 131072 // V)))
        return _sample(T, V, rng.choice(["fp32", "bf16", "fp16"]), ld=V if rng.random() < 0.7 else V + rng.choice([1, 8, 61]),
                       spread=rng.choice([0.3, 1.2, 2.5, 4.0]), rows=rng.choice(["same", "same", "own"]), temperature=rng.choice([0.3, 0.7, 1.0, 1.5]),
                       top_k=rng.choice([0, 0, 1, 20, 50, rng.randint(2, 3000)]), top_p=rng.choice([1.0, 0.5, 0.9, 0.95]),
                       min_p=rng.choice([0.0, 0.0, 0.02, 0.1]))
    cache = rng.choice(["bf16", "fp16", "e4m3", "e4m3"])
    dtype = rng.choice(["bf16", "fp16"]) if cache == "e4m3" else cache
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 16])
    head_dim = rng.choice([64, 80, 96, 128, 128, 192, 256, 16 * rng.randint(1, 16)])
    page = rng.choice([1, 8, 16, 24, 32, 64, 100, 128, 256])
    row = kv_heads * head_dim
    if op in ("append", "read"):
        B = _log_int(rng, 1, 128)
        most = 16384 * 512 if op == "append" else 65536 * 512  # values of a key
        n_hi = _log_int(rng, 1, max(1, most // (row * B)))
        n_lo = int(n_hi * rng.choice([0, 0.1, 0.5, 1.0]))
        if op == "append":
            return _append(B, n_lo, n_hi, kv_heads, head_dim, page, cache, dtype=rng.choice([dtype, "fp32"]), before=rng.choice([0, 5, 300]),
                           fused=rng.random() < 0.7, pad=rng.choice([0, 0, 3, 40]))
        return _read(B, n_lo, n_hi, kv_heads, head_dim, page, cache, dtype=rng.choice([dtype, "fp32"]), before=rng.choice([0, 5, 300]))
    B = _log_int(rng, 1, 256)
    group = rng.choice([1, 2, 3, 4, 7, 8, 8, 16, rng.randint(1, 24)])
    len_hi = _log_int(rng, 1, max(1, min(131072, 64 * 8192 * 512 // (row * B))))
    # many queries a key cost operations
    while len_hi > 1 and B * len_hi * group * row > 64 * 8192 * 512 * 8:
        len_hi //= 2
    return _attend(B, int(len_hi * rng.choice([0, 0.1, 0.5, 1.0])), len_hi, group * kv_heads, kv_heads, head_dim, page, cache, dtype=dtype,
                   window=rng.choice([0, 0, 0, rng.randint(1, 4096)]))


# ------------------------------------------------------------------- inputs

def _gen(seed, n=0):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 131 + n)


def _randn(shape, seed, n, dtype="fp32"):
    return torch.randn(shape, generator=_gen(seed, n), device="cuda").to(DTYPES[dtype])


def _spread(B, lo, hi):
    """B whole numbers from lo to hi in even steps (the same for every seed); hi alone for one."""
    return [hi] if B == 1 else [lo + (hi - lo) * i // (B - 1) for i in range(B)]


def _shuffled(values, seed, n):
    g = torch.Generator().manual_seed(int(seed) * 131 + n)
    return torch.tensor(values, dtype=torch.int64)[torch.randperm(len(values), generator=g)]


def _news(case):
    return _spread(case["B"], case["n_lo"], case["n_hi"])


def _lengths(case):
    if case["op"] == "attend":
        return _spread(case["B"], case["len_lo"], case["len_hi"])
    return None


def _plan(case, seed, lengths):
    """Page tables of sequences of these lengths: every page of the pool is
    somewhere, in random order; what a sequence does not need holds -1."""
    B, page = case["B"], case["page"]
    need = (lengths + page - 1) // page
    width, total = max(1, int(need.max())), int(need.sum())
    pages = total + 3
    order = torch.randperm(pages, generator=_gen(seed, 21), device="cuda").to(torch.int32)
    need = need.cuda()
    first = torch.cumsum(need, 0) - need
    j = torch.arange(width, device="cuda")[None, :]
    table = torch.where(j < need[:, None], order[(first[:, None] + j).clamp(max=pages - 1)], -1).to(torch.int32)
    return {"table": table.contiguous(), "lengths": lengths.to(torch.int32).cuda(), "pages": pages}


def _quantised(x):
    """(e4m3 values, FP32 scales) of the last axis: the largest value becomes 448."""
    x = x.double()
    s = (x.abs().amax(-1) / E4M3_MAX).clamp(min=FLT_MIN)
    return (x / s[..., None]).clamp(-E4M3_MAX, E4M3_MAX).float().to(torch.float8_e4m3fn), s.float()


def _pools(case, pages, seed):
    """Pages as earlier steps left them."""
    shape = (pages, case["kv_heads"], case["page"], case["head_dim"])
    st = {}
    for name, n in (("k", 11), ("v", 12)):
        st[name + "_scale"] = None
        if case["cache"] != "e4m3":
            st[name] = _randn(shape, seed, n, case["cache"])
            continue
        # tokens differ in size; quantised a slice at a time (64-bit temporaries)
        x = _randn(shape, seed, n)
        x *= torch.exp(0.4 * _randn(shape[:3] + (1,), seed, n + 5))
        done = [_quantised(part) for part in x.split(max(1, (1 << 26) // max(1, x[0].numel())))]
        st[name], st[name + "_scale"] = torch.cat([d[0] for d in done]), torch.cat([d[1] for d in done])
    return st


def _inputs(case, seed):
    op = case["op"]
    if op == "sample":
        T, V = case["T"], case["V"]
        st = {"logits": (case["spread"] * _randn((T, case["ld"]), seed, 1)).to(DTYPES[case["dtype"]])[:, :V],
              "u": torch.rand((T,), generator=_gen(seed, 2), device="cuda")}
        if case["rows"] == "same":
            return dict(st, **{n: case[n] for n in ("temperature", "top_k", "top_p", "min_p")})
        i = _shuffled(list(range(T)), seed, 3).cuda()  # each combination for the same share of users
        of = lambda values, step, dt: torch.tensor(values, device="cuda", dtype=dt)[(i // step) % len(values)]  # noqa: E731
        return dict(st, temperature=of([0.0, 0.6, 0.8, 1.0], 1, torch.float32), top_k=of([0, 20, 50, 1000], 4, torch.int32),
                    top_p=of([1.0, 0.9, 0.95], 2, torch.float32), min_p=of([0.0, 0.0, 0.05], 3, torch.float32))
    if op == "attend":
        st = _plan(case, seed, _shuffled(_lengths(case), seed, 4))
        st.update(_pools(case, st["pages"], seed))
        # queries inside fused projection rows, large enough that some positions stand out
        wide = (case["heads"] + 2 * case["kv_heads"]) * case["head_dim"]
        rows = (1.5 * _randn((case["B"], wide), seed, 5)).to(DTYPES[case["dtype"]])
        st["q"] = rows[:, :case["heads"] * case["head_dim"]].view(case["B"], case["heads"], case["head_dim"])
        return st
    # (the same pairs of old and new positions for every seed, so that the pool's size is)
    new, before = torch.tensor(_news(case)), _shuffled(_spread(case["B"], 0, case["before"]), 0, 7)
    order = _shuffled(list(range(case["B"])), seed, 6)
    new, before = new[order], before[order]
    st = _plan(case, seed, before + new)
    st.update(_pools(case, st["pages"], seed))
    st["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(new, 0)]).to(torch.int32).cuda()
    st["rows"] = int(new.sum())
    if op == "append":
        T, n, heads = st["rows"] + case["pad"], case["kv_heads"] * case["head_dim"], 4 * case["kv_heads"] if case["fused"] else 0
        wide = _randn((T, heads * case["head_dim"] + 2 * n), seed, 8)
        wide = (wide * torch.exp(0.4 * _randn((T, 1), seed, 9))).to(DTYPES[case["dtype"]])
        st["new_k"] = wide[:, heads * case["head_dim"]:][:, :n].view(T, case["kv_heads"], case["head_dim"])
        st["new_v"] = wide[:, heads * case["head_dim"]:][:, n:].view(T, case["kv_heads"], case["head_dim"])
        if case["n_lo"] == case["n_hi"] == 1 and not case["pad"]:
            st["cu"] = None  # a decode step: row b is sequence b's
    return st


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if own and case["op"] != "sample":
        from paper_2608_06690_gb300 import pmpe
        st["cache"] = pmpe.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
    return st


# -------------------------------------------------------------- plain forms

def _row_slots(st, rows):
    """(slot, real): the cache slot (page * page_size + place) of each row, and whether it has one."""
    table, lengths, page = st["table"].long(), st["lengths"].long(), st["case"]["page"]
    cu = st["cu"].long() if st["cu"] is not None else torch.arange(lengths.numel() + 1, device="cuda")
    r = torch.arange(rows, device="cuda")
    b = (r[:, None] >= cu[None, 1:]).sum(1)
    real = b < lengths.numel()
    b = b.clamp(max=lengths.numel() - 1)
    pos = lengths[b] - cu[b + 1] + r
    real = real & (pos >= 0) & (pos < lengths[b])
    pos = torch.where(real, pos, 0)
    return table[b, pos // page] * page + pos % page, real


def _token_major(pool):
    """[pages, heads, page, ...] as [pages, page, heads, ...]: a view whose first two axes are a slot's."""
    return pool.transpose(1, 2)


def _plain_append(case, st):
    rows = st["new_k"].shape[0]
    slot, real = _row_slots(st, rows)
    slot, page = slot[real], case["page"]
    for name in ("k", "v"):
        x = st["new_" + name][real]
        if case["cache"] == "e4m3":
            q, s = _quantised(x)
            _token_major(st[name]).view(torch.uint8)[slot // page, slot % page] = q.view(torch.uint8)
            _token_major(st[name + "_scale"])[slot // page, slot % page] = s
        else:
            _token_major(st[name])[slot // page, slot % page] = x.float().to(DTYPES[case["cache"]])
    return _state(case, st)


def _state(case, st):
    names = ("k", "v", "k_scale", "v_scale") if case["cache"] == "e4m3" else ("k", "v")
    return {n: st[n] for n in names}


def _values(case, st, name, page, place):
    """The cached values [..., heads, head_dim] of slots, in 32 bits."""
    x = _token_major(st[name])
    if case["cache"] != "e4m3":
        return x[page, place].float()
    return x.view(torch.uint8)[page, place].view(torch.float8_e4m3fn).float() * _token_major(st[name + "_scale"])[page, place][..., None]


def _plain_read(case, st):
    slot, real = _row_slots(st, st["rows"])
    page, place = slot // case["page"], slot % case["page"]
    return {n: torch.where(real[:, None, None], _values(case, st, n, page, place), 0.0).to(DTYPES[case["dtype"]]) for n in ("k", "v")}


def _plain_attend(case, st):
    B, G = case["B"], case["heads"] // case["kv_heads"]
    lengths, width = st["lengths"].long(), max(1, case["len_hi"])
    pos = torch.arange(width, device="cuda")[None, :]
    live = pos < lengths[:, None]
    if case["window"]:
        live = live & (pos >= lengths[:, None] - case["window"])
    page = torch.gather(st["table"].long().clamp(min=0), 1, (pos // case["page"]).expand(B, width))
    place = (pos % case["page"]).expand(B, width)
    k, v = (_values(case, st, n, page, place).transpose(1, 2) for n in ("k", "v"))  # [B, kv_heads, width, head_dim]
    q = st["q"].float().view(B, case["kv_heads"], G, case["head_dim"])
    s = torch.matmul(q, k.transpose(2, 3)) * case["head_dim"] ** -0.5
    s = torch.where(live[:, None, None, :], s, -math.inf)
    top = s.amax(3, keepdim=True)
    e = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(3, keepdim=True)
    out = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return {"out": out.view(B, case["heads"], case["head_dim"]).to(DTYPES[case["dtype"]]), "lse": lse.view(B, case["heads"])}


def _column(v, T, dtype):
    """One setting a row, [T, 1]."""
    return v.to(dtype)[:, None] if torch.is_tensor(v) else torch.full((T, 1), v, dtype=dtype, device="cuda")


def _plain_sample(case, st):
    T, V = case["T"], case["V"]
    # settings are 32-bit numbers; sums and what lies next to a border are in 64 bits
    temperature, top_p, min_p = (_column(st[n], T, torch.float32).double() for n in ("temperature", "top_p", "min_p"))
    top_k = _column(st["top_k"], T, torch.int64)
    z = st["logits"].double()
    z, sel = torch.sort(torch.where(z > -math.inf, z.clamp(max=FLT_MAX), -math.inf), dim=1, descending=True, stable=True)
    greedy = temperature <= 0
    d = torch.where(z > -math.inf, z - z[:, :1].clamp(min=-FLT_MAX), -math.inf)
    ratio = torch.where(greedy, (d == 0).double(), torch.exp(d / torch.where(greedy, 1.0, temperature)))  # to the best
    place = torch.arange(V, device="cuda")[None, :]
    keep = (ratio >= LEAST) & (place < torch.where(greedy, 1, torch.where(top_k > 0, top_k, V)))
    w = torch.where(keep, ratio, 0.0)
    below = torch.cumsum(w, 1) - w
    keep = keep & ((below < top_p * w.sum(1, keepdim=True)) | (top_p >= 1) | (place == 0)) & (ratio >= min_p)
    w = torch.zeros_like(w).scatter_(1, sel, torch.where(keep, ratio, 0.0))  # by id
    total = torch.cumsum(w, 1)
    target = st["u"].double()[:, None] * total[:, -1:]
    token = ((total > target) & (w > 0)).to(torch.int8).argmax(1)
    mass = total[:, -1]
    prob = torch.gather(w, 1, token[:, None])[:, 0] / torch.where(mass > 0, mass, 1.0)
    return {"token": torch.where(mass > 0, token, -1).to(torch.int32), "prob": prob.float()}


PLAIN = {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "sample": _plain_sample}


def run(st):
    case = st["case"]
    if not own:
        return PLAIN[case["op"]](case, st)
    if case["op"] == "sample":
        from paper_2608_06690_gb300 import pmpe
        s = pmpe.sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
        return {"token": s.token, "prob": s.prob}
    cache = st["cache"]
    if case["op"] == "append":
        cache.append(st["new_k"], st["new_v"], st["table"], st["lengths"], cu_seqlens=st["cu"])
        return _state(case, st)
    if case["op"] == "read":
        k, v = cache.read(st["table"], st["lengths"], cu_seqlens=st["cu"], rows=st["rows"], dtype=DTYPES[case["dtype"]])
        return {"k": k, "v": v}
    a = cache.attend(st["q"], st["table"], st["lengths"], window=case["window"])
    return {"out": a.out, "lse": a.lse}


# --------------------------------------------------------------------- work

def work(case):
    if case["op"] == "sample":
        n = case["T"] * case["V"]
        return {"bytes": float(n * SIZE[case["dtype"]] + case["T"] * (12 + (16 if case["rows"] == "own" else 0))), "flops": 4.0 * n}
    D, c = case["head_dim"], case["cache"]
    held = 2 * case["kv_heads"] * (D * SIZE[c] + (4 if c == "e4m3" else 0))  # a position's keys and values
    if case["op"] in ("append", "read"):
        n = sum(_news(case))
        rows = 2 * n * case["kv_heads"] * D * SIZE[case["dtype"]]
        return {"bytes": float(rows + n * held + 4 * (-(-n // case["page"]) + 2 * case["B"])), "flops": 2.0 * n * case["kv_heads"] * D}
    seen = sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))
    rows = case["B"] * case["heads"] * (2 * D * SIZE[case["dtype"]] + 4)
    return {"bytes": float(seen * held + rows + 4 * (-(-seen // case["page"]) + case["B"])), "flops": 4.0 * seen * case["heads"] * D}


# ------------------------------------------------------------ the same in 64 bits

def _e4m3(v):
    """v rounded to the nearest e4m3 value (ties to even mantissas), in 64 bits."""
    _, ex = torch.frexp(v)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def _walk(case, st):
    """(sequence, its rows, pages and places of their positions), one sequence after another."""
    lengths, table = st["lengths"].tolist(), st["table"].long()
    cu = st["cu"].tolist() if st.get("cu") is not None else list(range(len(lengths) + 1))
    for b, n in enumerate(lengths):
        pos = torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda")
        yield b, slice(cu[b], cu[b + 1]), table[b, pos // case["page"]], pos % case["page"]


def _stored64(case, st, name):
    x = st[name].double() if case["cache"] != "e4m3" else st[name].float().double()
    return x if case["cache"] != "e4m3" else torch.einsum("phtd,pht->phtd", x, st[name + "_scale"].double())


def _exact_append(case, st):
    out = {n: st[n].float().double() for n in (("k", "v", "k_scale", "v_scale") if case["cache"] == "e4m3" else ("k", "v"))}
    for _, rows, page, place in _walk(case, st):
        for n in ("k", "v"):
            x = st["new_" + n][rows].double()
            if case["cache"] == "e4m3":
                s = torch.linalg.vector_norm(x, ord=math.inf, dim=2) / E4M3_MAX
                s = torch.maximum(s, torch.full_like(s, FLT_MIN))
                out[n + "_scale"][page, :, place] = s
                x = _e4m3(torch.einsum("thd,th->thd", x, 1.0 / s).clamp(-E4M3_MAX, E4M3_MAX))
            out[n][page, :, place] = x
    return out


def _exact_read(case, st):
    out = {}
    for n in ("k", "v"):
        x = _stored64(case, st, n)
        out[n] = torch.cat([x[page, :, place] for _, _, page, place in _walk(case, st)])
    return out


def _exact_attend(case, st):
    B, H, D = st["q"].shape
    G = H // case["kv_heads"]
    out, lse = torch.zeros((B, H, D), dtype=torch.float64, device="cuda"), torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["lengths"].tolist()):
        pos = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device="cuda")
        if pos.numel() == 0:
            continue
        page, place = st["table"].long()[b, pos // case["page"]], pos % case["page"]
        kv = []
        for name in ("k", "v"):
            x = _token_major(st[name]).view(torch.uint8 if case["cache"] == "e4m3" else st[name].dtype)[page, place]
            x = x.view(torch.float8_e4m3fn).float().double() if case["cache"] == "e4m3" else x.double()
            if case["cache"] == "e4m3":
                x = x * _token_major(st[name + "_scale"])[page, place].double()[..., None]
            kv.append(x)
        s = torch.einsum("hgd,nhd->hgn", st["q"][b].double().view(case["kv_heads"], G, D), kv[0]) / math.sqrt(D)
        out[b] = torch.einsum("hgn,nhd->hgd", torch.softmax(s, 2), kv[1]).reshape(H, D)
        lse[b] = torch.logsumexp(s, 2).reshape(H)
    return {"out": out, "lse": lse}


def _exact_sample(case, st):
    """Row by row: the kept tokens one prefix of the sorted row, then the first whose running sum passes u."""
    prob = torch.zeros((case["T"],), dtype=torch.float64)
    at = lambda n, t: float(st[n][t]) if torch.is_tensor(st[n]) else float(torch.tensor(st[n], dtype=torch.float32))  # noqa: E731
    for t in range(case["T"]):
        z = st["logits"][t].double()
        ids = torch.argsort(z, descending=True, stable=True)
        T = at("temperature", t)
        if T <= 0:
            prob[t] = 1.0
            continue
        k = int(at("top_k", t))
        ids = ids[:k] if k > 0 else ids
        ids = ids[(z[ids] - z[ids[0]]) / T >= math.log(LEAST)]
        p = torch.softmax(z[ids] / T, 0)
        if at("top_p", t) < 1:
            before = torch.cat([p.new_zeros(1), torch.cumsum(p, 0)[:-1]])
            ids = ids[:max(1, int((before < at("top_p", t)).sum()))]
        best = z[ids[0]]
        ids = ids[(z[ids] - best) / T >= (math.log(at("min_p", t)) if at("min_p", t) > 0 else -math.inf)]
        ids = torch.sort(ids).values
        p = torch.softmax(z[ids] / T, 0)
        n = int((torch.cumsum(p, 0) <= float(st["u"][t])).sum())
        prob[t] = p[min(n, ids.numel() - 1)]
    return {"token": None, "prob": prob}


EXACT = {"append": _exact_append, "read": _exact_read, "attend": _exact_attend, "sample": _exact_sample}


def exact(case, seed):
    return EXACT[case["op"]](case, _inputs(case, seed))
