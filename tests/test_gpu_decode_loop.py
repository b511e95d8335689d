"""A decoding loop as a user writes it, from the prompt on: norm, projections,
the cache, attention over it, the expert layer and the next token; eagerly and
captured into a graph whose replays make the further tokens."""
import numpy as np
import pytest
import torch

import operators_ref as ref
from paper_2608_06690_gb300 import pmpe
from paper_2608_06690_gb300.inputs import LayerShape
from pmpe_testlib import make_layer, to_device

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
HEADS, KV, D, H, V, PAGE = 8, 2, 64, 256, 3001, 16
PROMPTS = [5, 0, 33, 16, 1]  # the second slot of the batch is empty
STEPS = 6


class Model:
    """One block around the layer and the two ends of a model."""

    def __init__(self, cache_dtype):
        B = len(PROMPTS)
        self.shape = LayerShape(T=B, H=H, I=128, E_pub=8, E_priv=4, E_sh=1, k=2, renormalize=True)
        weights, _, _ = to_device(*make_layer(self.shape, 3, policy="iid"))
        self.layer = pmpe.MoeLayer(self.shape, weights)
        self.policy = torch.tensor([1, 0, 0, 1, 1], dtype=torch.uint8).cuda()
        g = torch.Generator().manual_seed(5)
        w = lambda *s: (torch.randn(s, generator=g) / s[-1] ** 0.5).to(BF16).cuda()  # noqa: E731
        self.embed, self.w_qkv, self.w_o, self.w_out = w(V, H) * 16, w((HEADS + 2 * KV) * D, H), w(H, HEADS * D), 3 * w(V, H)
        self.norms = [1 + 0.1 * w(H).float() for _ in range(3)]
        self.cache = pmpe.KvCache.empty(40, PAGE, KV, D, cache_dtype)
        self.table = torch.randperm(40, generator=g)[:B * 5].view(B, 5).to(torch.int32).cuda()
        self.lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(B, device="cuda")
        self.seen = {}

    def qkv(self, x):
        rows = pmpe.rms_norm(x, self.norms[0]).y @ self.w_qkv.T
        heads = rows.view(-1, HEADS + 2 * KV, D)  # views of the fused rows, as they are
        return heads[:, :HEADS], heads[:, HEADS:HEADS + KV], heads[:, HEADS + KV:]

    def prompt(self):
        """The prompts' keys and values (padded by three rows), and their last tokens."""
        g = torch.Generator().manual_seed(9)
        T = sum(PROMPTS)
        tokens = torch.randint(0, V, (T + 3,), generator=g).cuda()
        cu = torch.tensor(np.concatenate([[0], np.cumsum(PROMPTS)]), dtype=torch.int32).cuda()
        self.lengths.copy_(torch.tensor(PROMPTS, dtype=torch.int32))
        _, k, v = self.qkv(self.embed[tokens])
        self.cache.append(k, v, self.table, self.lengths, cu_seqlens=cu)
        back_k, back_v = self.cache.read(self.table, self.lengths, cu_seqlens=cu, rows=T)
        return (k[:T], v[:T]), (back_k, back_v), torch.randint(0, V, (len(PROMPTS),), generator=g).to(torch.int32).cuda()

    def step(self, token):
        x = self.embed[token.long().clamp(min=0)]
        self.lengths += (self.lengths > 0).int()  # empty slots stay empty
        q, k, v = self.qkv(x)
        self.cache.append(k, v, self.table, self.lengths)
        a = self.cache.attend(q, self.table, self.lengths)
        n = pmpe.rms_norm(a.out.flatten(1) @ self.w_o.T, self.norms[1], residual=x)
        h = n.h + self.layer.forward(n.y, self.policy)
        logits = (pmpe.rms_norm(h, self.norms[2]).y @ self.w_out.T).float()
        s = pmpe.sample(logits, self.u, temperature=0.8, top_k=200, top_p=0.95)
        self.seen = dict(q=q, a=a, logits=logits, sample=s)
        return s.token


def us(i):
    return torch.rand(len(PROMPTS), generator=torch.Generator().manual_seed(100 + i))


def attention64(m):
    """The attention of the last step in 64 bits, from what the cache holds."""
    outs = []
    for b, n in enumerate(m.lengths.tolist()):
        page, place = ref.kv_seen(m.table[b].cpu().numpy(), n, 0, 40, PAGE)
        kv = []
        for t, sc in ((m.cache.k, m.cache.k_scale), (m.cache.v, m.cache.v_scale)):
            x = t.float().double().cpu().numpy()
            kv.append((x if sc is None else x * sc.double().cpu().numpy()[..., None])[page, :, place])
        outs.append(ref.attend(m.seen["q"][b].double().cpu().numpy(), *kv, D ** -0.5))
    return outs


@pytest.mark.parametrize("cache_dtype", [BF16, E4M3])
def test_a_decoding_loop(cache_dtype):
    eager, graphed = Model(cache_dtype), Model(cache_dtype)
    (k, v), back, token = eager.prompt()
    for x, y in zip((k, v), back):  # a head's largest rounding: none in 16 bits, half an e4m3 step of values up to its amax
        tol = 0.0 if cache_dtype == BF16 else 2.0 ** -4 + 2.0 ** -8
        assert ((x.float() - y.float()).abs() <= tol * x.float().abs() + (cache_dtype == E4M3) * 2.0 ** -18 * x.float().abs().amax(2, keepdim=True)).all()
    tokens = [token]
    for i in range(STEPS):
        eager.u.copy_(us(i))
        tokens.append(eager.step(tokens[-1]))
        torch.cuda.synchronize()
        for b, (want, lse, size, scores) in enumerate(attention64(eager)):
            got = eager.seen["a"].out[b].double().cpu().numpy()
            assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -15 + 2.0 ** -15 * scores[:, None]) * size + 1e-30).all()
        z = eager.seen["logits"].double().cpu().numpy()
        for b in range(len(PROMPTS)):
            t, p, _ = ref.sample_row(z[b], float(eager.u[b]), float(np.float32(0.8)), 200, float(np.float32(0.95)))
            assert t == int(tokens[-1][b]) and abs(p - float(eager.seen["sample"].prob[b])) <= 2.0 ** -22 * p
    assert eager.lengths.tolist() == [n + STEPS if n else 0 for n in PROMPTS]
    assert not eager.seen["a"].out[1].any()

    # the same from a graph: a warm-up step on a side stream is taken back first
    _, _, token = graphed.prompt()
    current = token.clone()
    held = [t.clone() for t in graphed.cache._held if t is not None], graphed.lengths.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(current)
    torch.cuda.current_stream().wait_stream(side)
    for t, w in zip((t for t in graphed.cache._held if t is not None), held[0]):
        t.copy_(w)
    graphed.lengths.copy_(held[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        current.copy_(graphed.step(current))
    for i in range(STEPS):
        graphed.u.copy_(us(i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(current, tokens[i + 1]), i
    assert torch.equal(graphed.seen["a"].out, eager.seen["a"].out) and torch.equal(graphed.seen["a"].lse, eager.seen["a"].lse)
    assert torch.equal(graphed.cache.k.view(torch.uint8), eager.cache.k.view(torch.uint8))


def test_two_streams_at_once():
    """Two batches over caches of their own on streams of their own, at the same time."""
    models = [Model(BF16), Model(E4M3)]
    alone = []
    for m in models:
        _, _, token = m.prompt()
        m.u.copy_(us(0))
        t = m.step(token)
        alone.append((t.clone(), m.seen["a"].out.clone()))
    torch.cuda.synchronize()
    again = [Model(BF16), Model(E4M3)]
    streams, got = [torch.cuda.Stream() for _ in again], []
    starts = [m.prompt()[2] for m in again]
    torch.cuda.synchronize()
    for m, s, token in zip(again, streams, starts):
        with torch.cuda.stream(s):
            m.u.copy_(us(0))
            t = m.step(token)
            got.append((t, m.seen["a"].out))
    torch.cuda.synchronize()
    for (t, o), (wt, wo) in zip(got, alone):
        assert torch.equal(t, wt) and torch.equal(o, wo)
