"""Refusals of the decoding loop's operators, and their references' own checks:
nothing here reaches a CUDA kernel."""
import ctypes
import math
import os
import shutil

import numpy as np
import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                reason="no CUDA toolkit to build the library")

P = 0x10000000  # a device address that is never dereferenced
FAR = 1 << 30


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("pages", "page_size", "kv_heads", "head_dim", "type")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class Sequences(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("table_width", ctypes.c_int), ("table", ctypes.c_void_p), ("table_ld", ctypes.c_int64),
                ("lengths", ctypes.c_void_p), ("cu_seqlens", ctypes.c_void_p)]


class Append(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("type", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("k_ld", "k_head_ld", "v_ld", "v_head_ld")]


class Attend(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int), ("type", ctypes.c_int), ("window", ctypes.c_int), ("scale", ctypes.c_float), ("q", ctypes.c_void_p),
                ("q_ld", ctypes.c_int64), ("q_head_ld", ctypes.c_int64), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class SampleDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("V", ctypes.c_int), ("logits_type", ctypes.c_int), ("logits", ctypes.c_void_p), ("ld", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("u", "temperatures", "top_ps", "min_ps", "top_ks")] + \
               [(n, ctypes.c_float) for n in ("temperature", "top_p", "min_p")] + [("top_k", ctypes.c_int), ("token", ctypes.c_void_p), ("prob", ctypes.c_void_p)]


CACHE = dict(pages=10, page_size=16, kv_heads=4, head_dim=128, type=1, k=P, v=P + FAR, k_scale=None, v_scale=None)
SEQS = dict(B=3, table_width=5, table=P + 2 * FAR, table_ld=5, lengths=P + 2 * FAR + 4096, cu_seqlens=None)
BAD_CACHE = [(-1, dict(pages=0)), (-1, dict(page_size=0)), (-1, dict(kv_heads=0)), (-1, dict(head_dim=0)), (-1, dict(type=0)), (-1, dict(type=4)),
             (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(k_scale=P + 3 * FAR)), (-1, dict(type=3)),
             (-1, dict(type=3, k_scale=P + 3 * FAR)), (-1, dict(v=P)), (-1, dict(v=P + 4096)), (-1, dict(type=3, k_scale=P + 256, v_scale=P + 3 * FAR)),
             (-1, dict(type=3, k_scale=P + 3 * FAR, v_scale=P + 3 * FAR + 64)),
             (-2, dict(pages=(1 << 30) + 1)), (-2, dict(page_size=4097)), (-2, dict(kv_heads=65536)), (-2, dict(head_dim=264)), (-2, dict(head_dim=100)),
             (-2, dict(head_dim=72, type=3, k_scale=P + 3 * FAR, v_scale=P + 4 * FAR)), (-2, dict(k=P + 8)), (-2, dict(v=P + FAR + 8)),
             (-2, dict(pages=1 << 30, page_size=4096, kv_heads=65535)), (-2, dict(type=3, k_scale=P + 3 * FAR + 2, v_scale=P + 4 * FAR))]
BAD_SEQS = [(-1, dict(B=-1)), (-1, dict(table_width=0)), (-1, dict(table=None)), (-1, dict(lengths=None)), (-1, dict(table_ld=4)), (-2, dict(B=65536)),
            (-2, dict(table_width=1 << 27, table_ld=1 << 27)), (-2, dict(table=P + 2)), (-2, dict(lengths=P + 2))]


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import build
    build.build()
    from paper_2608_06690_gb300 import pmpe as m
    return m


def desc(cls, base, **over):
    return ctypes.byref(cls(**dict(base, **over)))


def every_cache_and_sequences(call):
    for code, over in BAD_CACHE:
        assert call(desc(Cache, CACHE, **over), desc(Sequences, SEQS)) == code, over
    for code, over in BAD_SEQS:
        assert call(desc(Cache, CACHE), desc(Sequences, SEQS, **over)) == code, over
    assert call(None, desc(Sequences, SEQS)) == -1
    assert call(desc(Cache, CACHE), None) == -1


def test_append_refusals(pmpe):
    f = pmpe._lib.pmpe_kv_append
    base = dict(T=3, type=1, k=P + 5 * FAR, v=P + 6 * FAR, k_ld=512, k_head_ld=128, v_ld=512, v_head_ld=128)
    every_cache_and_sequences(lambda c, s: f(c, s, desc(Append, base), None))

    def rc(seqs={}, cache={}, **over):
        return f(desc(Cache, CACHE, **cache), desc(Sequences, SEQS, **seqs), desc(Append, base, **over), None)

    assert f(desc(Cache, CACHE), desc(Sequences, SEQS), None, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(T=-1), dict(T=4), dict(type=3), dict(type=-1), dict(k=None), dict(v=None), dict(k_ld=-1), dict(v_ld=-1), dict(k_head_ld=-1),
                dict(v_head_ld=-1),
                dict(k=P), dict(v=P + FAR), dict(k=P + FAR - 2), dict(v=P + 10 * 16 * 512 * 2 - 2)):  # rows inside the cache
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(k=P + 5 * FAR + 1), dict(v=P + 6 * FAR + 2, type=0), dict(k_ld=1 << 61), dict(v_head_ld=1 << 62)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(seqs=dict(cu_seqlens=P), T=(1 << 30) + 1) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc(seqs=dict(cu_seqlens=P + 2)) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc(seqs=dict(cu_seqlens=P), T=0, k=None, v=None) == pmpe.OK
    assert rc(seqs=dict(B=0, table=None, lengths=None), T=0) == pmpe.OK
    assert rc(seqs=dict(B=0, cu_seqlens=P), T=7) == pmpe.OK  # rows of no sequence


def test_read_refusals(pmpe):
    f = pmpe._lib.pmpe_kv_read
    every_cache_and_sequences(lambda c, s: f(c, s, 3, 1, P + 5 * FAR, P + 6 * FAR, None))

    def rc(T=3, type=1, k=P + 5 * FAR, v=P + 6 * FAR, **seqs):
        return f(desc(Cache, CACHE), desc(Sequences, SEQS, **seqs), T, type, k, v, None)

    for bad in (dict(T=-1), dict(T=2), dict(type=3), dict(k=None), dict(v=None), dict(k=P), dict(v=P + FAR), dict(v=P + 5 * FAR + 1024), dict(k=P - 1024)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(k=P + 5 * FAR + 1), dict(v=P + 6 * FAR + 2, type=0), dict(T=(1 << 30) + 1, cu_seqlens=P)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(T=0, k=None, v=None, cu_seqlens=P) == pmpe.OK


def test_attend_refusals(pmpe):
    f, size = pmpe._lib.pmpe_kv_attend, pmpe._lib.pmpe_kv_attend_workspace_size
    need = size(3, 32, 4, 128)
    assert need > 0 and size(-1, 32, 4, 128) == 0 and size(65536, 32, 4, 128) == 0 and size(3, 33, 4, 128) == 0 and size(3, 2, 4, 128) == 0
    assert size(3, 32, 0, 128) == 0 and size(3, 32, 4, 100) == 0 and size(3, 32, 4, 264) == 0 and size(3, 65536, 4, 128) == 0 and size(0, 32, 4, 128) > 0
    base = dict(heads=32, type=1, window=0, scale=0.1, q=P + 5 * FAR, q_ld=4096, q_head_ld=128, out=P + 6 * FAR, lse=P + 7 * FAR, workspace=P + 8 * FAR,
                workspace_bytes=need)
    every_cache_and_sequences(lambda c, s: f(c, s, desc(Attend, base), None))

    def rc(cache={}, seqs={}, **over):
        return f(desc(Cache, CACHE, **cache), desc(Sequences, SEQS, **seqs), desc(Attend, base, **over), None)

    assert f(desc(Cache, CACHE), desc(Sequences, SEQS), None, None) == pmpe.ERR_INVALID_ARG
    eight = dict(type=3, k_scale=P + 9 * FAR, v_scale=P + 10 * FAR)
    for bad in (dict(heads=0), dict(heads=-4), dict(heads=33), dict(type=2), dict(type=0), dict(window=-1), dict(scale=math.nan), dict(scale=math.inf),
                dict(q=None), dict(out=None), dict(q_ld=-1), dict(q_head_ld=-1), dict(out=P + 5 * FAR), dict(out=P + 5 * FAR + 3 * 8192 - 2), dict(out=P),
                dict(out=P + FAR), dict(lse=P + 6 * FAR + 64), dict(lse=P + 5 * FAR), dict(lse=P + 64), dict(cache=eight, type=0), dict(cache=eight, type=3)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(heads=65540, q_ld=1 << 30), dict(q=P + 5 * FAR + 1), dict(out=P + 6 * FAR + 1), dict(lse=P + 7 * FAR + 2), dict(q_ld=1 << 61)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    for bad in (dict(workspace=None), dict(workspace=P + 8 * FAR + 8), dict(workspace_bytes=need - 1)):
        assert rc(**bad) == pmpe.ERR_WORKSPACE, bad
    assert rc(seqs=dict(B=0, table=None, lengths=None), q=None, out=None, workspace=None) == pmpe.OK


def test_sample_refusals(pmpe):
    f = pmpe._lib.pmpe_sample
    base = dict(T=3, V=1000, logits_type=0, logits=P, ld=1000, u=P + FAR, temperatures=None, top_ps=None, min_ps=None, top_ks=None, temperature=1.0, top_p=0.9,
                min_p=0.1, top_k=5, token=P + 2 * FAR, prob=P + 3 * FAR)

    def rc(**over):
        return f(desc(SampleDesc, base, **over), None)

    assert f(None, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(T=-1), dict(V=0), dict(logits_type=3), dict(ld=-1), dict(logits=None), dict(u=None), dict(token=None), dict(prob=None),
                dict(temperature=-0.5), dict(temperature=math.nan), dict(temperature=math.inf), dict(top_p=-0.1), dict(top_p=1.1), dict(top_p=math.nan),
                dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=math.nan), dict(top_k=-1), dict(token=P + 64), dict(prob=P + 11996), dict(token=P + FAR),
                dict(prob=P + 2 * FAR + 8), dict(top_ks=P + 3 * FAR)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(T=(1 << 30) + 1), dict(V=(1 << 21) + 1, ld=1 << 22), dict(ld=1 << 31), dict(logits=P + 2), dict(logits=P + 1, logits_type=1), dict(u=P + FAR + 2),
                dict(token=P + 2 * FAR + 2), dict(prob=P + 3 * FAR + 1), dict(temperatures=P + 1), dict(top_ps=P + 2), dict(min_ps=P + 2), dict(top_ks=P + 2)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(T=0, logits=None, u=None, token=None, prob=None) == pmpe.OK
    # what rows have of their own is not the host's to check
    assert rc(T=0, temperatures=P, top_ps=P, min_ps=P, top_ks=P, temperature=-1.0, top_p=7.0, min_p=-2.0, top_k=-4) == pmpe.OK


def test_host_tensors_and_other_types_are_refused(pmpe):
    k = torch.zeros(4, 2, 8, 16, dtype=torch.bfloat16)
    with pytest.raises(pmpe.PmpeError, match="CUDA"):
        pmpe.KvCache(k, k.clone())
    k8, s = k.to(torch.float8_e4m3fn), torch.zeros(4, 2, 8)
    for bad in ((None, k), (k, None), (k, k.half()), (k, k[:3]), (k.float(), k.float()), (k[..., :8], k[..., :8]), (k[0], k[0]), (k, k, s, s), (k8, k8), (k8, k8, s, None),
                (k8, k8, s, s[:3]), (k8, k8, s, s.double()), (k8, k8, s.transpose(1, 2).contiguous().transpose(1, 2), s), (k, k, 1.0)):
        with pytest.raises(pmpe.PmpeError):
            pmpe.KvCache(*bad)
    z, u = torch.zeros(2, 8), torch.zeros(2)
    for call in (lambda: pmpe.sample(z, u), lambda: pmpe.sample(None, u), lambda: pmpe.sample([[0.0]], u), lambda: pmpe._ops.sample(z, u)):
        with pytest.raises(pmpe.PmpeError):
            call()


# ------------------------------------------------ the references themselves

def test_reference_entries_by_hand():
    table = np.array([[3, 7], [1, -1], [9, 2]])
    lengths, cu = np.array([5, 4, 3]), np.array([0, 2, 2, 5])
    # sequence 0's positions 3 and 4, none of sequence 1's, 2's positions 0 to 2 (page 9 is none of 8), padding
    assert ref.kv_entries(table, lengths, cu, 6, 8, 4) == [(3, 3), (7, 0), None, None, None, None]
    assert ref.kv_entries(table, lengths, None, 3, 10, 4) == [(7, 0), (1, 3), (9, 2)]
    assert ref.kv_entries(table, np.array([1, 9, 0]), None, 3, 10, 4) == [(3, 0), None, None]  # past the table; an empty sequence
    assert ref.kv_entries(table, np.array([1, 2, 2]), cu, 5, 10, 4)[:2] == [None, (3, 0)]      # more rows than positions
    page, place = ref.kv_seen([3, -1, 4], 11, 9, 8, 4)
    assert page.tolist() == [3, 3, 4, 4, 4] and place.tolist() == [2, 3, 0, 1, 2]
    assert [len(x) for x in ref.kv_seen([3, 4], 99, 0, 8, 4)] == [8, 8] and len(ref.kv_seen([3], -5, 0, 8, 4)[0]) == 0


def test_reference_attention_by_hand():
    q, k = np.array([[2.0, 0.0], [0.0, 0.0]]), np.array([[[0.5, 9.0]], [[-0.5, 7.0]]])
    v = np.array([[[1.0, 0.0]], [[0.0, 1.0]]])
    out, lse, size, scores = ref.attend(q, k, v, 0.5)
    a = 1 / (1 + math.exp(-1.0))
    assert np.allclose(out, [[a, 1 - a], [0.5, 0.5]]) and np.allclose(lse, [math.log(math.exp(0.5) + math.exp(-0.5)), math.log(2)])
    assert np.allclose(scores, [0.5, 0.0]) and np.allclose(size, out)
    out, lse, _, _ = ref.attend(q, k[:0], v[:0], 0.5)
    assert not out.any() and (lse == -np.inf).all()


def test_reference_e4m3():
    x = torch.linspace(-500, 500, 4001, dtype=torch.float64)
    x = torch.cat([x, x * 2.0 ** -12, x * 2.0 ** -17])
    want = x.clamp(-448, 448).float().to(torch.float8_e4m3fn).double()
    assert np.array_equal(ref.e4m3(x.numpy()), want.numpy())


def test_reference_sampling_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.1, 0.3, 0.1]))
    assert ref.sample_row(z, 0.05)[:1] == (0,) and ref.sample_row(z, 0.11)[0] == 1 and ref.sample_row(z, 0.999)[0] == 4
    assert ref.sample_row(z, 0.0, top_k=2)[2].tolist() == [1, 3] and ref.sample_row(z, 0.6, top_k=2)[0] == 3
    assert ref.sample_row(z, 0.0, top_k=3)[2].tolist() == [0, 1, 3]  # equal ones by the lower id
    assert ref.sample_row(z, 0.0, top_p=0.39)[2].tolist() == [1] and ref.sample_row(z, 0.0, top_p=0.41)[2].tolist() == [1, 3]
    assert ref.sample_row(z, 0.0, top_k=2, top_p=0.5)[2].tolist() == [1]  # 4 / 7 of the two
    assert ref.sample_row(z, 0.0, min_p=0.5)[2].tolist() == [1, 3] and ref.sample_row(z, 0.9, min_p=1.0)[2].tolist() == [1]
    assert ref.sample_row(z, 0.9, temperature=0.0)[:2] == (1, 1.0) and ref.sample_row(z * 0 - np.inf, 0.9)[:2] == (-1, 0.0)
    assert abs(ref.sample_row(z, 0.7, temperature=0.5)[1] - 0.09 / 0.28) < 1e-12
    assert ref.sample_row([0.0, -28.0, np.nan], 0.0)[2].tolist() == [0]  # 40 ln 2 is 27.7
