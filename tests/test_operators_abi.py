"""Refusals of the operators around the layer, and their references' own
checks: nothing here reaches a CUDA kernel."""
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


class RmsNormDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("H", ctypes.c_int), ("type", ctypes.c_int), ("weight_type", ctypes.c_int),
                ("quant", ctypes.c_int), ("eps", ctypes.c_float), ("x", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("x_ld", ctypes.c_int64), ("residual_ld", ctypes.c_int64), ("h", ctypes.c_void_p), ("y", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("rstd", ctypes.c_void_p)]


class RmsNormBackwardDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("H", ctypes.c_int), ("type", ctypes.c_int), ("weight_type", ctypes.c_int),
                ("dy_type", ctypes.c_int), ("dx_type", ctypes.c_int), ("dy", ctypes.c_void_p), ("h", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("rstd", ctypes.c_void_p), ("d_h", ctypes.c_void_p), ("dx", ctypes.c_void_p), ("dw", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class RouteDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("T", "E_pub", "E_priv", "k", "logits_type", "score", "renormalize", "groups_pub",
                                            "top_groups_pub", "groups_priv", "top_groups_priv", "group_score")] + \
               [("scale", ctypes.c_float), ("logits", ctypes.c_void_p), ("ld", ctypes.c_int64), ("policy", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("topk_idx", ctypes.c_void_p), ("topk_w", ctypes.c_void_p), ("load", ctypes.c_void_p)]


class Grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int)]


@pytest.fixture(scope="module")
def pmpe():
    from paper_2608_06690_gb300 import build
    build.build()
    from paper_2608_06690_gb300 import pmpe as m
    return m


def desc(cls, base, **over):
    d = cls(**dict(base, **over))
    return ctypes.byref(d)


def test_rms_norm_refusals(pmpe):
    f = pmpe._lib.pmpe_rms_norm
    base = dict(T=4, H=256, type=1, weight_type=1, quant=0, eps=1e-6, x=P, residual=P, weight=P, x_ld=256, residual_ld=256,
                h=P, y=P, scale=None, rstd=P)

    def rc(**over):
        return f(desc(RmsNormDesc, base, **over), None)

    assert f(None, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(T=-1), dict(H=0), dict(H=-5), dict(type=3), dict(type=-1), dict(weight_type=2), dict(quant=3), dict(quant=-1),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(x=None), dict(weight=None),
                dict(y=None), dict(x_ld=255), dict(residual_ld=255), dict(quant=1), dict(scale=P)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(T=(1 << 30) + 1), dict(H=16385, x_ld=16385, residual_ld=16385), dict(x=P + 1), dict(residual=P + 1), dict(h=P + 1), dict(y=P + 1),
                dict(weight=P + 2, weight_type=0), dict(rstd=P + 2), dict(quant=1, scale=P + 2)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(T=0, x=None, weight=None, y=None) == pmpe.OK


def test_rms_norm_outputs_that_share_memory_are_refused(pmpe):
    """Rows of 256 BF16 values (512 bytes), four of them, 600 elements apart."""
    f = pmpe._lib.pmpe_rms_norm
    far = 1 << 20
    base = dict(T=4, H=256, type=1, weight_type=1, quant=0, eps=1e-6, x=P, residual=P + far, weight=P + 2 * far, x_ld=600, residual_ld=256,
                h=P + 3 * far, y=P + 4 * far, scale=None, rstd=P + 5 * far)
    bad = [dict(h=P), dict(y=P),                                          # on rows of another pitch
           dict(h=P - 2046), dict(h=P + 510), dict(h=P + 3600 + 510), dict(y=P + 1000), dict(y=P + far + 512), dict(h=P + far + 2),
           dict(h=P + far - 2), dict(y=P + far + 2046), dict(h=P + 2 * far), dict(y=P + 2 * far + 510), dict(y=P + 2 * far - 2046),
           dict(h=P + 4 * far), dict(h=P + 4 * far + 2046), dict(h=P + far, x=P + far + 512, x_ld=256)]
    for quant in (1, 2):
        bad += [dict(quant=quant, scale=P + 6 * far, y=P + far), dict(quant=quant, scale=P + 6 * far, y=P + far - 1023),
                dict(quant=quant, scale=P + 6 * far, y=P + far + 2047)]
    for over in bad:
        assert f(desc(RmsNormDesc, base, **over), None) == pmpe.ERR_INVALID_ARG, over


def test_rms_norm_backward_refusals(pmpe):
    f, size = pmpe._lib.pmpe_rms_norm_backward, pmpe._lib.pmpe_rms_norm_backward_workspace_size
    need = size(4, 256)
    assert need > 0 and size(-1, 256) == 0 and size(4, 0) == 0 and size(4, 16385) == 0 and size(0, 256) > 0
    assert size(1 << 20, 256) == size(1 << 21, 256)  # bounded: a partial sum a CTA
    base = dict(T=4, H=256, type=1, weight_type=1, dy_type=0, dx_type=1, dy=P, h=P, weight=P, rstd=P, d_h=P, dx=P, dw=P,
                workspace=P, workspace_bytes=need)

    def rc(**over):
        return f(desc(RmsNormBackwardDesc, base, **over), None)

    assert f(None, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(T=-1), dict(H=0), dict(type=9), dict(weight_type=2), dict(dy_type=2), dict(dx_type=2), dict(dy=None),
                dict(h=None), dict(weight=None), dict(rstd=None), dict(dx=None)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(T=(1 << 30) + 1), dict(H=16385), dict(dy=P + 2), dict(h=P + 1), dict(d_h=P + 1), dict(dx=P + 1), dict(dw=P + 2), dict(rstd=P + 2)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    for bad in (dict(workspace=None), dict(workspace=P + 8), dict(workspace_bytes=need - 1)):
        assert rc(**bad) == pmpe.ERR_WORKSPACE, bad
    assert rc(T=0, dw=None, dy=None, h=None, workspace=None) == pmpe.OK


ROUTE = dict(T=4, E_pub=16, E_priv=4, k=2, logits_type=0, score=0, renormalize=1, groups_pub=1, top_groups_pub=1, groups_priv=1,
             top_groups_priv=1, group_score=0, scale=1.0, logits=P, ld=20, policy=P, bias=P, topk_idx=P, topk_w=P, load=P)


def test_route_refusals(pmpe):
    f = pmpe._lib.pmpe_route

    def rc(**over):
        return f(desc(RouteDesc, ROUTE, **over), None)

    assert f(None, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(T=-1), dict(k=0), dict(k=5), dict(E_pub=1), dict(E_priv=-1), dict(E_priv=1), dict(logits_type=3), dict(score=2),
                dict(score=-1), dict(renormalize=2), dict(scale=math.inf), dict(scale=math.nan), dict(ld=19), dict(logits=None),
                dict(topk_idx=None), dict(topk_w=None), dict(group_score=2), dict(groups_pub=0), dict(groups_pub=3),
                dict(groups_pub=4, top_groups_pub=0), dict(groups_pub=4, top_groups_pub=5), dict(groups_pub=33),
                dict(groups_pub=16, top_groups_pub=1), dict(groups_priv=4, top_groups_priv=1), dict(groups_priv=3),
                dict(E_priv=0)):  # a policy without a private pool
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(T=(1 << 30) + 1), dict(E_pub=257, ld=300), dict(E_priv=257, ld=300), dict(E_pub=64, E_priv=64, ld=128, k=33), dict(logits=P + 2),
                dict(topk_idx=P + 1), dict(topk_w=P + 2), dict(bias=P + 2), dict(load=P + 2)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(T=0, logits=None, topk_idx=None, topk_w=None) == pmpe.OK
    assert rc(T=0, E_priv=0, policy=None, groups_priv=0) == pmpe.OK
    with pytest.raises(pmpe.PmpeError):
        pmpe.Router(16, 4, 5)
    with pytest.raises(pmpe.PmpeError):
        pmpe.Router(16, 4, 2, score="tanh")
    with pytest.raises(pmpe.PmpeError):
        pmpe.Router(16, 4, 2, group_score="mean")
    with pytest.raises(pmpe.PmpeError):
        pmpe.Router(16, 4, 2, groups=(5, 1))


def test_route_backward_refusals(pmpe):
    f = pmpe._lib.pmpe_route_backward

    def rc(dw=P, d_logits=P, **over):
        return f(desc(RouteDesc, ROUTE, **over), dw, d_logits, None)

    for bad in (dict(dw=None), dict(d_logits=None), dict(k=0), dict(T=-1), dict(ld=3), dict(topk_idx=None)):
        assert rc(**bad) == pmpe.ERR_INVALID_ARG, bad
    for bad in (dict(dw=P + 2), dict(d_logits=P + 2), dict(d_logits=P + 1, logits_type=1)):
        assert rc(**bad) == pmpe.ERR_UNSUPPORTED_SHAPE, bad
    assert rc(T=0, dw=None, d_logits=None, logits=None, topk_idx=None) == pmpe.OK


def test_clip_refusals(pmpe):
    f, size = pmpe._lib.pmpe_clip_grad_norm, pmpe._lib.pmpe_clip_workspace_size
    assert size(-1) == 0 and size(0) > 0 and size(5000) > size(5)

    def rc(tensors, max_norm=1.0, norm=P, ws=P, nb=None, n=None):
        table = (Grad * max(1, len(tensors)))(*tensors)
        return f(table, len(tensors) if n is None else n, max_norm, norm, ws, size(len(tensors)) if nb is None else nb, None)

    ok = (P, None, 1000, 0)
    assert f(None, 1, 1.0, P, P, 1 << 20, None) == pmpe.ERR_INVALID_ARG
    assert rc([ok], n=-1) == pmpe.ERR_INVALID_ARG
    assert rc([ok], max_norm=-1.0) == pmpe.ERR_INVALID_ARG
    assert rc([ok], max_norm=math.nan) == pmpe.ERR_INVALID_ARG
    assert rc([ok], norm=None) == pmpe.ERR_INVALID_ARG
    assert rc([(P, None, -1, 0)]) == pmpe.ERR_INVALID_ARG
    assert rc([(P, None, 4, 7)]) == pmpe.ERR_INVALID_ARG
    assert rc([(None, None, 4, 0)]) == pmpe.ERR_INVALID_ARG
    assert rc([ok, ok]) == pmpe.ERR_INVALID_ARG                                # the same tensor twice
    assert rc([ok, (P + 3996, None, 10, 0)]) == pmpe.ERR_INVALID_ARG           # the last element shared
    assert rc([ok, (P + 8000, P + 400, 10, 0)]) == pmpe.ERR_INVALID_ARG        # an output inside another gradient
    assert rc([(P, P + 4, 1000, 0)]) == pmpe.ERR_INVALID_ARG                   # an output that overlaps its own gradient
    assert rc([(P + 2, None, 4, 0)]) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc([(P, P + 0x100001, 4, 1)]) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc([(P, None, 1 << 45, 0)]) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc([(P, None, 1 << 44, 0)]) == pmpe.ERR_INVALID_ARG                 # more chunks than a launch counts
    assert rc([ok], norm=P + 0x100002) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert rc([ok], ws=None) == pmpe.ERR_WORKSPACE
    assert rc([ok], ws=P + 0x100008) == pmpe.ERR_WORKSPACE
    assert rc([ok], nb=size(1) - 1) == pmpe.ERR_WORKSPACE


def test_clip_refuses_more_tensors_than_it_counts(pmpe):
    f, size = pmpe._lib.pmpe_clip_grad_norm, pmpe._lib.pmpe_clip_workspace_size
    per = size(1)  # of a launch's 1024 tensors
    assert size(1024) == per and size(1025) == 2 * per and size(1 << 30) == per << 20
    for n in ((1 << 30) + 1, 2 ** 31 - 1000, 2 ** 31 - 1):
        assert size(n) == 0
        assert f(P, n, 1.0, P, P, 1 << 40, None) == pmpe.ERR_UNSUPPORTED_SHAPE  # before the host array is read


def test_host_tensors_are_refused(pmpe):
    x, w = torch.zeros(2, 8), torch.ones(8)
    for call in (lambda: pmpe.rms_norm(x, w), lambda: pmpe.rms_norm_backward(x, x, w, torch.ones(2)),
                 lambda: pmpe.Router(8, 0, 2).route(x), lambda: pmpe.clip_grad_norm([x], 1.0), lambda: pmpe.clip_grad_norm([], 1.0),
                 lambda: pmpe.clip_grad_norm({"a": x}, 1.0, out={"b": x})):
        with pytest.raises(pmpe.PmpeError):
            call()


def test_arguments_of_other_types_are_refused(pmpe):
    """Nothing but tensors reaches a tensor's place, and errors of Python's own
    conversions come through as they are."""
    x, w, r = torch.zeros(2, 8), torch.ones(8), pmpe.Router(8, 0, 2)
    for call in (lambda: pmpe.rms_norm(None, w), lambda: pmpe.rms_norm(x, 1.0), lambda: pmpe.rms_norm(x, w, residual=[x]),
                 lambda: pmpe.rms_norm(x, w, quant="tensor"), lambda: pmpe.rms_norm(x, w, quant=1), lambda: pmpe.rms_norm(x, w, h_out="h"),
                 lambda: pmpe.rms_norm_backward(x, None, w, w), lambda: pmpe.rms_norm_backward(x, x, w, w, d_h=0),
                 lambda: r.route([[0.0] * 8]), lambda: r.route(x, policy=1), lambda: r.route(x, load={}), lambda: r.backward(x, None, None, x),
                 lambda: pmpe.clip_grad_norm(x, 1.0), lambda: pmpe.clip_grad_norm([None], 1.0), lambda: pmpe.clip_grad_norm([x], 1.0, out=x),
                 lambda: pmpe.clip_grad_norm(iter([x]), 1.0), lambda: pmpe._ops.rms_norm(x, w), lambda: pmpe._ops.route(b"", x, None, None, None),
                 lambda: pmpe._ops.route_backward(r._desc)):
        with pytest.raises(pmpe.PmpeError):
            call()
    for call in (lambda: pmpe.rms_norm(x, w, eps="small"), lambda: pmpe.clip_grad_norm([x], "1"), lambda: pmpe.Router(8, 0, "two")):
        with pytest.raises((TypeError, ValueError)):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_weights_of_another_size_type_or_order_are_refused(pmpe, dtype):
    """Whatever the rows' type is; the weight is looked at before the device is,
    so that its own message shows."""
    x, r = torch.zeros(2, 8, dtype=dtype), torch.ones(2)
    other = torch.float16 if dtype is torch.bfloat16 else torch.bfloat16
    for w in (torch.ones(8, dtype=other), torch.ones(8).double(), torch.ones(8, dtype=torch.int32), torch.ones(7, dtype=dtype), torch.ones(7),
              torch.ones(9), torch.ones(0), torch.ones(1, 8), torch.ones(1).expand(8), torch.ones(16)[::2], torch.ones(())):
        with pytest.raises(pmpe.PmpeError, match="rms_norm: weight is"):
            pmpe.rms_norm(x, w)
        with pytest.raises(pmpe.PmpeError, match="rms_norm_backward: weight is"):
            pmpe.rms_norm_backward(x, x, w, r)
    for w in (torch.ones(8, dtype=dtype), torch.ones(8)):  # nothing but the device is wrong
        with pytest.raises(pmpe.PmpeError, match="x is a CUDA tensor"):
            pmpe.rms_norm(x, w)
        with pytest.raises(pmpe.PmpeError, match="h is a CUDA tensor"):
            pmpe.rms_norm_backward(x, x, w, r)


def test_the_layers_rows_are_checked(pmpe):
    """Host tensors, and hidden states in a backward that cannot be the
    forward's, are refused before anything is allocated or launched."""
    from paper_2608_06690_gb300.inputs import LayerShape
    layer = pmpe.MoeLayer(LayerShape(6, 256, 128, 8, 4, 0, 2, True), {}, device="cpu")
    h, pol = torch.zeros(6, 256, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.uint8)
    idx, w = torch.zeros(6, 2, dtype=torch.int32), torch.zeros(6, 2)
    for kw in (dict(), dict(route=(idx, w))):
        with pytest.raises(pmpe.PmpeError, match="MoeLayer.forward: CUDA tensors"):
            layer.forward(h, pol, **kw)
    for given in (False, True):
        layer._given, layer._route_out = given, (idx, w)
        backs = (layer.backward_routed,) if given else (layer.backward, layer.backward_private, layer.backward_input)
        for back in backs:
            for hidden in (h, h.float(), h[:, :128], h.t().contiguous().t(), torch.zeros(6, 512, dtype=torch.bfloat16)[:, ::2]):
                with pytest.raises(pmpe.PmpeError, match="hidden is the forward's"):
                    back(hidden, pol, h)


WITHOUT_OPS = """
import sys, torch
from paper_2608_06690_gb300 import pmpe
from paper_2608_06690_gb300.inputs import LayerShape
s = LayerShape(64, 256, 128, 8, 4, 0, 2, True)
assert pmpe.workspace_size(s) > 0 and pmpe.MoeLayer(s, {}, device="cpu").shape is s
x = torch.zeros(2, 8)
for call in (lambda: pmpe.rms_norm(x, x[0]), lambda: pmpe.rms_norm_backward(x, x, x[0], x[:, 0]), lambda: pmpe.Router(8, 0, 2),
             lambda: pmpe.clip_grad_norm([x], 1.0)):
    try:
        call()
    except ImportError as e:
        assert "_ops.so" in str(e) and sys.argv[1] in str(e) and "build" in str(e), e
    else:
        raise AssertionError("no ImportError")
"""


@pytest.mark.parametrize("kind", ["missing", "broken", "another", "older"])
def test_the_layer_does_not_need_the_operators_module(pmpe, kind, tmp_path):
    """Without _ops, with one that does not load or one that was built for
    another PyTorch, the layer is there and the operators say what is missing."""
    import subprocess
    import sys
    src = os.path.dirname(pmpe.__file__)
    to = tmp_path / "paper_2608_06690_gb300"
    to.mkdir()
    for f in os.listdir(src):
        if f.endswith(".py") or f == "libpmpe.so":
            shutil.copy(os.path.join(src, f), to / f)
    says = "No module named"
    if kind == "broken":
        (to / "_ops.so").write_bytes(b"not a library")
        says = "_ops.so"
    elif kind == "another":
        (to / "_ops.py").write_text("built_for = '1.0'")
        says = "built for PyTorch 1.0"
    elif kind == "older":
        (to / "_ops.py").write_text("")
        says = "of another version"
    subprocess.run([sys.executable, "-c", WITHOUT_OPS, says], cwd=tmp_path, check=True, env=dict(os.environ, PYTHONPATH=str(tmp_path)))


def test_the_library_is_built_where_the_module_cannot_be(pmpe, tmp_path, monkeypatch):
    from paper_2608_06690_gb300 import build

    def no_torch():
        raise ImportError("No module named 'torch'")

    for command in (lambda: (["false"], "another"), no_torch):
        monkeypatch.setattr(build, "OUT", str(tmp_path / "libpmpe.so"))
        monkeypatch.setattr(build, "OPS_OUT", str(tmp_path / "_ops.so"))
        monkeypatch.setattr(build, "_ops_command", command)
        (tmp_path / "_ops.so").write_bytes(b"of another PyTorch")
        with pytest.raises(RuntimeError, match="building _ops.so failed"):
            build.build()
        assert (tmp_path / "libpmpe.so").exists() and not (tmp_path / "_ops.so").exists()
        os.remove(tmp_path / "libpmpe.so")


# ------------------------------------------------ the references themselves

def test_reference_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    h, w, dy, dh = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    eps, step = 1e-3, 1e-6

    def loss(h, w):
        return (ref.rms_norm(h, w, eps)[0] * dy).sum() + (h * dh).sum()

    dx, dw, _, _ = ref.rms_norm_backward(dy, h, w, ref.rms_norm(h, w, eps)[1], dh)
    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = step
        assert abs((loss(h + e, w) - loss(h - e, w)) / (2 * step) - dx[i]) < 1e-7  # step^2 f''' / 6 + 2^-52 |f| / step
    for i in range(7):
        e = np.zeros_like(w)
        e[i] = step
        assert abs((loss(h, w + e) - loss(h, w - e)) / (2 * step) - dw[i]) < 1e-7


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_reference_route_gradient_against_differences(sigmoid, renorm):
    rng = np.random.default_rng(1)
    z, policy = rng.normal(size=(3, 9)), np.array([0, 1, 7], np.uint8)
    idx, _ = ref.route(z, policy, 5, 4, 3, sigmoid, renorm, 2.5)
    dw = rng.normal(size=(3, 3))
    d, _ = ref.route_backward(z, policy, idx, dw, 5, 4, sigmoid, renorm, 2.5)

    def loss(z):
        total = 0.0
        for t in range(3):
            lo, hi = ref.pool_of(t, policy, 5, 4)
            total += (ref.weights(z[t, lo:hi], idx[t] - lo, sigmoid, renorm, 2.5) * dw[t]).sum()
        return total

    for i in np.ndindex(z.shape):
        e = np.zeros_like(z)
        e[i] = 1e-6
        assert abs((loss(z + e) - loss(z - e)) / 2e-6 - d[i]) < 1e-7


def test_reference_route_by_hand():
    z = np.array([[0.0, 2.0, 2.0, -np.inf, 1.0, 3.0]])
    idx, w = ref.route(z, None, 6, 0, 3)
    assert idx.tolist() == [[5, 1, 2]]  # equal logits by the lower id
    assert np.allclose(w, np.exp([[3, 2, 2]]) / np.exp([3, 2, 2]).sum())
    idx, _ = ref.route(z, None, 6, 0, 2, groups=(3, 1))  # groups {0, 1}, {2, -}, {1, 3}: the last by its best
    assert idx.tolist() == [[5, 4]]
    idx, _ = ref.route(z, None, 6, 0, 2, sigmoid=True, groups=(3, 1), top2=True, bias=np.array([9.0, 0, 0, 0, 0, 0]))
    assert idx.tolist() == [[0, 1]]
    idx, w = ref.route(np.full((1, 6), -np.inf), None, 6, 0, 2)
    assert idx.tolist() == [[-1, -1]] and w.tolist() == [[0.0, 0.0]]


def test_routed_layer_refusals(pmpe):
    """A given route needs both of its arrays, and no control."""
    from paper_2608_06690_gb300.inputs import LayerShape

    class Fake:
        def __init__(self, addr=P):
            self.addr = addr

        def data_ptr(self):
            return self.addr

        def numel(self):
            return 1 << 40

        def element_size(self):
            return 1

    p = Fake()
    W = {n: p for n in ("router_pub", "router_priv", "gate_pub", "up_pub", "down_pub", "gate_priv", "up_priv", "down_priv")}
    shape = LayerShape(64, 256, 128, 8, 4, 0, 2, True)
    fwd, bwd = pmpe._lib.pmpe_moe_forward_routed, pmpe._lib.pmpe_moe_backward_routed
    need = pmpe._lib.pmpe_moe_backward_step_workspace_size(64, 256, 128, 8, 4, 0, 2)

    def d(**over):
        kw = dict(topk_idx=p, topk_w=p)
        kw.update(over)
        return ctypes.byref(pmpe.make_desc(kw.pop("shape", shape), W, p, None, p, kw.pop("workspace", p), **kw))

    def back(desc=None, grads=(P,) * 6, nb=need):
        return bwd(d() if desc is None else desc, *grads, P, nb, None)

    assert fwd(None, None) == pmpe.ERR_INVALID_ARG and bwd(None, P, P, P, P, P, P, P, need, None) == pmpe.ERR_INVALID_ARG
    for bad in (dict(topk_idx=None), dict(topk_w=None), dict(unmasked_control=True)):
        assert fwd(d(**bad), None) == pmpe.ERR_INVALID_ARG, bad
        assert back(d(**bad)) == pmpe.ERR_INVALID_ARG, bad
    assert fwd(d(topk_idx=Fake(P + 4)), None) == pmpe.ERR_UNSUPPORTED_SHAPE
    assert fwd(d(workspace=None), None) == pmpe.ERR_WORKSPACE
    for i in range(6):  # dout, d_w, d_gate, d_up, d_down, d_hidden
        for v in (None, P + 4):
            assert back(grads=tuple(v if j == i else P for j in range(6))) == pmpe.ERR_INVALID_ARG, (i, v)
    assert back(nb=need - 1) == pmpe.ERR_WORKSPACE
    empty = LayerShape(0, 256, 128, 8, 4, 0, 2, True)
    assert fwd(d(shape=empty, topk_idx=None, topk_w=None, workspace=None), None) == pmpe.OK
