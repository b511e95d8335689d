"""Binding over libpmpe.so (the C ABI of include/pmpe.h): ctypes for the layer,
the module _ops for the operators around it.

Argument marshalling only: every step runs in the library's CUDA kernels.  PyTorch supplies device memory and streams.  If the library
has not been built this module raises on import -- there is no fallback.  Where
only _ops is missing (it is compiled against one PyTorch) the layer works, and
the operators raise ImportError when they are called.
"""
from __future__ import annotations

import ctypes
import importlib
import os
from typing import NamedTuple

import numpy as np
import torch

from .inputs import LayerShape

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpmpe.so")
_BUILD = "build it with `python -c 'import __graft_entry__ as g; g.build()'`"

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: {_BUILD}")

_lib = ctypes.CDLL(LIB_PATH)


class _NoOps:
    """In the place of _ops where it cannot be loaded: says so at the first use."""

    def __init__(self, why):
        self.__dict__["why"] = why

    def __getattr__(self, name):
        raise ImportError(f"the operators around the layer need {os.path.join(_HERE, '_ops.so')} ({self.why}): {_BUILD}")


def _load_ops():
    try:
        ops = importlib.import_module("._ops", __package__)
    except ImportError as e:
        return _NoOps(e)
    built_for = getattr(ops, "built_for", "of another version")
    if built_for != torch.__version__:
        return _NoOps(f"built for PyTorch {built_for}, this is {torch.__version__}")
    return ops


_ops = _load_ops()

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED_SHAPE = -2
ERR_WORKSPACE = -3
ERR_CUDA = -4
ERR_TIMEOUT = -5
ERR_DEVICE_STATUS = -6

STATUS_DISPATCH_MISMATCH = 0x1
STATUS_PIPELINE_TIMEOUT = 0x2
STATUS_BAD_EXPERT_ID = 0x4

STAGE_ROUTE = 0x01
STAGE_PERMUTE = 0x02
STAGE_GATEUP = 0x04
STAGE_DOWN = 0x08
STAGE_COMBINE = 0x10
STAGE_ALL = 0x1F

# Kernels one full forward launches: the router/top-k (with the policy
# resolve), one persistent launch that derives the dispatch order and runs the
# gate/up GEMM (rows gathered from the hidden states) and the down GEMM, and
# the combine; no memset.  For small experts (H * I < 2^20, the tiny test
# layer) the dispatch is a kernel of its own: 4.  (Where the persistent grid
# cannot be resident at once, the GEMMs take two launches as well.)
KERNELS_PER_FORWARD = 3


def kernels_per_forward(shape) -> int:
    """Kernels of this library one full forward of `shape` launches on a GPU
    where the persistent expert grid is resident at once (the rule the
    library applies when it launches the forward).  At most 128 tokens (H
    up to 2048, pools of at most 256 experts): a kernel clearing the expert
    launch's counters and the expert launch (routing, dispatch order, both
    GEMMs, combine).  Otherwise the router, the expert GEMMs and the
    combine, plus a dispatch kernel unless the expert launch derives the
    dispatch order (experts of at least 2^20 weights a projection)."""
    if shape.T <= 128 and shape.H <= 2048 and max(shape.E_pub, shape.E_priv) <= 256:
        return 2
    return 3 if shape.H * shape.I >= (1 << 20) else 4
# kernels one private-branch backward launches: the dispatched rows of the
# private experts, dout row gather, the dL/da GEMM, the gate/up recompute GEMM
# with the SwiGLU backward, router gradient, router weight-gradient partials
# and their reduction, the expert weight-gradient GEMM
KERNELS_PER_BACKWARD = 8


def kernels_per_backward_private(shape) -> int:
    """Kernels one private-branch backward launches: KERNELS_PER_BACKWARD,
    plus, for the pool softmax, the pool token lists and the logits GEMM."""
    return KERNELS_PER_BACKWARD + (0 if shape.renormalize else 2)


def kernels_per_backward_input(shape) -> int:
    """Kernels one input-gradient backward launches (one less after a forward
    that saved its accumulators: no dispatched rows): the dispatched rows, the
    dout row gather, Z,
    the gate/up recompute with the SwiGLU backward and dA over the routed
    experts (the same three again over the shared experts, if any), the
    router's softmax gradient and the per-token sum; for the pool softmax
    also the pool token lists, the logits GEMM and the router-term GEMM."""
    return 7 + (3 if shape.E_sh > 0 else 0) + (0 if shape.renormalize else 3)


def kernels_per_backward_step(shape) -> int:
    """Kernels one combined backward launches: the dispatched rows, the dout
    row gather, Z, the
    gate/up recompute and dA over the routed experts (the same three over the
    shared experts, if any), the router's dz, its weight-gradient partials
    and their sum, the expert weight-gradient GEMM and the per-token sum; for
    the pool softmax also the pool token lists, the logits GEMM and the
    router-term GEMM."""
    return 9 + (3 if shape.E_sh > 0 else 0) + (0 if shape.renormalize else 3)

EXPORTED = ("pmpe_moe_workspace_size", "pmpe_moe_workspace_layout", "pmpe_audit_words", "pmpe_policy_resolve",
            "pmpe_moe_forward", "pmpe_moe_forward_stages", "pmpe_audit_reset", "pmpe_audit_read",
            "pmpe_status_string", "pmpe_moe_forward_noalloc", "pmpe_selftest_wait_timeout",
            "pmpe_policy_from_requests", "pmpe_moe_backward_workspace_size", "pmpe_moe_backward_private",
            "pmpe_moe_backward_input_workspace_size", "pmpe_moe_backward_input",
            "pmpe_moe_backward_step_workspace_size", "pmpe_moe_backward_step", "pmpe_saved_gu_floats",
            "pmpe_moe_forward_routed", "pmpe_moe_backward_routed",
            "pmpe_rms_norm", "pmpe_rms_norm_backward_workspace_size", "pmpe_rms_norm_backward", "pmpe_route",
            "pmpe_route_backward", "pmpe_clip_workspace_size", "pmpe_clip_grad_norm")

# Bytes of the library's static scratch array used by pmpe_moe_forward_noalloc.
STATIC_SCRATCH_BYTES = 32 << 20

_vp = ctypes.c_void_p


class MoeDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("H", ctypes.c_int), ("I", ctypes.c_int), ("E_pub", ctypes.c_int),
                ("E_priv", ctypes.c_int), ("E_shared", ctypes.c_int), ("k", ctypes.c_int),
                ("renormalize", ctypes.c_int),
                ("hidden", _vp), ("policy", _vp),
                ("w_router_pub", _vp), ("w_router_priv", _vp),
                ("w_gate_pub", _vp), ("w_up_pub", _vp), ("w_down_pub", _vp),
                ("w_gate_priv", _vp), ("w_up_priv", _vp), ("w_down_priv", _vp),
                ("w_gate_sh", _vp), ("w_up_sh", _vp), ("w_down_sh", _vp),
                ("out", _vp), ("topk_idx", _vp), ("topk_w", _vp), ("audit", _vp),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t), ("unmasked_control", ctypes.c_int),
                ("saved_gu", _vp)]


class WorkspaceLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("total", "tau", "counts", "offsets", "topk_idx", "topk_w", "slot_of", "ticket",
                                                "tok_of_slot", "w_of_slot", "router_rows", "a_perm", "act", "y", "act_sh", "y_sh",
                                                "tile_done", "router_lists", "router_meta", "gemm_ready",
                                                "tile_counts")]


_lib.pmpe_rms_norm.restype = ctypes.c_int
_lib.pmpe_rms_norm.argtypes = [_vp, _vp]
_lib.pmpe_rms_norm_backward_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_rms_norm_backward_workspace_size.argtypes = [ctypes.c_int] * 2
_lib.pmpe_rms_norm_backward.restype = ctypes.c_int
_lib.pmpe_rms_norm_backward.argtypes = [_vp, _vp]
_lib.pmpe_route.restype = ctypes.c_int
_lib.pmpe_route.argtypes = [_vp, _vp]
_lib.pmpe_route_backward.restype = ctypes.c_int
_lib.pmpe_route_backward.argtypes = [_vp, _vp, _vp, _vp]
_lib.pmpe_clip_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_clip_workspace_size.argtypes = [ctypes.c_int]
_lib.pmpe_clip_grad_norm.restype = ctypes.c_int
_lib.pmpe_clip_grad_norm.argtypes = [_vp, ctypes.c_int, ctypes.c_float, _vp, _vp, ctypes.c_size_t, _vp]
_lib.pmpe_moe_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_moe_workspace_size.argtypes = [ctypes.c_int] * 7
_lib.pmpe_moe_workspace_layout.restype = ctypes.c_int
_lib.pmpe_moe_workspace_layout.argtypes = [ctypes.c_int] * 7 + [ctypes.POINTER(WorkspaceLayout)]
_lib.pmpe_audit_words.restype = ctypes.c_size_t
_lib.pmpe_audit_words.argtypes = [ctypes.c_int, ctypes.c_int]
_lib.pmpe_policy_resolve.restype = ctypes.c_int
_lib.pmpe_policy_resolve.argtypes = [_vp, ctypes.c_int, _vp, _vp]
_lib.pmpe_moe_forward.restype = ctypes.c_int
_lib.pmpe_moe_forward.argtypes = [ctypes.POINTER(MoeDesc), _vp]
_lib.pmpe_moe_forward_stages.restype = ctypes.c_int
_lib.pmpe_moe_forward_stages.argtypes = [ctypes.POINTER(MoeDesc), ctypes.c_uint, _vp]
_lib.pmpe_moe_forward_noalloc.restype = ctypes.c_int
_lib.pmpe_moe_forward_noalloc.argtypes = [ctypes.POINTER(MoeDesc), _vp]
_lib.pmpe_moe_backward_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_moe_backward_workspace_size.argtypes = [ctypes.c_int] * 7
_lib.pmpe_moe_backward_private.restype = ctypes.c_int
_lib.pmpe_moe_backward_private.argtypes = [ctypes.POINTER(MoeDesc), _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
_lib.pmpe_moe_backward_input_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_moe_backward_input_workspace_size.argtypes = [ctypes.c_int] * 7
_lib.pmpe_moe_backward_input.restype = ctypes.c_int
_lib.pmpe_moe_backward_input.argtypes = [ctypes.POINTER(MoeDesc), _vp, _vp, _vp, ctypes.c_size_t, _vp]
_lib.pmpe_moe_backward_step_workspace_size.restype = ctypes.c_size_t
_lib.pmpe_moe_backward_step_workspace_size.argtypes = [ctypes.c_int] * 7
_lib.pmpe_moe_backward_step.restype = ctypes.c_int
_lib.pmpe_moe_backward_step.argtypes = [ctypes.POINTER(MoeDesc)] + [_vp] * 7 + [ctypes.c_size_t, _vp]
_lib.pmpe_moe_forward_routed.restype = ctypes.c_int
_lib.pmpe_moe_forward_routed.argtypes = [ctypes.POINTER(MoeDesc), _vp]
_lib.pmpe_moe_backward_routed.restype = ctypes.c_int
_lib.pmpe_moe_backward_routed.argtypes = [ctypes.POINTER(MoeDesc)] + [_vp] * 7 + [ctypes.c_size_t, _vp]
_lib.pmpe_saved_gu_floats.restype = ctypes.c_size_t
_lib.pmpe_saved_gu_floats.argtypes = [ctypes.c_int] * 4
_lib.pmpe_policy_from_requests.restype = ctypes.c_int
_lib.pmpe_policy_from_requests.argtypes = [_vp, _vp, ctypes.c_int, ctypes.c_int, _vp, _vp]
_lib.pmpe_selftest_wait_timeout.restype = ctypes.c_int
_lib.pmpe_selftest_wait_timeout.argtypes = [_vp, ctypes.c_int, _vp]
_lib.pmpe_audit_reset.restype = ctypes.c_int
_lib.pmpe_audit_reset.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp]
_lib.pmpe_audit_read.restype = ctypes.c_int
_lib.pmpe_audit_read.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp, _vp, ctypes.c_int]
_lib.pmpe_status_string.restype = ctypes.c_char_p
_lib.pmpe_status_string.argtypes = [ctypes.c_int]


class PmpeError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {status_string(code)} ({code})")
        self.code = code


def status_string(code: int) -> str:
    return _lib.pmpe_status_string(code).decode()


def _check(code: int, what: str):
    if code != OK:
        raise PmpeError(code, what)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def workspace_size(s: LayerShape) -> int:
    return int(_lib.pmpe_moe_workspace_size(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k))


def workspace_layout(s: LayerShape) -> dict:
    L = WorkspaceLayout()
    _check(_lib.pmpe_moe_workspace_layout(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k, ctypes.byref(L)),
           "pmpe_moe_workspace_layout")
    return {n: int(getattr(L, n)) for n, _ in WorkspaceLayout._fields_}


def audit_words(T: int, E: int) -> int:
    return int(_lib.pmpe_audit_words(T, E))


def audit_fields(words: np.ndarray, T: int, E: int) -> dict:
    """Split an audit buffer read back to the host into its named counters."""
    a = np.asarray(words, dtype=np.uint32)
    return dict(status=int(a[0]), shared_rows=int(a[1]), route_count=a[2:2 + E], exec_rows=a[2 + E:2 + 2 * E],
                exec_tiles=a[2 + 2 * E:2 + 3 * E], route_priv_rows=a[2 + 3 * E:2 + 3 * E + T],
                exec_priv_rows=a[2 + 3 * E + T:2 + 3 * E + 2 * T])


def private_gradient_shapes(s: LayerShape) -> dict:
    """Shapes of the gradients the private-branch backward writes: the
    private router and the private experts' gate, up and down weights, the
    only parameters trained (G2, Sec. 2.2).  No public parameter has one."""
    return {"d_router": (s.E_priv, s.H), "d_gate": (s.E_priv, s.I, s.H), "d_up": (s.E_priv, s.I, s.H),
            "d_down": (s.E_priv, s.H, s.I)}


def policy_from_requests(req_policy, cu_seqlens, T: int, out=None, stream=None):
    """Per-token policy bytes (uint8 [T], device) from one byte per request
    and the requests' cumulative token offsets (int32 [n+1], device);
    fail-closed on malformed offsets."""
    if out is None:
        out = torch.empty(T, dtype=torch.uint8, device="cuda")
    n = cu_seqlens.numel() - 1
    _check(_lib.pmpe_policy_from_requests(_ptr(req_policy), _ptr(cu_seqlens), n, T, _ptr(out), _stream(stream)),
           "pmpe_policy_from_requests")
    return out


def policy_resolve(policy, T: int, tau=None, stream=None):
    """tau[t] = (policy[t] == 0x01) on the device; policy None = all DENY."""
    if tau is None:
        tau = torch.empty(T, dtype=torch.uint8, device="cuda")
    _check(_lib.pmpe_policy_resolve(_ptr(policy), T, _ptr(tau), _stream(stream)), "pmpe_policy_resolve")
    return tau


def audit_reset(audit, T: int, E: int, stream=None):
    _check(_lib.pmpe_audit_reset(_ptr(audit), T, E, _stream(stream)), "pmpe_audit_reset")


def audit_read(audit, T: int, E: int, stream=None, timeout_ms: int = 10000, check_status: bool = True) -> dict:
    host = torch.empty(audit_words(T, E), dtype=torch.int32).pin_memory()
    rc = _lib.pmpe_audit_read(_ptr(audit), T, E, ctypes.c_void_p(host.data_ptr()), _stream(stream), timeout_ms)
    if rc == ERR_DEVICE_STATUS and not check_status:
        rc = OK
    _check(rc, "pmpe_audit_read")
    return audit_fields(host.numpy().view(np.uint32).copy(), T, E)


def selftest_wait_timeout(status, limit_us: int, stream=None):
    """Enqueue the bounded-wait self-test: a barrier wait that can never
    complete expires after ``limit_us`` microseconds and ORs
    STATUS_PIPELINE_TIMEOUT into the device word ``status[0]``."""
    _check(_lib.pmpe_selftest_wait_timeout(_ptr(status), int(limit_us), _stream(stream)),
           "pmpe_selftest_wait_timeout")


def make_desc(s: LayerShape, weights: dict, hidden, policy, out, workspace, topk_idx=None, topk_w=None,
              audit=None, unmasked_control: bool = False, saved_gu=None) -> MoeDesc:
    """Fill the C descriptor from torch tensors (device pointers only)."""
    W = weights
    return MoeDesc(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k, int(bool(s.renormalize)),
                   _ptr(hidden), _ptr(policy),
                   _ptr(W["router_pub"]), _ptr(W["router_priv"]),
                   _ptr(W["gate_pub"]), _ptr(W["up_pub"]), _ptr(W["down_pub"]),
                   _ptr(W["gate_priv"]), _ptr(W["up_priv"]), _ptr(W["down_priv"]),
                   _ptr(W.get("gate_sh")), _ptr(W.get("up_sh")), _ptr(W.get("down_sh")),
                   _ptr(out), _ptr(topk_idx), _ptr(topk_w), _ptr(audit),
                   _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                   int(bool(unmasked_control)), _ptr(saved_gu))


def forward_desc(desc: MoeDesc, stages: int = STAGE_ALL, stream=None):
    """Enqueue the layer (or a subset of its stages) for a prepared descriptor."""
    if stages == STAGE_ALL:
        rc = _lib.pmpe_moe_forward(ctypes.byref(desc), _stream(stream))
    else:
        rc = _lib.pmpe_moe_forward_stages(ctypes.byref(desc), stages, _stream(stream))
    _check(rc, "pmpe_moe_forward")


class Workspace:
    """A device scratch buffer that grows on demand; layers that run one after
    another on the same stream can share one."""

    def __init__(self, device="cuda"):
        self.device = torch.device(device)
        self._buf = None

    def get(self, nbytes: int) -> torch.Tensor:
        if self._buf is None or self._buf.numel() < nbytes:
            self._buf = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=self.device)
        return self._buf


class MoeLayer:
    """One policy-masked MoE layer with its weights resident on the GPU and
    a reusable workspace.  ``forward`` enqueues the C-ABI call on the
    current stream and returns the output tensor."""

    def __init__(self, shape: LayerShape, weights: dict, device="cuda", workspace: "Workspace | None" = None):
        self.shape = shape
        self.weights = weights
        self.device = torch.device(device)
        self._ws = workspace if workspace is not None else Workspace(self.device)
        self._bws = None
        self._route_out = (None, None)  # the last forward's caller-owned route outputs
        self._saved_gu = None           # the last forward's saved G | U, when it saved them
        self._saved_buf = None
        self._given = False             # the last forward ran a given route

    def workspace(self, T: int) -> torch.Tensor:
        return self._ws.get(workspace_size(self._shape_T(T)))

    def _shape_T(self, T: int) -> LayerShape:
        s = self.shape
        return LayerShape(T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k, s.renormalize)

    def forward(self, hidden, policy, out=None, topk_idx=None, topk_w=None, audit=None, stages=STAGE_ALL,
                stream=None, unmasked_control: bool = False, save_for_backward: bool = False, route=None):
        """Enqueue the layer on ``stream`` (default: the current stream; the
        caller orders another one's work after what the current stream has).
        ``route``: (idx, w), int32 and FP32 [T, k], as ``Router.route`` gives
        them, in the place of the layer's own router; its backward is
        ``backward_routed``.  A pick outside the token's pool, or of -1, is
        not taken (another expert runs in its place with weight 0, so padding
        should hold finite numbers).
        ``unmasked_control`` runs the paper's soft-router control instead of
        the method: routing over the concatenated pool without the hard mask.
        ``save_for_backward`` also keeps the gate and up accumulators of the
        routed rows and the shared experts (FP32, owned by the layer), which
        the backward calls after this forward then read instead of
        recomputing them."""
        T = hidden.shape[0]
        s = self._shape_T(T)
        assert hidden.is_contiguous() and hidden.dtype == torch.bfloat16 and hidden.shape == (T, s.H)
        if policy is not None:
            assert policy.dtype == torch.uint8 and policy.numel() == T and policy.is_contiguous()
        dev = hidden.get_device()
        if dev < 0 or policy is not None and policy.get_device() != dev or out is not None and out.get_device() != dev or \
                topk_idx is not None and topk_idx.get_device() != dev or topk_w is not None and topk_w.get_device() != dev or \
                audit is not None and audit.get_device() != dev:
            _bad("MoeLayer.forward: CUDA tensors of one device are wanted")
        if out is None:
            out = torch.empty_like(hidden)
        saved = None
        if save_for_backward:
            n = _lib.pmpe_saved_gu_floats(T, s.I, s.E_sh, s.k)
            if self._saved_buf is None or self._saved_buf.numel() < n:
                self._saved_buf = torch.empty(max(n, 4), dtype=torch.float32, device=hidden.device)
            saved = self._saved_buf
        if route is not None:
            if topk_idx is not None or topk_w is not None or unmasked_control or stages != STAGE_ALL:
                _bad("MoeLayer.forward: a given route takes the place of the route log, the control and the stages")
            topk_idx, topk_w = route
            for v, dt in ((topk_idx, torch.int32), (topk_w, torch.float32)):
                if not _matrix(v, T, s.k, dev, dt):
                    _bad("MoeLayer.forward: route is (idx, w), int32 and FP32 [T, k] on the layer's device")
        ws = self.workspace(T)
        desc = make_desc(s, self.weights, hidden, policy, out, ws, topk_idx, topk_w, audit, unmasked_control, saved)
        if route is not None:
            _check(_lib.pmpe_moe_forward_routed(ctypes.byref(desc), _stream(stream)), "pmpe_moe_forward_routed")
        else:
            forward_desc(desc, stages, stream)
        if stream is not None:
            self._hold(stream, hidden, policy, out, ws, topk_idx, topk_w, audit, saved)
        self._given = route is not None
        self._route_out = (topk_idx, topk_w)
        self._saved_gu = saved
        return out

    @staticmethod
    def _hold(stream, *tensors):
        """The memory of a call on a stream of its own (arguments, results and
        scratch, from the current stream's pool) is not handed out again before
        that stream is done with it."""
        if stream.cuda_stream != torch._C._cuda_getCurrentRawStream(stream.device_index):
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)

    @staticmethod
    def _rows(hidden, dout, what: str):
        """A backward's hidden states are the forward's: BF16 rows as dout's."""
        if not hidden.is_cuda or hidden.dtype != torch.bfloat16 or not hidden.is_contiguous() or hidden.shape != dout.shape or \
                hidden.device != dout.device:
            _bad(f"MoeLayer.{what}: hidden is the forward's, BF16 [T, H] without gaps on dout's CUDA device")

    def _own_route(self, what: str):
        if self._given:
            _bad(f"MoeLayer.{what}: the last forward ran a given route: backward_routed is its backward")

    def backward_routed(self, hidden, policy, dout, stream=None):
        """Backward of the forward just run with a given route, the same hidden
        states and policy on the same stream: (grads, d_hidden, d_w).  grads:
        the private experts' d_gate, d_up and d_down (FP32); d_hidden: that of
        the hidden states through the experts (FP32, without the caller's
        router's part); d_w: that of the route's weights (FP32 [T, k]), for
        ``Router.backward``."""
        T = hidden.shape[0]
        s = self._shape_T(T)
        if not self._given:
            _bad("MoeLayer.backward_routed: the last forward ran the layer's own router")
        if T != self._route_out[0].shape[0]:
            _bad("MoeLayer.backward_routed: the last forward ran another number of tokens")
        assert dout.is_contiguous() and dout.dtype == torch.bfloat16 and dout.shape == (T, s.H)
        self._rows(hidden, dout, "backward_routed")
        dev = hidden.device
        g = {n: torch.empty(shp, dtype=torch.float32, device=dev) for n, shp in private_gradient_shapes(s).items()
             if n != "d_router"}
        d_hidden = torch.empty((T, s.H), dtype=torch.float32, device=dev)
        d_w = torch.empty((T, s.k), dtype=torch.float32, device=dev)
        nb = _lib.pmpe_moe_backward_step_workspace_size(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k)
        if nb == 0:
            raise PmpeError(ERR_UNSUPPORTED_SHAPE, "pmpe_moe_backward_step_workspace_size")
        if self._bws is None or self._bws.numel() < nb:
            self._bws = torch.empty(nb, dtype=torch.uint8, device=dev)
        bws, ws = self._bws, self.workspace(T)
        topk_idx, topk_w = self._route_out
        desc = make_desc(s, self.weights, hidden, policy, dout, ws, topk_idx, topk_w,
                         saved_gu=self._saved_gu)
        _check(_lib.pmpe_moe_backward_routed(ctypes.byref(desc), _ptr(dout), _ptr(d_w), _ptr(g["d_gate"]), _ptr(g["d_up"]),
                                             _ptr(g["d_down"]), _ptr(d_hidden), _ptr(bws), bws.numel(), _stream(stream)),
               "pmpe_moe_backward_routed")
        if stream is not None:
            self._hold(stream, hidden, policy, dout, topk_idx, topk_w, self._saved_gu, ws, bws, *g.values(), d_hidden, d_w)
        return g, d_hidden, d_w

    def backward_private(self, hidden, policy, dout, topk_idx=None, topk_w=None, stream=None) -> dict:
        """Gradients of sum(dout * out) with respect to the private parameters
        (router, gate, up, down; FP32) for the forward just run with the same
        hidden states and policy on the same stream (its workspace holds the
        route and the activations; the route outputs default to those that
        forward wrote).  The public parameters get none."""
        self._own_route("backward_private")
        T = hidden.shape[0]
        s = self._shape_T(T)
        assert dout.is_contiguous() and dout.dtype == torch.bfloat16 and dout.shape == (T, s.H)
        self._rows(hidden, dout, "backward_private")
        dev = hidden.device
        g = {n: torch.empty(shp, dtype=torch.float32, device=dev) for n, shp in private_gradient_shapes(s).items()}
        nb = _lib.pmpe_moe_backward_workspace_size(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k)
        if nb == 0:
            raise PmpeError(ERR_UNSUPPORTED_SHAPE, "pmpe_moe_backward_workspace_size")
        if self._bws is None or self._bws.numel() < nb:
            self._bws = torch.empty(nb, dtype=torch.uint8, device=dev)
        bws, ws = self._bws, self.workspace(T)
        if topk_idx is None and topk_w is None:
            topk_idx, topk_w = self._route_out
        # the descriptor's output pointer is never written by the backward
        desc = make_desc(s, self.weights, hidden, policy, dout, ws, topk_idx, topk_w,
                         saved_gu=self._saved_gu)
        _check(_lib.pmpe_moe_backward_private(ctypes.byref(desc), _ptr(dout), _ptr(g["d_router"]), _ptr(g["d_gate"]),
                                              _ptr(g["d_up"]), _ptr(g["d_down"]), _ptr(bws), bws.numel(),
                                              _stream(stream)), "pmpe_moe_backward_private")
        if stream is not None:
            self._hold(stream, hidden, policy, dout, topk_idx, topk_w, self._saved_gu, ws, bws, *g.values())
        return g

    def backward(self, hidden, policy, dout, topk_idx=None, topk_w=None, stream=None):
        """Both backward results of the forward just run with the same hidden
        states and policy on the same stream, in one pass: the private
        parameters' gradients (as backward_private) and the gradient of the
        hidden states (as backward_input), each bitwise as those calls give."""
        self._own_route("backward")
        T = hidden.shape[0]
        s = self._shape_T(T)
        assert dout.is_contiguous() and dout.dtype == torch.bfloat16 and dout.shape == (T, s.H)
        self._rows(hidden, dout, "backward")
        dev = hidden.device
        g = {n: torch.empty(shp, dtype=torch.float32, device=dev) for n, shp in private_gradient_shapes(s).items()}
        d_hidden = torch.empty((T, s.H), dtype=torch.float32, device=dev)
        nb = _lib.pmpe_moe_backward_step_workspace_size(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k)
        if nb == 0:
            raise PmpeError(ERR_UNSUPPORTED_SHAPE, "pmpe_moe_backward_step_workspace_size")
        if self._bws is None or self._bws.numel() < nb:
            self._bws = torch.empty(nb, dtype=torch.uint8, device=dev)
        bws, ws = self._bws, self.workspace(T)
        if topk_idx is None and topk_w is None:
            topk_idx, topk_w = self._route_out
        desc = make_desc(s, self.weights, hidden, policy, dout, ws, topk_idx, topk_w,
                         saved_gu=self._saved_gu)
        _check(_lib.pmpe_moe_backward_step(ctypes.byref(desc), _ptr(dout), _ptr(g["d_router"]), _ptr(g["d_gate"]),
                                           _ptr(g["d_up"]), _ptr(g["d_down"]), _ptr(d_hidden), _ptr(bws),
                                           bws.numel(), _stream(stream)), "pmpe_moe_backward_step")
        if stream is not None:
            self._hold(stream, hidden, policy, dout, topk_idx, topk_w, self._saved_gu, ws, bws, *g.values(), d_hidden)
        return g, d_hidden

    def backward_input(self, hidden, policy, dout, topk_idx=None, topk_w=None, stream=None) -> torch.Tensor:
        """Gradient of sum(dout * out) with respect to the hidden states [T, H]
        (FP32), through the frozen layer, for the forward just run with the
        same hidden states and policy on the same stream: the routed experts
        of each token's pool, the shared experts and that pool's router."""
        self._own_route("backward_input")
        T = hidden.shape[0]
        s = self._shape_T(T)
        assert dout.is_contiguous() and dout.dtype == torch.bfloat16 and dout.shape == (T, s.H)
        self._rows(hidden, dout, "backward_input")
        dev = hidden.device
        d_hidden = torch.empty((T, s.H), dtype=torch.float32, device=dev)
        nb = _lib.pmpe_moe_backward_input_workspace_size(s.T, s.H, s.I, s.E_pub, s.E_priv, s.E_sh, s.k)
        if nb == 0:
            raise PmpeError(ERR_UNSUPPORTED_SHAPE, "pmpe_moe_backward_input_workspace_size")
        if self._bws is None or self._bws.numel() < nb:
            self._bws = torch.empty(nb, dtype=torch.uint8, device=dev)
        bws, ws = self._bws, self.workspace(T)
        if topk_idx is None and topk_w is None:
            topk_idx, topk_w = self._route_out
        desc = make_desc(s, self.weights, hidden, policy, dout, ws, topk_idx, topk_w,
                         saved_gu=self._saved_gu)
        _check(_lib.pmpe_moe_backward_input(ctypes.byref(desc), _ptr(dout), _ptr(d_hidden), _ptr(bws), bws.numel(),
                                            _stream(stream)), "pmpe_moe_backward_input")
        if stream is not None:
            self._hold(stream, hidden, policy, dout, topk_idx, topk_w, self._saved_gu, ws, bws, d_hidden)
        return d_hidden


# ------------------------------------------- operators around the layer
#
# Checks, outputs and launches are in _ops (csrc/bind_ops.cpp): a call's host
# time counts as much as its kernel's at decode sizes.
#
# Neither these functions nor MoeLayer record anything for autograd: what they
# return has no history, whatever the arguments require, and the backward
# functions are the caller's to call.  What the functions here write to in place
# (h_out, load, clipped gradients and out) counts up its version, so that
# autograd refuses a backward that had saved it.

QUANT_BLOCK = 128  # columns that share a scale with quant="block"


def _bad(what: str):
    raise PmpeError(ERR_INVALID_ARG, what)


def _on(stream, fn, t, *args):
    """The call on ``stream``: outputs and scratch are allocated there, so that
    the caching allocator reuses them in order, and the arguments' memory is
    not reused before the stream is done with it.  (The caller orders the
    streams' work.)"""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _bad(f"{fn.__name__}: CUDA tensors are wanted")
    if stream.device != t.device:
        _bad(f"{fn.__name__}: the stream is of another device than the tensors")
    with torch.cuda.stream(stream):
        result = fn(*args)
    for a in args:
        for v in a if isinstance(a, (list, tuple)) else (a,):
            if isinstance(v, torch.Tensor):
                v.record_stream(stream)
    return result


def _matrix(t, rows: int, cols: int, dev: int, dtype) -> bool:
    return t.dtype is dtype and t.get_device() == dev and t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols and \
        t.is_contiguous()


class RmsNorm(NamedTuple):
    y: torch.Tensor             # [T, H], the input's type or float8_e4m3fn
    scale: torch.Tensor | None  # FP32 [T, ceil(H / 128)] ("block") or [T, 1] ("row") of an 8-bit y
    h: torch.Tensor             # [T, H], x + residual; x itself without a residual
    rstd: torch.Tensor          # FP32 [T], for the backward


def rms_norm(x, weight, residual=None, eps: float = 1e-6, quant=None, h_out=None, stream=None) -> RmsNorm:
    """Root-mean-square norm of ``h = x + residual`` (x without a residual),
    times ``weight``.

    x and residual: [T, H] of one type (FP32, BF16 or FP16), rows of any pitch;
    weight: [H] of that type or FP32.  h is rounded to the type, and the norm
    is that of the rounded h.  ``quant``: None for y in x's type; "block" or
    "row" for y in e4m3 with an FP32 scale per row and 128 columns or per row
    (y stands for ``y.float() * scale``).  ``h_out``: where h goes (may be
    ``residual`` or ``x``; anything else that shares their memory is refused).  ``stream``: the stream to run on (default: the
    current one).  H up to 16384, eps at least 1e-20."""
    if stream is not None:
        return _on(stream, rms_norm, x, x, weight, residual, eps, quant, h_out)
    return _ops.rms_norm(x, weight, residual, eps, quant, h_out)


def rms_norm_backward(dy, h, weight, rstd, d_h=None, dx_dtype=None, need_dw: bool = True, stream=None):
    """(dx, dw) of ``rms_norm``: dx is the gradient of x and of the residual
    alike, dw that of the weight (FP32; None unless ``need_dw``).

    dy: [T, H] of h's type or FP32; h and rstd as the forward returned them;
    d_h: the gradient that reaches h itself, of dx's type.  ``dx_dtype``: h's
    type (default) or FP32.  Matrices without gaps.  An 8-bit y passes its
    gradient as the identity."""
    if stream is not None:
        return _on(stream, rms_norm_backward, h, dy, h, weight, rstd, d_h, dx_dtype, need_dw)
    return _ops.rms_norm_backward(dy, h, weight, rstd, d_h, dx_dtype, need_dw)


class Router:
    """Routing from given logits for models whose router is not the layer's
    own softmax: softmax or sigmoid scores, a bias for balance, group limits,
    top-k and weights, each token inside the pool its policy byte selects.
    ``MoeLayer.forward(route=...)`` runs the experts with the result.

    score: "softmax" (over the token's pool) or "sigmoid".  groups,
    groups_priv: (groups of the pool, groups kept); group_score: "max" or
    "top2", the sum of a group's two best.  E_priv = 0: one pool, no policy."""

    def __init__(self, E_pub: int, E_priv: int, k: int, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                 groups=(1, 1), groups_priv=(1, 1), group_score: str = "max"):
        if score not in ("softmax", "sigmoid"):
            _bad('Router: score is "softmax" or "sigmoid"')
        if group_score not in ("max", "top2"):
            _bad('Router: group_score is "max" or "top2"')
        self.E_pub, self.E_priv, self.k, self.E = int(E_pub), int(E_priv), int(k), int(E_pub) + int(E_priv)
        # refuses what the library would refuse, before the first call
        self._desc = _ops.router(self.E_pub, self.E_priv, self.k, int(score == "sigmoid"), int(bool(renormalize)), int(groups[0]),
                                 int(groups[1]), int(groups_priv[0]), int(groups_priv[1]), int(group_score == "top2"), float(scale))

    def route(self, logits, policy=None, bias=None, load=None, stream=None):
        """(idx, w): the k chosen experts of each token (int32 [T, k], global
        ids, best first, -1 where there is none) and their weights (FP32).

        logits: [T, E_pub + E_priv], rows of any pitch; -inf (or NaN) takes an
        expert out of a token's choice.  policy: uint8 [T], 0x01 for the
        private pool (None: all public).  bias: FP32 [E], added to the scores
        for the choice alone.  load: int32 [E], to which the tokens of each
        expert are added (for the bias's update)."""
        if stream is not None:
            return _on(stream, self.route, logits, logits, policy, bias, load)
        return _ops.route(self._desc, logits, policy, bias, load)

    def backward(self, logits, policy, idx, dw, stream=None):
        """The gradient of the logits ([T, E], their type) from that of the
        weights (FP32 [T, k]) for the selection ``idx``."""
        if stream is not None:
            return _on(stream, self.backward, logits, logits, policy, idx, dw)
        return _ops.route_backward(self._desc, logits, policy, idx, dw)


def clip_grad_norm(grads, max_norm: float, out=None, stream=None):
    """The global norm of ``grads`` (a list of tensors, or a dict of them as the
    backward returns it), as an FP32 device scalar; the gradients are scaled in
    place by min(1, max_norm / (norm + 1e-6)), or into the tensors of ``out``.

    FP32, BF16 and FP16 tensors may be mixed; each lies in memory without gaps.
    max_norm = inf: the norm alone.  A norm that is not finite as FP32
    clips nothing.  No tensor may share memory with another."""
    if isinstance(grads, dict):
        if out is not None:
            if not isinstance(out, dict) or out.keys() != grads.keys():
                _bad("clip_grad_norm: out is as grads")
            out = [out[n] for n in grads]
        grads = list(grads.values())
    if stream is not None:
        return _on(stream, clip_grad_norm, grads[0] if len(grads) else None, grads, max_norm, out)
    return _ops.clip_grad_norm(grads, max_norm, out)


if not isinstance(_ops, _NoOps):
    _ops.setup(PmpeError, RmsNorm, *(ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in (
        "pmpe_rms_norm", "pmpe_rms_norm_backward_workspace_size", "pmpe_rms_norm_backward", "pmpe_route", "pmpe_route_backward",
        "pmpe_clip_workspace_size", "pmpe_clip_grad_norm")))
