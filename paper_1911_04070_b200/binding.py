"""Thin Python binding of the C ABI in include/bpt.h (argument marshalling only).

PyTorch supplies device memory and the current stream; every step of the path
runs in the CUDA kernels of libbpt.so.  There is no CPU fallback: a missing
library or a failing call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbpt.so")
CHECK_LIB_PATH = os.path.join(_HERE, "libbpt_check.so")   # the build with index checks; set LIB_PATH to it before the first call

BPT_BIDIR, BPT_LEFT_ONLY, BPT_MODE_PAD, BPT_MODE_ALG1 = 0, 1, 0, 2
BPT_F32, BPT_BF16 = 0, 1
BPT_PATH_AUTO, BPT_PATH_MMA, BPT_PATH_TC5 = 0, 1, 2
NORM_KINDS = {None: 0, "layer": 1, "rms": 2}   # BPT_NORM_*
ACTIVATIONS = {"relu": 0, "silu": 1, "gelu": 2}        # BPT_ACT_*

EXPORTS = ("bpt_graph_dims_query", "bpt_build_graph", "bpt_attn_workspace_bytes", "bpt_attn_fwd",
           "bpt_attn_bwd", "bpt_status_str", "bpt_trace_begin", "bpt_trace_end",
           "bpt_static_scratch_bytes", "bpt_attn_bwd_static_scratch", "bpt_attn_fwd_varlen", "bpt_attn_bwd_varlen",
           "bpt_attn_fwd_ex", "bpt_attn_bwd_ex", "bpt_attn_fwd_rows", "bpt_attn_bwd_min_workspace_bytes", "bpt_check",
           "bpt_selftest_wait_timeout", "bpt_debug_bounds", "bpt_out_proj_norm", "bpt_res_norm_fwd",
           "bpt_res_norm_bwd_workspace_bytes", "bpt_res_norm_bwd", "bpt_gated_ff_workspace_bytes", "bpt_gated_ff_fwd", "bpt_gated_ff_bwd",
           "bpt_gated_ff_few_rows", "bpt_check_device")


class BptError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_str(status), status))


class GraphDims(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("k", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("n_levels", ctypes.c_int32), ("n_nodes", ctypes.c_int32), ("n_rel", ctypes.c_int32),
                ("n_edges", ctypes.c_int64), ("build_workspace_bytes", ctypes.c_size_t)]


class GraphStruct(ctypes.Structure):
    _fields_ = [("row_ptr", ctypes.c_void_p), ("col", ctypes.c_void_p), ("rel", ctypes.c_void_p),
                ("t_ptr", ctypes.c_void_p), ("t_dst", ctypes.c_void_p), ("t_eid", ctypes.c_void_p),
                ("dims", GraphDims)]


class AttnOptions(ctypes.Structure):
    _fields_ = [("lengths", ctypes.c_void_p), ("dropout_p", ctypes.c_float), ("dropout_seed", ctypes.c_uint64),
                ("path", ctypes.c_uint32)]


class ResNormArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("gate_groups", ctypes.c_int64), ("D", ctypes.c_int32), ("dtype", ctypes.c_int),
                ("param_dtype", ctypes.c_int), ("gate_dtype", ctypes.c_int), ("norm", ctypes.c_int32), ("post_norm", ctypes.c_int32),
                ("alpha", ctypes.c_float), ("eps", ctypes.c_float), ("h", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("post_weight", ctypes.c_void_p),
                ("post_bias", ctypes.c_void_p), ("gate", ctypes.c_void_p)]


# When set, the autograd wrappers in layer.py ask bpt_check after every attention and gated feed-forward call (a stream
# synchronisation per call): for debugging.  Training loops ask bpt_check_device once per step, which covers the gated
# feed-forward calls, backward passes among them.
CHECK_DEVICE_STATUS = False

_lib = None


def load_library() -> ctypes.CDLL:
    """Load libbpt.so from the package directory; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libbpt.so is missing: run `python -m paper_1911_04070_b200.build` "
                              "(there is no fallback implementation)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, u32, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_float
        lib.bpt_graph_dims_query.restype = ctypes.c_int
        lib.bpt_graph_dims_query.argtypes = [i32, i32, u32, ctypes.POINTER(GraphDims)]
        lib.bpt_build_graph.restype = ctypes.c_int
        lib.bpt_build_graph.argtypes = [ctypes.POINTER(GraphDims), vp, vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(GraphStruct)]
        lib.bpt_attn_workspace_bytes.restype = sz
        lib.bpt_attn_workspace_bytes.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, ctypes.c_int]
        lib.bpt_attn_bwd_min_workspace_bytes.restype = sz
        lib.bpt_attn_bwd_min_workspace_bytes.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int]
        lib.bpt_check.restype = ctypes.c_int
        lib.bpt_check.argtypes = [vp, vp]
        lib.bpt_check_device.restype = ctypes.c_int
        lib.bpt_check_device.argtypes = [vp]
        lib.bpt_selftest_wait_timeout.restype = ctypes.c_int
        lib.bpt_selftest_wait_timeout.argtypes = [vp, ctypes.c_int64, i32, vp]
        lib.bpt_out_proj_norm.restype = ctypes.c_int
        lib.bpt_out_proj_norm.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int64, i32, f32, vp, vp]
        rn = ctypes.POINTER(ResNormArgs)
        lib.bpt_res_norm_fwd.restype = ctypes.c_int
        lib.bpt_res_norm_fwd.argtypes = [rn, vp, vp, vp, vp]
        lib.bpt_res_norm_bwd_workspace_bytes.restype = sz
        lib.bpt_res_norm_bwd_workspace_bytes.argtypes = [rn]
        lib.bpt_res_norm_bwd.restype = ctypes.c_int
        lib.bpt_res_norm_bwd.argtypes = [rn, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        i64 = ctypes.c_int64
        lib.bpt_gated_ff_few_rows.restype = i32
        lib.bpt_gated_ff_few_rows.argtypes = [i64, i32, i32]
        lib.bpt_gated_ff_workspace_bytes.restype = sz
        lib.bpt_gated_ff_workspace_bytes.argtypes = [i64, i32, i32, ctypes.c_int]
        lib.bpt_gated_ff_fwd.restype = ctypes.c_int
        lib.bpt_gated_ff_fwd.argtypes = [vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, sz, vp]
        lib.bpt_gated_ff_bwd.restype = ctypes.c_int
        lib.bpt_gated_ff_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, sz, vp]
        lib.bpt_debug_bounds.restype = ctypes.c_int
        lib.bpt_debug_bounds.argtypes = [ctypes.POINTER(ctypes.c_uint32), vp]
        lib.bpt_attn_fwd.restype = ctypes.c_int
        lib.bpt_attn_fwd.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                     vp, vp, vp, sz, vp]
        lib.bpt_attn_bwd.restype = ctypes.c_int
        lib.bpt_attn_bwd.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                     vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.bpt_attn_fwd_varlen.restype = ctypes.c_int
        lib.bpt_attn_fwd_varlen.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                            vp, vp, vp, vp, sz, vp]
        lib.bpt_attn_bwd_varlen.restype = ctypes.c_int
        lib.bpt_attn_bwd_varlen.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                            vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.bpt_attn_fwd_ex.restype = ctypes.c_int
        lib.bpt_attn_fwd_ex.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                        ctypes.POINTER(AttnOptions), vp, vp, vp, sz, vp]
        lib.bpt_attn_bwd_ex.restype = ctypes.c_int
        lib.bpt_attn_bwd_ex.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                        ctypes.POINTER(AttnOptions), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.bpt_attn_fwd_rows.restype = ctypes.c_int
        lib.bpt_attn_fwd_rows.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp, f32,
                                          ctypes.POINTER(AttnOptions), vp, i32, vp, vp, vp]
        lib.bpt_static_scratch_bytes.restype = sz
        lib.bpt_static_scratch_bytes.argtypes = []
        lib.bpt_attn_bwd_static_scratch.restype = ctypes.c_int
        lib.bpt_attn_bwd_static_scratch.argtypes = [ctypes.POINTER(GraphStruct), i32, i32, i32, ctypes.c_int, vp, vp, vp, vp,
                                                    f32, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.bpt_trace_begin.restype = ctypes.c_int
        lib.bpt_trace_begin.argtypes = [i32, vp]
        lib.bpt_trace_end.restype = ctypes.c_int
        lib.bpt_trace_end.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(f32), ctypes.POINTER(ctypes.c_char_p), i32]
        lib.bpt_status_str.restype = ctypes.c_char_p
        lib.bpt_status_str.argtypes = [ctypes.c_int]
        _lib = lib
    return _lib


_native = None


def load_native():
    """The C++ autograd functions over the library (csrc_torch/autograd.cpp), bound to the loaded library; raises if not built."""
    global _native
    if _native is None:
        lib = load_library()
        from . import build
        have, want = build.built_for(build.LIB_TORCH), build.torch_key()
        if have != want:        # not loaded: a binary of another PyTorch may load and misread its structures
            raise ImportError("_bpt_torch.so is %s, not for %s: run `python -m paper_1911_04070_b200.build` (there is no fallback "
                              "implementation)" % ("missing or of an earlier build" if have is None else "built for " + have, want))
        from . import _bpt_torch as native
        native.bind_library([ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in (
            "bpt_res_norm_fwd", "bpt_res_norm_bwd_workspace_bytes", "bpt_res_norm_bwd", "bpt_gated_ff_few_rows",
            "bpt_gated_ff_workspace_bytes", "bpt_gated_ff_fwd", "bpt_gated_ff_bwd")])
        _native = native
    return _native


def status_str(status: int) -> str:
    return load_library().bpt_status_str(int(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise BptError(status, where)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# The position-wise operators are called for single tokens, where what surrounds the library call is most of the time: the
# current stream and device are read through torch's C functions (0.1 us against 3.2 and 1.5 us), and the device is
# switched only where it is another one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_SAME_DEVICE = contextlib.nullcontext()


def _on_device(index: int):
    return _SAME_DEVICE if _current_device() == index else torch.cuda.device(index)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return BPT_F32
    if t.dtype == torch.bfloat16:
        return BPT_BF16
    raise TypeError("only float32 and bfloat16 tensors are supported, got %s" % t.dtype)


def bpt_graph_dims_query(n: int, k: int, flags: int = 0) -> GraphDims:
    dims = GraphDims()
    _check(load_library().bpt_graph_dims_query(n, k, flags, ctypes.byref(dims)), "bpt_graph_dims_query")
    return dims


class Graph:
    """Device-resident BPT graph: owns the index tensors the C struct points at."""

    def __init__(self, dims: GraphDims, device, with_transpose: bool):
        E, N = dims.n_edges, dims.n_nodes
        i32 = dict(dtype=torch.int32, device=device)
        self.dims = dims
        self.row_ptr = torch.empty(N + 1, **i32)
        self.col = torch.empty(E, **i32)
        self.rel = torch.empty(E, **i32)
        self.t_ptr = torch.empty(N + 1, **i32) if with_transpose else None
        self.t_dst = torch.empty(E, **i32) if with_transpose else None
        self.t_eid = torch.empty(E, **i32) if with_transpose else None
        self.c = GraphStruct()

    n = property(lambda s: s.dims.n)
    k = property(lambda s: s.dims.k)
    n_nodes = property(lambda s: s.dims.n_nodes)
    n_edges = property(lambda s: s.dims.n_edges)
    n_rel = property(lambda s: s.dims.n_rel)


def bpt_build_graph(n: int, k: int, flags: int = 0, device="cuda", with_transpose: bool = True) -> Graph:
    """Builds the graph of (n, k, flags) on `device` with the library's kernels."""
    lib = load_library()
    dims = bpt_graph_dims_query(n, k, flags)
    device = torch.device(device)
    with torch.cuda.device(device):
        g = Graph(dims, device, with_transpose)
        ws = torch.empty(max(int(dims.build_workspace_bytes), 1), dtype=torch.uint8, device=device)
        _check(lib.bpt_build_graph(ctypes.byref(dims), _ptr(g.row_ptr), _ptr(g.col), _ptr(g.rel),
                                   _ptr(g.t_ptr), _ptr(g.t_dst), _ptr(g.t_eid), _ptr(ws), _stream(),
                                   ctypes.byref(g.c)), "bpt_build_graph")
        g._build_ws = ws  # keep alive until the stream has run the build
    return g


def bpt_attn_workspace_bytes(g: Graph, B: int, H: int, d: int, dtype_code: int, backward: bool) -> int:
    return int(load_library().bpt_attn_workspace_bytes(ctypes.byref(g.c), B, H, d, dtype_code, int(backward)))


def bpt_attn_bwd_min_workspace_bytes(g: Graph, B: int, H: int, d: int, dtype_code: int) -> int:
    """The smallest workspace bpt_attn_bwd accepts (it then works through the problem in more passes)."""
    return int(load_library().bpt_attn_bwd_min_workspace_bytes(ctypes.byref(g.c), B, H, d, dtype_code))


def bpt_check(workspace) -> int:
    """Waits for the current stream and returns the status the last attention call left in `workspace`
    (0 = ok, 5 = a bounded device-side wait expired: that call's results are invalid)."""
    dev = torch.cuda.current_device() if workspace is None else workspace.device
    with torch.cuda.device(dev):
        return int(load_library().bpt_check(_ptr(workspace), _stream()))


def bpt_check_device(device=None) -> int:
    """Waits for the current stream of `device` (the current one) and returns 0, or 5 when a bounded device-side wait of a gated
    feed-forward call, forward or backward, expired there since the last such question: what was computed since is invalid."""
    with torch.cuda.device(device):
        return int(load_library().bpt_check_device(_stream()))


def bpt_out_proj_norm(a, w_o, h, gamma, beta, eps: float = 1e-5, z=None, workspace=None):
    """z = LayerNorm(h + a @ w_o.T) * gamma + beta over the last axis, in one kernel (bf16 in and out, fp32
    accumulation and statistics).  a, h: [..., D] bfloat16 contiguous; w_o: [D, D] bfloat16; gamma, beta: [D]
    float32; D in (128, 256, 512).  Forward only."""
    D = a.shape[-1]
    for t in (a, h):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.shape != a.shape or not t.is_cuda:
            raise ValueError("a and h must be contiguous bfloat16 CUDA tensors of one shape")
    if w_o.dtype != torch.bfloat16 or w_o.shape != (D, D) or not w_o.is_contiguous():
        raise ValueError("w_o must be a contiguous bfloat16 [D, D] tensor")
    for t in (gamma, beta):
        if t.dtype != torch.float32 or t.shape != (D,) or not t.is_contiguous():
            raise ValueError("gamma and beta must be contiguous float32 [D] tensors")
    rows = a.numel() // D
    with torch.cuda.device(a.device):
        z = torch.empty_like(a) if z is None else z
        _check(load_library().bpt_out_proj_norm(_ptr(a), _ptr(w_o), _ptr(h), _ptr(gamma), _ptr(beta), _ptr(z), rows, D, float(eps),
                                                _ptr(workspace), _stream()), "bpt_out_proj_norm")
    return z


def bpt_gated_ff_workspace_bytes(rows: int, D: int, F: int, backward: bool) -> int:
    return int(load_library().bpt_gated_ff_workspace_bytes(rows, D, F, int(backward)))


def _check_gated_ff(x, w_gate, w_up, w_down, act, *like_x):
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s" % ", ".join(map(repr, ACTIVATIONS)))
    dt, dev, shape = x.dtype, x.get_device(), x.shape
    if dt != torch.bfloat16:
        raise TypeError("only bfloat16 tensors are supported, got %s" % dt)
    if dev < 0 or not shape or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor [..., D]")
    D = shape[-1]
    F = w_gate.shape[0] if w_gate.dim() == 2 else 0
    for t, want in ((w_gate, (F, D)), (w_up, (F, D)), (w_down, (D, F))):
        if t.shape != want or t.dtype != dt or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("w_gate and w_up must be [F, D], w_down [D, F], contiguous, with the dtype and device of x")
    for t in like_x:
        if t is not None and (t.shape != shape or t.dtype != dt or t.get_device() != dev or not t.is_contiguous()):
            raise ValueError("y, dy and dx must be contiguous and share shape, dtype and device with x")
    return x.numel() // D if D else 0, D, F, dev


def _scratch(workspace, size, like):
    if workspace is None:
        return like.new_empty(size, dtype=torch.uint8)
    if workspace.dtype != torch.uint8 or workspace.get_device() != like.get_device() or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the inputs")
    return workspace


def bpt_gated_ff_fwd(x, w_gate, w_up, w_down, act: str = "silu", y=None, workspace=None):
    """y = (act(x @ w_gate.T) * (x @ w_up.T)) @ w_down.T over the last axis: both projections, activation and product in
    one kernel, the second product in another.  x: [..., D] bfloat16 contiguous; w_gate, w_up: [F, D]; w_down: [D, F]; D and F
    multiples of 8.  The call's status block stays reachable as `y._bpt_workspace` for bpt_check (the workspace does not);
    None for the few rows of a decoding step, whose kernels wait for nothing."""
    rows, D, F, dev = _check_gated_ff(x, w_gate, w_up, w_down, act, y)
    lib = load_library()
    with _on_device(dev):
        y = torch.empty_like(x) if y is None else y
        workspace = _scratch(workspace, lib.bpt_gated_ff_workspace_bytes(rows, D, F, 0), x)
        status = None if lib.bpt_gated_ff_few_rows(rows, D, F) else x.new_empty(256, dtype=torch.uint8)
        y._bpt_workspace = status
        _check(lib.bpt_gated_ff_fwd(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), y.data_ptr(), rows, D, F,
                                    ACTIVATIONS[act], _ptr(status), workspace.data_ptr(), workspace.numel(), _raw_stream(dev)),
               "bpt_gated_ff_fwd")
    return y


def bpt_gated_ff_bwd(x, w_gate, w_up, w_down, dy, act: str = "silu", dx=None, dw_gate=None, dw_up=None, dw_down=None, workspace=None,
                     need_dx: bool = True, need_dw: bool = True):
    """Gradients of bpt_gated_ff_fwd from its inputs and dy: (dx, dw_gate, dw_up, dw_down), bfloat16; None where not needed (the
    three weight gradients together).  Bit-reproducible.  The call's status block stays reachable as `_bpt_workspace` of
    the first gradient for bpt_check."""
    rows, D, F, dev = _check_gated_ff(x, w_gate, w_up, w_down, act, dy, dx)
    if not (need_dx or need_dw):
        raise ValueError("no gradient was asked for")
    for t, w in ((dw_gate, w_gate), (dw_up, w_up), (dw_down, w_down)):
        if t is not None and (t.shape != w.shape or t.dtype != w.dtype or t.get_device() != dev or not t.is_contiguous()):
            raise ValueError("weight gradients must be contiguous and share shape, dtype and device with their weights")
    lib = load_library()
    with _on_device(dev):
        dx = (torch.empty_like(x) if dx is None else dx) if need_dx else None
        dws = [(torch.empty_like(w) if t is None else t) if need_dw else None
               for t, w in ((dw_gate, w_gate), (dw_up, w_up), (dw_down, w_down))]
        workspace = _scratch(workspace, lib.bpt_gated_ff_workspace_bytes(rows, D, F, 1), x)
        status = x.new_empty(256, dtype=torch.uint8)
        (dx if need_dx else dws[0])._bpt_workspace = status
        _check(lib.bpt_gated_ff_bwd(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), dy.data_ptr(), _ptr(dx),
                                    *map(_ptr, dws), rows, D, F, ACTIVATIONS[act], status.data_ptr(), workspace.data_ptr(),
                                    workspace.numel(), _raw_stream(dev)), "bpt_gated_ff_bwd")
    return (dx, *dws)


def _res_norm_args(h, b, weight, bias, norm, post_norm, post_weight, post_bias, gate, alpha, eps):
    """Checks the tensors of a bpt_res_norm call and fills its argument struct."""
    code = _dtype_code(h)
    dt, dev, shape = h.dtype, h.get_device(), h.shape
    if dev < 0 or not shape or not h.is_contiguous():
        raise ValueError("h must be a contiguous CUDA tensor [..., D]")
    D = shape[-1]
    if norm not in NORM_KINDS or post_norm not in NORM_KINDS:
        raise ValueError("norm and post_norm must be None, 'layer' or 'rms'")
    if b is None:
        if post_norm is not None or gate is not None:
            raise ValueError("post_norm and gate belong to b, which is missing")
    elif b.shape != shape or b.dtype != dt or b.get_device() != dev or not b.is_contiguous():
        raise ValueError("b must be contiguous and share shape, dtype and device with h")
    if (norm is None and (weight is not None or bias is not None)) or (post_norm is None and (post_weight is not None or post_bias is not None)):
        raise ValueError("a weight or bias was given for a norm that is None")
    pt, ptrs = None, []
    for t in (weight, bias, post_weight, post_bias):
        if t is None:
            ptrs.append(None)
            continue
        pt = t.dtype if pt is None else pt
        if t.shape != (D,) or t.dtype != pt or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("weights and biases must be contiguous [D] tensors of one dtype on the device of h")
        pcode = _dtype_code(t)
        ptrs.append(t.data_ptr())
    groups = 1
    if gate is not None:
        # the gate's rows: a leading part of h's axes, the others of length one (or missing in front: a gate [D])
        gs = (1,) * (len(shape) - gate.dim()) + tuple(gate.shape)
        lead = len(shape) - 1
        while lead > 0 and gs[lead - 1] == 1:
            lead -= 1
        if not gate.dim() or len(gs) != len(shape) or gs[-1] != D or gs[:lead] != tuple(shape[:lead]) or gate.get_device() != dev or not gate.is_contiguous():
            raise ValueError("gate must be contiguous, [D] or h's shape with the trailing row axes of length one, on the device of h")
        for x in gs[:lead]:
            groups *= x
    rows = h.numel() // D if D else 0
    return ResNormArgs(rows, max(groups, 1), D, code, code if pt is None else pcode, code if gate is None else _dtype_code(gate),
                       NORM_KINDS[norm], NORM_KINDS[post_norm], alpha, eps, h.data_ptr(), None if b is None else b.data_ptr(), *ptrs,
                       None if gate is None else gate.data_ptr()), dev


def _check_like(h, *ts):
    for t in ts:
        if t is not None and (t.shape != h.shape or t.dtype != h.dtype or t.get_device() != h.get_device() or not t.is_contiguous()):
            raise ValueError("results and gradients must be contiguous and share shape, dtype and device with h")


def _check_stats(rows, h, stats):
    if stats is not None and (stats.dtype != torch.float32 or stats.shape != (rows, 4) or stats.get_device() != h.get_device()
                              or not stats.is_contiguous()):
        raise ValueError("stats must be a contiguous float32 tensor [rows, 4] on the device of h")


def bpt_res_norm_fwd(h, b=None, weight=None, bias=None, norm="layer", post_norm=None, post_weight=None, post_bias=None, gate=None,
                     alpha: float = 1.0, eps: float = 1e-5, want_sum: bool = False, y=None, r=None, stats=None):
    """n = post_norm(b), r = alpha * h + gate * n, y = norm(r) over the last axis, in one kernel.  h, b: [..., D] float32 or
    bfloat16, contiguous; norm / post_norm: None, "layer" or "rms" with weights and biases [D]; gate: [D], or h's shape with
    the trailing row axes of length one (one gate row per sequence, per row ...).  Returns (y, r); y is None without a norm,
    r is None unless want_sum (or norm is None).  stats: a float32 tensor [rows, 4] to fill for the backward, or None."""
    args, dev = _res_norm_args(h, b, weight, bias, norm, post_norm, post_weight, post_bias, gate, alpha, eps)
    _check_like(h, y, r)
    _check_stats(args.rows, h, stats)
    with _on_device(dev):
        y = torch.empty_like(h) if y is None and norm is not None else y
        r = torch.empty_like(h) if r is None and (want_sum or norm is None) else r
        _check(load_library().bpt_res_norm_fwd(ctypes.byref(args), _ptr(y), _ptr(r), _ptr(stats), _raw_stream(dev)), "bpt_res_norm_fwd")
    return y, r


def bpt_res_norm_bwd(h, b, dy, dr, stats, weight=None, bias=None, norm="layer", post_norm=None, post_weight=None, post_bias=None, gate=None,
                     alpha: float = 1.0, eps: float = 1e-5, workspace=None, need=(True,) * 7):
    """Backward of bpt_res_norm_fwd from its inputs, its stats and the gradients of y and r (either may be None: zero).  Returns
    (dh, db, d_weight, d_bias, d_post_weight, d_post_bias, d_gate), each in the type of what it belongs to; None where that
    is None or where `need` says so.  Bit-reproducible."""
    args, dev = _res_norm_args(h, b, weight, bias, norm, post_norm, post_weight, post_bias, gate, alpha, eps)
    _check_like(h, dy, dr)
    _check_stats(args.rows, h, stats)
    lib = load_library()
    with _on_device(dev):
        grads = [torch.empty_like(t) if n and t is not None else None
                 for n, t in zip(need, (h, b, weight, bias, post_weight, post_bias, gate))]
        workspace = _scratch(workspace, lib.bpt_res_norm_bwd_workspace_bytes(ctypes.byref(args)), h)
        _check(lib.bpt_res_norm_bwd(ctypes.byref(args), _ptr(stats), _ptr(dy), _ptr(dr), *map(_ptr, grads), workspace.data_ptr(),
                                    workspace.numel(), _raw_stream(dev)), "bpt_res_norm_bwd")
    return tuple(grads)


def bpt_debug_bounds():
    """The index-check record of the checking build as (violations, site, index, limit); raises BptError
    with status 2 on the normal build, which carries no checks."""
    rec = (ctypes.c_uint32 * 4)()
    _check(load_library().bpt_debug_bounds(rec, _stream()), "bpt_debug_bounds")
    return tuple(int(x) for x in rec)


def bpt_selftest_wait_timeout(workspace, limit_cycles: int, arrive: bool):
    """Launches the library's wait self-test (see include/bpt.h); read the outcome with bpt_check."""
    with torch.cuda.device(workspace.device):
        _check(load_library().bpt_selftest_wait_timeout(_ptr(workspace), int(limit_cycles), int(arrive), _stream()),
               "bpt_selftest_wait_timeout")


def _check_layout(g: Graph, q, *same):
    if q.dim() != 4 or q.shape[1] != g.n_nodes:
        raise ValueError("expected [B, n_nodes=%d, H, d], got %s" % (g.n_nodes, tuple(q.shape)))
    for t in same:
        if t.shape != q.shape or t.dtype != q.dtype or t.device != q.device:
            raise ValueError("q, k, v, out, d_out must share shape, dtype and device")
    for t in (q,) + same:
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")
        if not t.is_cuda:
            raise ValueError("tensors must live on a CUDA device")


def _check_lengths(lengths, q):
    if lengths.dtype != torch.int32 or lengths.shape != (q.shape[0],) or lengths.device != q.device or not lengths.is_contiguous():
        raise ValueError("lengths must be a contiguous int32 tensor [B] on the device of q")


def bpt_attn_fwd(g: Graph, q, k, v, rel_emb, scale: float, out=None, lse=None, workspace=None, lengths=None,
                 dropout_p: float = 0.0, dropout_seed: int = 0, path: int = BPT_PATH_AUTO):
    """Returns (out [B,N,H,d], lse [B,N,H] fp32).  With `lengths` (int32 [B] on the device) batch entry b
    has lengths[b] real tokens; with dropout_p > 0 the attention weights are dropped (mask defined by
    dropout_seed); `path` forces a kernel family; see bpt_attn_fwd_varlen / bpt_attn_fwd_ex in include/bpt.h.
    A workspace the wrapper allocates itself stays reachable as `out._bpt_workspace` for bpt_check."""
    lib = load_library()
    _check_layout(g, q, k, v)
    B, N, H, d = q.shape
    code = _dtype_code(q)
    if rel_emb.shape != (g.n_rel, d) or rel_emb.dtype != q.dtype or not rel_emb.is_contiguous():
        raise ValueError("rel_emb must be contiguous [n_rel=%d, d] of the same dtype" % g.n_rel)
    with torch.cuda.device(q.device):
        out = torch.empty_like(q) if out is None else out
        lse = torch.empty((B, N, H), dtype=torch.float32, device=q.device) if lse is None else lse
        need = bpt_attn_workspace_bytes(g, B, H, d, code, False)
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ws_n = 0 if workspace is None else workspace.numel()
        out._bpt_workspace = workspace
        if dropout_p or path:
            if lengths is not None:
                _check_lengths(lengths, q)
            opt = AttnOptions(_ptr(lengths), float(dropout_p), int(dropout_seed), int(path))
            _check(lib.bpt_attn_fwd_ex(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                       float(scale), ctypes.byref(opt), _ptr(out), _ptr(lse), _ptr(workspace), ws_n,
                                       _stream()), "bpt_attn_fwd_ex")
        elif lengths is None:
            _check(lib.bpt_attn_fwd(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                    float(scale), _ptr(out), _ptr(lse), _ptr(workspace), ws_n, _stream()), "bpt_attn_fwd")
        else:
            _check_lengths(lengths, q)
            _check(lib.bpt_attn_fwd_varlen(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                           float(scale), _ptr(lengths), _ptr(out), _ptr(lse), _ptr(workspace), ws_n,
                                           _stream()), "bpt_attn_fwd_varlen")
    return out, lse


def bpt_attn_bwd(g: Graph, q, k, v, rel_emb, scale: float, out, lse, d_out, workspace=None,
                 dq=None, dk=None, dv=None, d_rel=None, lengths=None, dropout_p: float = 0.0, dropout_seed: int = 0,
                 path: int = BPT_PATH_AUTO):
    """Returns (dq, dk, dv [B,N,H,d], d_rel [n_rel, d] fp32).  `lengths`, `dropout_p`, `dropout_seed` as for
    bpt_attn_fwd (pass what the forward had).  A workspace the wrapper allocates itself stays reachable as
    `dq._bpt_workspace` for bpt_check."""
    lib = load_library()
    _check_layout(g, q, k, v, out, d_out)
    B, N, H, d = q.shape
    code = _dtype_code(q)
    with torch.cuda.device(q.device):
        dq = torch.empty_like(q) if dq is None else dq
        dk = torch.empty_like(q) if dk is None else dk
        dv = torch.empty_like(q) if dv is None else dv
        d_rel = torch.empty((g.n_rel, d), dtype=torch.float32, device=q.device) if d_rel is None else d_rel
        need = bpt_attn_workspace_bytes(g, B, H, d, code, True)
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ws_n = 0 if workspace is None else workspace.numel()
        dq._bpt_workspace = workspace
        if dropout_p or path:
            if lengths is not None:
                _check_lengths(lengths, q)
            opt = AttnOptions(_ptr(lengths), float(dropout_p), int(dropout_seed), int(path))
            _check(lib.bpt_attn_bwd_ex(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                       float(scale), ctypes.byref(opt), _ptr(out), _ptr(lse), _ptr(d_out), _ptr(dq),
                                       _ptr(dk), _ptr(dv), _ptr(d_rel), _ptr(workspace), ws_n, _stream()), "bpt_attn_bwd_ex")
        elif lengths is None:
            _check(lib.bpt_attn_bwd(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                    float(scale), _ptr(out), _ptr(lse), _ptr(d_out), _ptr(dq), _ptr(dk), _ptr(dv),
                                    _ptr(d_rel), _ptr(workspace), ws_n, _stream()), "bpt_attn_bwd")
        else:
            _check_lengths(lengths, q)
            _check(lib.bpt_attn_bwd_varlen(ctypes.byref(g.c), B, H, d, code, _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb),
                                           float(scale), _ptr(lengths), _ptr(out), _ptr(lse), _ptr(d_out), _ptr(dq),
                                           _ptr(dk), _ptr(dv), _ptr(d_rel), _ptr(workspace), ws_n, _stream()),
                   "bpt_attn_bwd_varlen")
    return dq, dk, dv, d_rel


def bpt_attn_fwd_rows(g: Graph, q, k, v, rel_emb, scale: float, rows, out, lse, lengths=None,
                      dropout_p: float = 0.0, dropout_seed: int = 0):
    """Recomputes the listed destination rows of (out, lse) in place.  rows: int32 [B, n_rows] node ids on the
    device (one list per batch entry).  The building block of step-by-step decoding: token i and its
    ancestors, with lengths = i + 1."""
    _check_layout(g, q, k, v, out)
    B, N, H, d = q.shape
    if rows.dtype != torch.int32 or rows.dim() != 2 or rows.shape[0] != B or not rows.is_contiguous() or rows.device != q.device:
        raise ValueError("rows must be a contiguous int32 tensor [B, n_rows] on the device of q")
    if lengths is not None:
        _check_lengths(lengths, q)
    opt = AttnOptions(_ptr(lengths), float(dropout_p), int(dropout_seed), 0)
    with torch.cuda.device(q.device):
        _check(load_library().bpt_attn_fwd_rows(ctypes.byref(g.c), B, H, d, _dtype_code(q), _ptr(q), _ptr(k), _ptr(v),
                                                _ptr(rel_emb), float(scale), ctypes.byref(opt), _ptr(rows), rows.shape[1],
                                                _ptr(out), _ptr(lse), _stream()), "bpt_attn_fwd_rows")
    return out, lse


def bpt_static_scratch_bytes() -> int:
    return int(load_library().bpt_static_scratch_bytes())


def bpt_attn_bwd_static_scratch(g: Graph, q, k, v, rel_emb, scale: float, out, lse, d_out, dq, dk, dv, d_rel):
    """Backward pass that takes its scratch from the library's built-in device array instead
    of a workspace tensor, for callers that are not allowed to allocate device memory.  The
    caller passes every input and output (this wrapper allocates nothing either); a problem
    of which one (batch entry, head) pair alone needs more than bpt_static_scratch_bytes() raises
    BptError with status 7.  Calls share the array:
    keep them ordered on one stream."""
    _check_layout(g, q, k, v, out, d_out, dq, dk, dv)
    B, N, H, d = q.shape
    with torch.cuda.device(q.device):
        _check(load_library().bpt_attn_bwd_static_scratch(
            ctypes.byref(g.c), B, H, d, _dtype_code(q), _ptr(q), _ptr(k), _ptr(v), _ptr(rel_emb), float(scale),
            _ptr(out), _ptr(lse), _ptr(d_out), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(d_rel), _stream()),
            "bpt_attn_bwd_static_scratch")
    return dq, dk, dv, d_rel


def bpt_trace_begin(capacity: int):
    """Start recording one CUDA event after every kernel the library launches."""
    _check(load_library().bpt_trace_begin(capacity, _stream()), "bpt_trace_begin")


def bpt_trace_end(capacity: int):
    """Stop recording; returns [(kernel name, milliseconds), ...] in launch order."""
    n = ctypes.c_int32(0)
    ms = (ctypes.c_float * capacity)()
    names = (ctypes.c_char_p * capacity)()
    _check(load_library().bpt_trace_end(ctypes.byref(n), ms, names, capacity), "bpt_trace_end")
    return [(names[i].decode(), float(ms[i])) for i in range(min(n.value, capacity))]
