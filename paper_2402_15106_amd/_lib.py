"""ctypes binding of libdsmpnn (the C ABI declared in include/dsmpnn.h).

Argument marshalling only: every step of the hot path runs in the HIP
library.  Tensors are PyTorch device tensors (device memory and streams are
the only things PyTorch provides); the caller's current stream is bound to the
handle before every call.  Output and scratch buffers are allocated here with
torch when the caller does not pass them.  If the shared library is missing
the import fails: there is no fallback.
"""

import ctypes
import math
import operator
import os
from dataclasses import dataclass
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "lib", "libdsmpnn.so")

OK, INVALID_ARG, CAPACITY, HIP_ERROR, UNSUPPORTED, WORKSPACE_TOO_SMALL = range(6)
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "CAPACITY", 3: "HIP_ERROR", 4: "UNSUPPORTED",
                5: "WORKSPACE_TOO_SMALL"}
CAP_KNN, CAP_RANDOM = 0, 1
F32, BF16 = 0, 1
ACT_IDENTITY, ACT_RELU, ACT_SILU, ACT_GELU = range(4)
ATTR_CONCAT, ATTR_DIFF = 0, 1
ROTATE_HALF, ROTATE_INTERLEAVED = 0, 1
GRAD_ACCUMULATE = 1
GRAD_X_ACCUMULATE = 2
EDGE_AUTO, EDGE_PER_EDGE, EDGE_AGGREGATE = 0, 1, 2

EXPORTED = ["dsmp_version", "dsmp_create", "dsmp_destroy", "dsmp_set_stream", "dsmp_last_error",
            "dsmp_sample_workspace", "dsmp_sample_nodes", "dsmp_sample_nodes_noalloc", "dsmp_gather_rows",
            "dsmp_scatter_rows",
            "dsmp_subdomain_workspace", "dsmp_subdomain_select",
            "dsmp_radius_graph_workspace", "dsmp_radius_graph_count", "dsmp_radius_graph_build",
            "dsmp_radius_graph_rows", "dsmp_radius_graph_edges",
            "dsmp_nnconv_packed_bytes", "dsmp_nnconv_pack", "dsmp_nnconv_workspace",
            "dsmp_nnconv_forward", "dsmp_nnconv_backward", "dsmp_profile_enable", "dsmp_profile_reset",
            "dsmp_profile_read", "dsmp_set_edge_algorithm", "dsmp_mlp_workspace", "dsmp_mlp_forward",
            "dsmp_mlp_backward", "dsmp_masked_mse_workspace", "dsmp_masked_mse",
            "dsmp_checkpoint_store", "dsmp_checkpoint_load", "dsmp_group_norm_workspace", "dsmp_group_norm_forward",
            "dsmp_group_norm_restore", "dsmp_group_norm_backward",
            "dsmp_qk_rotate_forward", "dsmp_qk_rotate_workspace", "dsmp_qk_rotate_backward",
            "dsmp_attention_workspace", "dsmp_attention_forward", "dsmp_attention_backward"]

# kernel classes of the opt-in timing (dsmp_profile_*)
KERNEL_CLASSES = ["sample", "gather", "graph", "edge_fwd", "node_fwd", "node_bwd", "edge_dh", "dh_final",
                  "dz", "dW3", "dW2", "dW1", "reduce", "edge_mlp", "outer_fwd", "gemm_fwd", "outer_dh",
                  "gemm_dh", "u_gemm", "attr", "mlp", "loss", "dh_u", "da1", "norm", "ckpt", "rotate",
                  "attn_fwd", "attn_bwd"]


class DsmpError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), msg))
        self.status = status


class GraphQuery(ctypes.Structure):
    _fields_ = [("pos", ctypes.c_void_p), ("n_src", ctypes.c_int64), ("n_dst", ctypes.c_int64),
                ("dim", ctypes.c_int32), ("r", ctypes.c_float), ("cap", ctypes.c_int32),
                ("cap_mode", ctypes.c_int32), ("seed", ctypes.c_uint64)]


class CGraph(ctypes.Structure):
    _fields_ = [("n_dst", ctypes.c_int64), ("n_src", ctypes.c_int64), ("n_edges", ctypes.c_int64),
                ("row_ptr", ctypes.c_void_p), ("col", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("csc_ptr", ctypes.c_void_p), ("csc_eid", ctypes.c_void_p)]


class LayerDesc(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("d", ctypes.c_int32), ("h1", ctypes.c_int32),
                ("h2", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("residual", ctypes.c_int32), ("attr_mode", ctypes.c_int32)]


class LayerParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("W1", "b1", "W2", "b2", "W3", "b3", "Wr", "br")]


class LayerGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dW1", "db1", "dW2", "db2", "dW3", "db3", "dWr", "dbr", "dattr")]


class MlpDesc(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int32), ("d_hid", ctypes.c_int32), ("d_out", ctypes.c_int32)]


class MlpParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("W1", "b1", "W2", "b2", "W3", "b3")]


class MlpGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dW1", "db1", "dW2", "db2", "dW3", "db3")]


class NormDesc(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("groups", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("y_dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("eps", ctypes.c_float)]


class RotateDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "head_dim", "dtype", "rot", "axes", "layout",
                                              "norm")] + [("eps", ctypes.c_float), ("amplitude", ctypes.c_float)]


class AttentionDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "head_dim", "dtype", "dim")] + [
        ("scale", ctypes.c_float), ("cap", ctypes.c_float)]


class CSegments(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("n_seg", ctypes.c_int64), ("ptr", ctypes.c_void_p)]


class CCheckpoint(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_SIZE = ctypes.POINTER(ctypes.c_size_t)
_ATTN = [_P, ctypes.POINTER(AttentionDesc), ctypes.POINTER(CSegments), ctypes.POINTER(CSegments)]
_MAT = [_P, _I64]
_SIG = {
    "dsmp_version": (ctypes.c_int, []),
    "dsmp_create": (ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]),
    "dsmp_destroy": (ctypes.c_int, [_P]),
    "dsmp_set_stream": (ctypes.c_int, [_P, _P]),
    "dsmp_set_edge_algorithm": (ctypes.c_int, [_P, ctypes.c_int32]),
    "dsmp_last_error": (ctypes.c_char_p, [_P]),
    "dsmp_sample_workspace": (ctypes.c_int, [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_sample_nodes": (ctypes.c_int, [_P, ctypes.c_int64, ctypes.c_int64, ctypes.c_uint64, _P, _P,
                                         ctypes.c_size_t]),
    "dsmp_sample_nodes_noalloc": (ctypes.c_int, [_P, ctypes.c_int64, ctypes.c_int64, ctypes.c_uint64, _P]),
    "dsmp_gather_rows": (ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int64, _P, ctypes.c_int64, _P]),
    "dsmp_scatter_rows": (ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, ctypes.c_int64]),
    "dsmp_subdomain_workspace": (ctypes.c_int, [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_subdomain_select": (ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_float),
                                             ctypes.POINTER(ctypes.c_float), ctypes.c_float, _P, _P, ctypes.c_size_t,
                                             ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]),
    "dsmp_radius_graph_workspace": (ctypes.c_int, [ctypes.POINTER(GraphQuery), ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_radius_graph_count": (ctypes.c_int, [_P, ctypes.POINTER(GraphQuery), _P, ctypes.c_size_t,
                                               ctypes.POINTER(ctypes.c_int64)]),
    "dsmp_radius_graph_build": (ctypes.c_int, [_P, ctypes.POINTER(GraphQuery), _P, ctypes.c_size_t,
                                               ctypes.c_int64, ctypes.POINTER(CGraph)]),
    "dsmp_radius_graph_rows": (ctypes.c_int, [_P, ctypes.POINTER(GraphQuery), _P, ctypes.c_size_t,
                                              ctypes.POINTER(CGraph), ctypes.POINTER(ctypes.c_int32)]),
    "dsmp_radius_graph_edges": (ctypes.c_int, [_P, ctypes.POINTER(GraphQuery), _P, ctypes.c_size_t, ctypes.c_int32,
                                               ctypes.c_int64, ctypes.POINTER(CGraph)]),
    "dsmp_nnconv_packed_bytes": (ctypes.c_int, [ctypes.POINTER(LayerDesc), ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_nnconv_pack": (ctypes.c_int, [_P, ctypes.POINTER(LayerDesc), ctypes.POINTER(LayerParams), _P]),
    "dsmp_nnconv_workspace": (ctypes.c_int, [ctypes.POINTER(LayerDesc), ctypes.POINTER(CGraph),
                                             ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t),
                                             ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_nnconv_forward": (ctypes.c_int, [_P, ctypes.POINTER(LayerDesc), _P, ctypes.POINTER(CGraph), _P, _P,
                                           _P, _P, _P, ctypes.c_size_t, _P, ctypes.c_size_t]),
    "dsmp_nnconv_backward": (ctypes.c_int, [_P, ctypes.POINTER(LayerDesc), _P, ctypes.POINTER(CGraph), _P, _P,
                                            _P, ctypes.c_size_t, _P, _P, ctypes.POINTER(LayerGrads),
                                            ctypes.c_int32, _P, ctypes.c_size_t]),
    "dsmp_mlp_workspace": (ctypes.c_int, [ctypes.POINTER(MlpDesc), ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t),
                                          ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_mlp_forward": (ctypes.c_int, [_P, ctypes.POINTER(MlpDesc), ctypes.POINTER(MlpParams), _P, ctypes.c_int64,
                                        _P, _P, _P, ctypes.c_size_t]),
    "dsmp_mlp_backward": (ctypes.c_int, [_P, ctypes.POINTER(MlpDesc), ctypes.POINTER(MlpParams), _P, ctypes.c_int64,
                                         _P, ctypes.c_size_t, _P, _P, ctypes.POINTER(MlpGrads), ctypes.c_int32, _P,
                                         ctypes.c_size_t]),
    "dsmp_masked_mse_workspace": (ctypes.c_int, [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_masked_mse": (ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, _P, _P, _P, ctypes.c_size_t]),
    "dsmp_checkpoint_store": (ctypes.c_int, [_P, _P, ctypes.c_int32, _I64, _I64, ctypes.c_int32,
                                             ctypes.POINTER(CCheckpoint)]),
    "dsmp_checkpoint_load": (ctypes.c_int, [_P, ctypes.POINTER(CCheckpoint), _I64, ctypes.c_int32, _P, ctypes.c_int32,
                                            _I64]),
    "dsmp_group_norm_workspace": (ctypes.c_int, [ctypes.POINTER(NormDesc), ctypes.POINTER(CSegments),
                                                 ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]),
    "dsmp_group_norm_forward": (ctypes.c_int, [_P, ctypes.POINTER(NormDesc), ctypes.POINTER(CSegments), _P, _I64, _P,
                                               _I64, _P, _I64, _P, _P, _P, _I64, _P, ctypes.POINTER(CCheckpoint), _P,
                                               ctypes.c_size_t]),
    "dsmp_group_norm_restore": (ctypes.c_int, [_P, ctypes.POINTER(NormDesc), ctypes.POINTER(CSegments),
                                               ctypes.POINTER(CCheckpoint), _P, _P, _P, _P, _I64]),
    "dsmp_group_norm_backward": (ctypes.c_int, [_P, ctypes.POINTER(NormDesc), ctypes.POINTER(CSegments), _P, _I64,
                                                ctypes.POINTER(CCheckpoint), _P, _P, _P, _P, _I64, _P, _I64, _P, _I64,
                                                _P, _P, ctypes.c_int32, _P, ctypes.c_size_t]),
    "dsmp_qk_rotate_forward": (ctypes.c_int, [_P, ctypes.POINTER(RotateDesc), _I64] + 2 * _MAT + 4 * [_P] + 2 * _MAT),
    "dsmp_qk_rotate_workspace": (ctypes.c_int, [ctypes.POINTER(RotateDesc), _I64, _SIZE]),
    "dsmp_qk_rotate_backward": (ctypes.c_int, [_P, ctypes.POINTER(RotateDesc), _I64] + 2 * _MAT + 4 * [_P] + 4 * _MAT
                                + [_P, _P, ctypes.c_int32, _P, ctypes.c_size_t]),
    "dsmp_attention_workspace": (ctypes.c_int, _ATTN[1:] + [_SIZE, _SIZE]),
    "dsmp_attention_forward": (ctypes.c_int, _ATTN + 3 * _MAT + 3 * [_P] + _MAT + [_P, _P, ctypes.c_size_t]),
    "dsmp_attention_backward": (ctypes.c_int, _ATTN + 3 * _MAT + 3 * [_P] + _MAT + [_P] + 4 * _MAT
                                + [_P, ctypes.c_size_t]),
    "dsmp_profile_enable": (ctypes.c_int, [_P, ctypes.c_int]),
    "dsmp_profile_reset": (ctypes.c_int, [_P]),
    "dsmp_profile_read": (ctypes.c_int, [_P, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                         ctypes.POINTER(ctypes.c_int64)]),
}

# address of the current stream of a device, without a Stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _current_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream if _raw_stream is None else _raw_stream(index)


# whether the current stream is being captured, without the function around it
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", torch.cuda.is_current_stream_capturing)


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libdsmpnn.so and declare every exported signature (no GPU needed)."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise ImportError("libdsmpnn.so is not built (%s); run __graft_entry__.build()" % path)
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIG.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path == LIB_PATH:
        _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


@dataclass
class Graph:
    """A radius graph held in device tensors (int32)."""
    n_dst: int
    n_src: int
    n_edges: int
    row_ptr: torch.Tensor
    col: torch.Tensor
    dst: torch.Tensor
    csc_ptr: torch.Tensor
    csc_eid: torch.Tensor

    def c(self) -> CGraph:
        return CGraph(self.n_dst, self.n_src, self.n_edges, self.row_ptr.data_ptr(),
                      self.col.data_ptr(), self.dst.data_ptr(), self.csc_ptr.data_ptr(),
                      self.csc_eid.data_ptr())


@dataclass
class Checkpoint:
    """Rows of values kept in 8 bits: q int8 [n, channels], scale float32
    [n, ceil(channels / 64)], both contiguous."""
    q: torch.Tensor
    scale: torch.Tensor

    @staticmethod
    def empty(n: int, channels: int, device) -> "Checkpoint":
        return Checkpoint(torch.empty(n, channels, dtype=torch.int8, device=device),
                          torch.empty(n, (channels + 63) // 64, dtype=torch.float32, device=device))


def norm_desc(channels, groups, x_dtype, y_dtype, act=ACT_IDENTITY, eps=1e-5) -> NormDesc:
    return NormDesc(channels, groups, x_dtype, y_dtype, act, eps)


def rotate_desc(heads, kv_heads, head_dim, dtype, rot, axes=1, layout=ROTATE_HALF, norm=True, eps=1e-6,
                amplitude=1.0) -> RotateDesc:
    return RotateDesc(heads, kv_heads, head_dim, dtype, rot, axes, layout, int(norm), eps, amplitude)


def attention_desc(heads, kv_heads, head_dim, dtype, dim=0, scale=None, cap=0.0) -> AttentionDesc:
    """scale: 1 / sqrt(head_dim) if not given."""
    return AttentionDesc(heads, kv_heads, head_dim, dtype, dim, head_dim ** -0.5 if scale is None else scale, cap)


def rotary_frequencies(rot, axes=1, base=10000.0, factor=1.0, extent=None, slow=1.0, fast=32.0, device=None):
    """Frequencies (float32 [rot / 2], radians per unit of a coordinate) of
    dsmp_qk_rotate_*: base^(-i / m) for the m = rot / 2 / axes pairs i of each axis.

    factor > 1 scales them for coordinates that reach `factor` times further than those a
    model was trained on: all by 1 / factor (interpolated positions, arXiv 2306.15595); or, with
    `extent` (the trained range), pairs that turn fewer than `slow` times over it by 1 / factor,
    those that turn more than `fast` times not at all, and those between by a linear mixture of
    both (arXiv 2309.00071, section 3.2)."""
    if axes < 1 or rot < 0 or rot % (2 * axes):
        raise DsmpError(INVALID_ARG, "rot must be a multiple of 2 axes")
    if not (base > 0 and factor > 0 and (extent is None or (extent > 0 and fast > slow))):
        raise DsmpError(INVALID_ARG, "base, factor and extent must be positive, and fast more than slow")
    m = rot // 2 // axes
    f = torch.pow(torch.tensor(float(base), dtype=torch.float64), -torch.arange(m, dtype=torch.float64) / max(m, 1))
    if extent is None:
        f = f / factor
    else:
        keep = ((f * extent / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f.repeat(axes).to(dtype=torch.float32, device=device)


_TORCH = {F32: torch.float32, BF16: torch.bfloat16}
_CODE = {torch.float32: F32, torch.bfloat16: BF16}


def layer_desc(dim, d, h1, h2, dtype, act=ACT_IDENTITY, residual=1, attr_mode=ATTR_CONCAT) -> LayerDesc:
    return LayerDesc(dim, d, h1, h2, dtype, act, residual, attr_mode)


def _torch_dtype(desc: LayerDesc):
    return torch.bfloat16 if desc.dtype == BF16 else torch.float32


class Dsmp:
    """A library handle on one device, with methods named after the C calls."""

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = torch.device("cuda", device)
        h = ctypes.c_void_p()
        self._check(self.lib.dsmp_create(ctypes.byref(h), device), None)
        self.h = h
        self._ws = {}
        self._index = device
        self._norm_sizes = {}
        self._attn_sizes = {}

    def close(self):
        if getattr(self, "h", None) is not None:
            self.lib.dsmp_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------ helpers
    def _check(self, st, h):
        if st != OK:
            msg = self.lib.dsmp_last_error(h).decode() if h is not None else ""
            raise DsmpError(st, msg)

    def _bind(self):
        s = torch.cuda.current_stream(self.device).cuda_stream
        self._check(self.lib.dsmp_set_stream(self.h, ctypes.c_void_p(s)), self.h)

    def dsmp_set_edge_algorithm(self, algorithm: int):
        """Edge-contraction form for later layer calls (EDGE_AUTO / EDGE_PER_EDGE / EDGE_AGGREGATE)."""
        self._check(self.lib.dsmp_set_edge_algorithm(self.h, int(algorithm)), self.h)

    def workspace(self, key: str, nbytes: int) -> torch.Tensor:
        """A cached uint8 device buffer of at least nbytes for scratch use."""
        buf = self._ws.get(key)
        if buf is None or buf.numel() < nbytes:
            buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            self._ws[key] = buf
        return buf

    # ------------------------------------------------------------ timing
    def dsmp_profile_enable(self, on: bool = True):
        self._check(self.lib.dsmp_profile_enable(self.h, int(bool(on))), self.h)

    def dsmp_profile_reset(self):
        self._check(self.lib.dsmp_profile_reset(self.h), self.h)

    def dsmp_profile_read(self) -> dict:
        """{kernel class: (total ms, launches)} since the last reset (synchronises)."""
        out = {}
        for i, name in enumerate(KERNEL_CLASSES):
            ms, n = ctypes.c_double(), ctypes.c_int64()
            self._check(self.lib.dsmp_profile_read(self.h, i, ctypes.byref(ms), ctypes.byref(n)), self.h)
            out[name] = (ms.value, n.value)
        return out

    # ------------------------------------------------------------ sampling
    def dsmp_sample_nodes(self, M: int, s: int, seed: int, out: Optional[torch.Tensor] = None):
        out = torch.empty(s, dtype=torch.int32, device=self.device) if out is None else out
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_sample_workspace(M, ctypes.byref(nb)), None)
        ws = self.workspace("sample", nb.value)
        self._bind()
        self._check(self.lib.dsmp_sample_nodes(self.h, M, s, ctypes.c_uint64(seed & (2 ** 64 - 1)),
                                               _ptr(out), _ptr(ws), ws.numel()), self.h)
        return out

    def dsmp_sample_nodes_noalloc(self, M: int, s: int, seed: int, out: torch.Tensor):
        """dsmp_sample_nodes on the library's own scratch (no workspace); out
        is the caller's int32 [s] device buffer."""
        self._bind()
        self._check(self.lib.dsmp_sample_nodes_noalloc(self.h, M, s, seed & (2 ** 64 - 1), _ptr(out)), self.h)
        return out

    def dsmp_gather_rows(self, src: torch.Tensor, idx: torch.Tensor, out: Optional[torch.Tensor] = None):
        src = src.contiguous()
        n = idx.numel()
        out = torch.empty((n,) + tuple(src.shape[1:]), dtype=src.dtype, device=self.device) if out is None else out
        row_bytes = src[0].numel() * src.element_size() if src.shape[0] > 0 else out[0].numel() * out.element_size()
        self._bind()
        self._check(self.lib.dsmp_gather_rows(self.h, _ptr(src), src.shape[0], row_bytes, _ptr(idx), n,
                                              _ptr(out)), self.h)
        return out

    def dsmp_scatter_rows(self, src: torch.Tensor, idx: torch.Tensor, out: torch.Tensor):
        """out[idx[i]] = src[i] (the inverse of dsmp_gather_rows)."""
        src = src.contiguous()
        n = idx.numel()
        row_bytes = out[0].numel() * out.element_size() if out.shape[0] > 0 else 4
        self._bind()
        self._check(self.lib.dsmp_scatter_rows(self.h, _ptr(src), n, row_bytes, _ptr(idx), _ptr(out),
                                               out.shape[0]), self.h)
        return out

    # ------------------------------------------------------------ sub-domains
    def dsmp_subdomain_select(self, pos: torch.Tensor, lo, hi, overlap: float,
                              out: Optional[torch.Tensor] = None):
        """Nodes of the box [lo, hi) with overlap: (idx [n_total] int32 with the
        owned nodes first, n_owned).  Synchronises."""
        pos = pos.contiguous()
        n, D = pos.shape
        out = torch.empty(max(n, 1), dtype=torch.int32, device=self.device) if out is None else out
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_subdomain_workspace(n, ctypes.byref(nb)), None)
        ws = self.workspace("subdomain", nb.value)
        clo = (ctypes.c_float * D)(*[float(v) for v in lo])
        chi = (ctypes.c_float * D)(*[float(v) for v in hi])
        n_own, n_tot = ctypes.c_int64(), ctypes.c_int64()
        self._bind()
        self._check(self.lib.dsmp_subdomain_select(self.h, _ptr(pos), n, D, clo, chi, float(overlap), _ptr(out),
                                                   _ptr(ws), ws.numel(), ctypes.byref(n_own),
                                                   ctypes.byref(n_tot)), self.h)
        return out[:n_tot.value], n_own.value

    # ------------------------------------------------------------ graph
    def _query(self, pos, n_dst, r, cap, cap_mode, seed):
        pos = pos.contiguous()
        return GraphQuery(pos.data_ptr() if pos.numel() else 0, pos.shape[0], n_dst, pos.shape[1],
                          float(r), int(cap), int(cap_mode), seed & (2 ** 64 - 1)), pos

    def _graph_ws(self, q):
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_radius_graph_workspace(ctypes.byref(q), ctypes.byref(nb)), None)
        return self.workspace("graph", nb.value)

    def dsmp_radius_graph_count(self, pos, n_dst, r, cap=0, cap_mode=CAP_KNN, seed=0) -> int:
        q, pos = self._query(pos, n_dst, r, cap, cap_mode, seed)
        ws = self._graph_ws(q)
        E = ctypes.c_int64()
        self._bind()
        self._check(self.lib.dsmp_radius_graph_count(self.h, ctypes.byref(q), _ptr(ws), ws.numel(),
                                                     ctypes.byref(E)), self.h)
        return E.value

    def dsmp_radius_graph_build(self, pos, n_dst, r, cap=0, cap_mode=CAP_KNN, seed=0,
                                capacity: Optional[int] = None, out: Optional[Graph] = None) -> Graph:
        q, pos = self._query(pos, n_dst, r, cap, cap_mode, seed)
        i32 = dict(dtype=torch.int32, device=self.device)
        if out is None and capacity is None:
            # the edge arrays allocated between the build's two halves, by the edge
            # count; the GPU idles from the first half's end to the second's start,
            # so all else is prepared ahead
            ws = self._graph_ws(q)
            row_ptr, e = torch.empty(n_dst + 1, **i32), torch.empty(0, **i32)
            out = Graph(n_dst, pos.shape[0], 0, row_ptr, e, e, torch.empty(pos.shape[0] + 1, **i32), e)
            cg, max_row, edges, new = out.c(), ctypes.c_int32(), self.lib.dsmp_radius_graph_edges, row_ptr.new_empty
            args, cgp = (self.h, ctypes.byref(q), _ptr(ws), ws.numel()), ctypes.byref(cg)
            self._bind()
            self._check(self.lib.dsmp_radius_graph_rows(*args, cgp, ctypes.byref(max_row)), self.h)
            E = cg.n_edges
            n = E or 1
            out.col, out.dst, out.csc_eid = col, dst, eid = new(n), new(n), new(n)
            cg.col, cg.dst, cg.csc_eid = col.data_ptr(), dst.data_ptr(), eid.data_ptr()
            self._check(edges(*args, max_row, E, cgp), self.h)
            out.n_edges = E
            return out
        if out is None:
            out = Graph(n_dst, pos.shape[0], 0, torch.empty(n_dst + 1, **i32),
                        torch.empty(max(capacity, 1), **i32), torch.empty(max(capacity, 1), **i32),
                        torch.empty(pos.shape[0] + 1, **i32), torch.empty(max(capacity, 1), **i32))
        cap_e = out.col.numel() if capacity is None else capacity
        ws = self._graph_ws(q)
        cg = out.c()
        self._bind()
        st = self.lib.dsmp_radius_graph_build(self.h, ctypes.byref(q), _ptr(ws), ws.numel(), cap_e,
                                              ctypes.byref(cg))
        out.n_edges = cg.n_edges
        out.n_dst, out.n_src = cg.n_dst, cg.n_src
        self._check(st, self.h)
        return out

    # ------------------------------------------------------------ layer
    def dsmp_nnconv_pack(self, desc: LayerDesc, params: dict, out: Optional[torch.Tensor] = None):
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_nnconv_packed_bytes(ctypes.byref(desc), ctypes.byref(nb)), None)
        out = torch.empty(nb.value, dtype=torch.uint8, device=self.device) if out is None else out
        P = {k: params[k].to(device=self.device, dtype=torch.float32).contiguous() for k in
             ("W1", "b1", "W2", "b2", "W3", "b3", "Wr", "br")}
        lp = LayerParams(*[P[k].data_ptr() for k in ("W1", "b1", "W2", "b2", "W3", "b3", "Wr", "br")])
        self._bind()
        self._check(self.lib.dsmp_nnconv_pack(self.h, ctypes.byref(desc), ctypes.byref(lp), _ptr(out)), self.h)
        out._keepalive = P   # the pack is asynchronous: keep inputs alive with the output
        return out

    def dsmp_nnconv_workspace(self, desc: LayerDesc, g: Graph):
        s, f, b = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        cg = g.c()
        self._check(self.lib.dsmp_nnconv_workspace(ctypes.byref(desc), ctypes.byref(cg), ctypes.byref(s),
                                                   ctypes.byref(f), ctypes.byref(b)), None)
        return s.value, f.value, b.value

    def dsmp_nnconv_forward(self, desc: LayerDesc, packed, g: Graph, node_attr, h_in, h_out=None,
                            h_out_lp=None, saved=None, ws=None):
        sb, fb, _ = self.dsmp_nnconv_workspace(desc, g)
        if h_out is None:
            h_out = torch.empty(g.n_dst, desc.d, dtype=torch.float32, device=self.device)
        if saved is None:
            saved = torch.empty(max(sb, 256), dtype=torch.uint8, device=self.device)
        if ws is None:
            ws = self.workspace("fwd", fb)
        cg = g.c()
        self._bind()
        self._check(self.lib.dsmp_nnconv_forward(self.h, ctypes.byref(desc), _ptr(packed), ctypes.byref(cg),
                                                 _ptr(node_attr), _ptr(h_in), _ptr(h_out), _ptr(h_out_lp),
                                                 _ptr(saved), saved.numel(), _ptr(ws), ws.numel()), self.h)
        return h_out, saved

    def dsmp_nnconv_backward(self, desc: LayerDesc, packed, g: Graph, node_attr, h_in, saved, grad_out,
                             grad_h=None, grads: Optional[dict] = None, flags: int = 0, ws=None):
        _, _, bb = self.dsmp_nnconv_workspace(desc, g)
        d, h1, h2 = desc.d, desc.h1, desc.h2
        de = 2 * desc.dim + 2 if desc.attr_mode == ATTR_CONCAT else desc.dim + 1
        f32 = dict(dtype=torch.float32, device=self.device)
        if grad_h is None:
            grad_h = torch.empty(g.n_src, d, **f32)
        if grads is None:
            grads = {"dW1": torch.empty(h1, de, **f32), "db1": torch.empty(h1, **f32),
                     "dW2": torch.empty(h2, h1, **f32), "db2": torch.empty(h2, **f32),
                     "dW3": torch.empty(d * d, h2, **f32), "db3": torch.empty(d * d, **f32),
                     "dWr": torch.empty(d, d, **f32), "dbr": torch.empty(d, **f32)}
        lg = LayerGrads(*[grads[k].data_ptr() for k in ("dW1", "db1", "dW2", "db2", "dW3", "db3", "dWr", "dbr")],
                        grads["dattr"].data_ptr() if grads.get("dattr") is not None else None)
        if ws is None:
            ws = self.workspace("bwd", bb)
        cg = g.c()
        self._bind()
        self._check(self.lib.dsmp_nnconv_backward(self.h, ctypes.byref(desc), _ptr(packed), ctypes.byref(cg),
                                                  _ptr(node_attr), _ptr(h_in), _ptr(saved), saved.numel(),
                                                  _ptr(grad_out), _ptr(grad_h), ctypes.byref(lg), flags,
                                                  _ptr(ws), ws.numel()), self.h)
        return grad_h, grads

    # ------------------------------------------------------------ encoder / decoder and loss
    def dsmp_mlp_workspace(self, desc: "MlpDesc", n: int):
        sb, wb = ctypes.c_size_t(), ctypes.c_size_t()
        self._check(self.lib.dsmp_mlp_workspace(ctypes.byref(desc), n, ctypes.byref(sb), ctypes.byref(wb)), None)
        return sb.value, wb.value

    def dsmp_mlp_forward(self, desc: "MlpDesc", params: dict, x, y=None, y_bf16=None, saved=None):
        """Three-layer perceptron on the rows of x (float32 [n, d_in]); returns (y, saved)."""
        n = x.shape[0]
        sb, _ = self.dsmp_mlp_workspace(desc, n)
        if y is None:
            y = torch.empty(n, desc.d_out, dtype=torch.float32, device=self.device)
        if saved is None:
            saved = torch.empty(max(sb, 256), dtype=torch.uint8, device=self.device)
        mp = MlpParams(*[params[k].data_ptr() for k in ("W1", "b1", "W2", "b2", "W3", "b3")])
        self._bind()
        self._check(self.lib.dsmp_mlp_forward(self.h, ctypes.byref(desc), ctypes.byref(mp), _ptr(x), n, _ptr(y),
                                              _ptr(y_bf16), _ptr(saved), saved.numel()), self.h)
        return y, saved

    def dsmp_mlp_backward(self, desc: "MlpDesc", params: dict, x, saved, grad_y, grad_x=None,
                          grads: Optional[dict] = None, flags: int = 0, ws=None):
        """Gradients of sum(grad_y * y); grad_x optional (None: not computed).  Returns grads."""
        n = x.shape[0]
        _, wb = self.dsmp_mlp_workspace(desc, n)
        f32 = dict(dtype=torch.float32, device=self.device)
        if grads is None:
            grads = {"dW1": torch.empty(desc.d_hid, desc.d_in, **f32), "db1": torch.empty(desc.d_hid, **f32),
                     "dW2": torch.empty(desc.d_hid, desc.d_hid, **f32), "db2": torch.empty(desc.d_hid, **f32),
                     "dW3": torch.empty(desc.d_out, desc.d_hid, **f32), "db3": torch.empty(desc.d_out, **f32)}
        mp = MlpParams(*[params[k].data_ptr() for k in ("W1", "b1", "W2", "b2", "W3", "b3")])
        mg = MlpGrads(*[grads[k].data_ptr() for k in ("dW1", "db1", "dW2", "db2", "dW3", "db3")])
        if ws is None:
            ws = self.workspace("mlp_bwd", wb)
        self._bind()
        self._check(self.lib.dsmp_mlp_backward(self.h, ctypes.byref(desc), ctypes.byref(mp), _ptr(x), n, _ptr(saved),
                                               saved.numel(), _ptr(grad_y), _ptr(grad_x), ctypes.byref(mg), flags,
                                               _ptr(ws), ws.numel()), self.h)
        return grads

    def dsmp_masked_mse(self, pred, target, mask, loss=None, grad=None):
        """Mean squared error over interior rows (mask uint8 [n]); returns (loss [1] device, grad)."""
        n, c = pred.shape
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_masked_mse_workspace(n, ctypes.byref(nb)), None)
        ws = self.workspace("mse", nb.value)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        self._bind()
        self._check(self.lib.dsmp_masked_mse(self.h, _ptr(pred), _ptr(target), _ptr(mask), n, c, _ptr(loss),
                                             _ptr(grad), _ptr(ws), ws.numel()), self.h)
        return loss, grad

    # ------------------------------------------------------------ checkpoints in 8 bits and group norm
    # Small inputs take less time on the GPU than a call takes here: the checks
    # look at each tensor once, sizes are asked for once.
    def _rows(self, t, name, shape, dtype):
        """(address, row distance) of a matrix whose rows are contiguous."""
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
                and t.get_device() == self._index):
            raise DsmpError(INVALID_ARG, "%s: a %s %s on %s is needed" % (name, dtype, list(shape), self.device))
        if t.is_contiguous():
            return t.data_ptr(), shape[1]
        ld, one = t.stride()
        if shape[0] <= 1:
            ld = shape[1]
        if ld < shape[1] or (one != 1 and shape[1] > 1):
            raise DsmpError(INVALID_ARG, "%s: rows must be contiguous and not overlap" % name)
        return t.data_ptr(), ld

    def _flat(self, t, name, shape, dtype=torch.float32):
        """Address of a contiguous array of a shape."""
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous()
                and t.get_device() == self._index):
            raise DsmpError(INVALID_ARG, "%s: a contiguous %s %s on %s is needed" % (name, dtype, list(shape), self.device))
        return t.data_ptr()

    def _checkpoint(self, ck, shape):
        if not isinstance(ck, Checkpoint):
            raise DsmpError(INVALID_ARG, "a Checkpoint is needed")
        return CCheckpoint(self._flat(ck.q, "q", shape, torch.int8),
                           self._flat(ck.scale, "scale", (shape[0], (shape[1] + 63) // 64)))

    def _segments(self, n, segments):
        if segments is None:
            return CSegments(n, 1, None)
        if isinstance(segments, torch.Tensor):
            k = segments.numel() - 1
            if k < 1:
                raise DsmpError(INVALID_ARG, "segments: bounds of one segment at least are needed")
            return CSegments(n, k, self._flat(segments, "segments", (k + 1,), torch.int32))
        try:
            k = operator.index(segments)
        except TypeError:
            raise DsmpError(INVALID_ARG, "segments: a whole number or a tensor of bounds is needed") from None
        if k < 1 or n % k:
            raise DsmpError(INVALID_ARG, "segments: %d do not divide %d rows" % (k, n))
        return CSegments(n, k, None)

    def _norm_params(self, C, gamma, beta):
        return (None if gamma is None else self._flat(gamma, "gamma", (C,)),
                None if beta is None else self._flat(beta, "beta", (C,)))

    def _bind_current(self):
        s = _current_stream(self._index)
        st = self.lib.dsmp_set_stream(self.h, s)
        if st:
            self._check(st, self.h)
        return s

    def _norm_size(self, desc, C, seg, n):
        """Workspace bytes of the forward and the backward call."""
        key = (C, desc.groups, n, seg.n_seg, seg.ptr is None)
        sizes = self._norm_sizes.get(key)
        if sizes is None:
            f, b = ctypes.c_size_t(), ctypes.c_size_t()
            self._check(self.lib.dsmp_group_norm_workspace(ctypes.byref(desc), ctypes.byref(seg), ctypes.byref(f),
                                                           ctypes.byref(b)), None)
            if len(self._norm_sizes) >= 1024:
                self._norm_sizes.clear()
            sizes = self._norm_sizes[key] = (f.value, b.value)
        return sizes

    def _norm_ws(self, desc, C, seg, n, backward, ws):
        """Binds the current stream; address and size of the scratch buffer: the caller's, or the one
        that the stream's calls share.  A captured call gets one from the graph's own memory: its address
        stays in the graph, while the shared one is replaced when a larger call comes, and is used by the
        stream's other calls while the graph may be replayed on another."""
        size = self._norm_size(desc, C, seg, n)[backward]
        stream = self._bind_current()
        if ws is not None:
            return self._flat(ws, "ws", (ws.numel(),) if isinstance(ws, torch.Tensor) else (), torch.uint8), ws.numel()
        if _capturing():
            ws = torch.empty(max(size, 256), dtype=torch.uint8, device=self.device)
        else:
            ws = self.workspace(("norm", stream), size)
        return ws.data_ptr(), ws.numel()

    def dsmp_group_norm_workspace(self, desc: NormDesc, n: int, segments=None):
        """Bytes of scratch that dsmp_group_norm_forward and _backward need for n rows (their ws): (forward, backward)."""
        return self._norm_size(desc, desc.channels, self._segments(n, segments), n)

    def dsmp_checkpoint_store(self, x: torch.Tensor, out: Optional[Checkpoint] = None) -> Checkpoint:
        """Keep the rows of x (float32 or bfloat16 [n, channels]) in 8 bits."""
        if not isinstance(x, torch.Tensor) or x.dim() != 2 or x.dtype not in _CODE:
            raise DsmpError(INVALID_ARG, "x: a float32 or bfloat16 matrix is needed")
        n, C = shape = x.shape
        p, ld = self._rows(x, "x", shape, x.dtype)
        out = Checkpoint.empty(n, C, self.device) if out is None else out
        ck = self._checkpoint(out, shape)
        self._bind_current()
        st = self.lib.dsmp_checkpoint_store(self.h, p, _CODE[x.dtype], ld, n, C, ck)
        if st:
            self._check(st, self.h)
        return out

    def dsmp_checkpoint_load(self, ck: Checkpoint, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The kept values (float32, or y's type)."""
        n, C = shape = ck.q.shape
        if y is None:
            y = torch.empty(n, C, dtype=torch.float32, device=self.device)
        if y.dtype not in _CODE:
            raise DsmpError(INVALID_ARG, "y: a float32 or bfloat16 matrix is needed")
        p, ld = self._rows(y, "y", shape, y.dtype)
        cck = self._checkpoint(ck, shape)
        self._bind_current()
        st = self.lib.dsmp_checkpoint_load(self.h, cck, n, C, p, _CODE[y.dtype], ld)
        if st:
            self._check(st, self.h)
        return y

    def dsmp_group_norm_forward(self, desc: NormDesc, x, gamma, beta, segments=None, addend=None, sum_out=None, y=None,
                                stats=None, checkpoint: Optional[Checkpoint] = None, ws=None):
        """y = act(norm(t) gamma + beta) with t = x (+ addend); returns (y, stats).

        segments: None (all rows), the number of equal segments (x.shape[0]:
        each row its own), or an int32 tensor of the n_seg + 1 segment bounds.
        sum_out receives t (needed with an addend; x or addend itself may be
        given); checkpoint, if given, receives t in 8 bits.  ws: scratch of the caller's
        own (uint8, dsmp_group_norm_workspace), in place of the library's; needed in a capture
        that torch.cuda.graph does not make."""
        C, n = desc.channels, x.shape[0]
        rows = (n, C)
        seg = self._segments(n, segments)
        xt, yt = _TORCH.get(desc.x_dtype), _TORCH.get(desc.y_dtype)
        xp, ldx = self._rows(x, "x", rows, xt)
        ap, lda = (None, 0) if addend is None else self._rows(addend, "addend", rows, xt)
        sp, lds = (None, 0) if sum_out is None else self._rows(sum_out, "sum_out", rows, xt)
        gp, bp = self._norm_params(C, gamma, beta)
        y = torch.empty(n, C, dtype=yt, device=self.device) if y is None else y
        yp, ldy = self._rows(y, "y", rows, yt)
        shape = (seg.n_seg, desc.groups, 2)
        stats = torch.empty(shape, dtype=torch.float32, device=self.device) if stats is None else stats
        stp = self._flat(stats, "stats", shape)
        ck = None if checkpoint is None else self._checkpoint(checkpoint, rows)
        ws, ws_bytes = self._norm_ws(desc, C, seg, n, False, ws)
        st = self.lib.dsmp_group_norm_forward(self.h, desc, seg, xp, ldx, ap, lda, sp, lds, gp, bp, yp, ldy, stp, ck, ws,
                                              ws_bytes)
        if st:
            self._check(st, self.h)
        return y, stats

    def dsmp_group_norm_restore(self, desc: NormDesc, checkpoint: Checkpoint, stats, gamma, beta, segments=None, y=None):
        """The forward's y again, from the checkpoint of t and the kept statistics."""
        C, n = desc.channels, checkpoint.q.shape[0]
        rows = (n, C)
        seg = self._segments(n, segments)
        yt = _TORCH.get(desc.y_dtype)
        ck = self._checkpoint(checkpoint, rows)
        stp = self._flat(stats, "stats", (seg.n_seg, desc.groups, 2))
        gp, bp = self._norm_params(C, gamma, beta)
        y = torch.empty(n, C, dtype=yt, device=self.device) if y is None else y
        yp, ldy = self._rows(y, "y", rows, yt)
        self._bind_current()
        st = self.lib.dsmp_group_norm_restore(self.h, desc, seg, ck, stp, gp, bp, yp, ldy)
        if st:
            self._check(st, self.h)
        return y

    def dsmp_group_norm_backward(self, desc: NormDesc, source, stats, gamma, beta, grad_y, segments=None,
                                 grad_addend=None, grad_x=None, grads: Optional[dict] = None, flags: int = 0, ws=None):
        """Gradients of the forward that left stats, from t itself or its
        Checkpoint (source); returns (grad_x, {"dgamma", "dbeta"}).  grad_addend
        (which may be grad_x itself) is added to grad_x.  ws: as for the forward."""
        kept = isinstance(source, Checkpoint)
        C, n = desc.channels, (source.q if kept else source).shape[0]
        rows = (n, C)
        seg = self._segments(n, segments)
        xp, ldx = (None, 0) if kept else self._rows(source, "x", rows, _TORCH.get(desc.x_dtype))
        ck = self._checkpoint(source, rows) if kept else None
        stp = self._flat(stats, "stats", (seg.n_seg, desc.groups, 2))
        gp, bp = self._norm_params(C, gamma, beta)
        dyp, ldgy = self._rows(grad_y, "grad_y", rows, torch.float32)
        gap, ldga = (None, 0) if grad_addend is None else self._rows(grad_addend, "grad_addend", rows, torch.float32)
        f32 = dict(dtype=torch.float32, device=self.device)
        grad_x = torch.empty(n, C, **f32) if grad_x is None else grad_x
        dxp, ldgx = self._rows(grad_x, "grad_x", rows, torch.float32)
        if gamma is None:
            grads, dg, db = {}, None, None
        else:
            grads = {"dgamma": torch.empty(C, **f32), "dbeta": torch.empty(C, **f32)} if grads is None else grads
            dg, db = self._flat(grads["dgamma"], "dgamma", (C,)), self._flat(grads["dbeta"], "dbeta", (C,))
        ws, ws_bytes = self._norm_ws(desc, C, seg, n, True, ws)
        st = self.lib.dsmp_group_norm_backward(self.h, desc, seg, xp, ldx, ck, stp, gp, bp, dyp, ldgy, gap, ldga, dxp,
                                               ldgx, dg, db, flags, ws, ws_bytes)
        if st:
            self._check(st, self.h)
        return grad_x, grads

    # ------------------------------------------------------------ attention
    def _scratch(self, key, size, ws):
        """Binds the current stream; address and size of the scratch buffer, as for the norms."""
        stream = self._bind_current()
        if ws is not None:
            return self._flat(ws, "ws", (ws.numel(),) if isinstance(ws, torch.Tensor) else (), torch.uint8), ws.numel()
        if size == 0:
            return None, 0
        if _capturing():
            ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        else:
            ws = self.workspace((key, stream), size)
        return ws.data_ptr(), ws.numel()

    def _out(self, t, name, shape, dtype):
        """(tensor, address, row distance) of an output, made if it is not given."""
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=self.device)
        return (t,) + self._rows(t, name, shape, dtype)

    def _rotate_inputs(self, desc, q, k, gamma_q, gamma_k, pos, freq):
        if q is None and k is None:
            raise DsmpError(INVALID_ARG, "queries or keys are needed")
        n, dt, hd = (k if q is None else q).shape[0], _TORCH.get(desc.dtype), desc.head_dim
        qs, ks = (n, desc.heads * hd), (n, desc.kv_heads * hd)
        qp = (None, 0) if q is None else self._rows(q, "q", qs, dt)
        kp = (None, 0) if k is None else self._rows(k, "k", ks, dt)
        rest = [None if gamma_q is None else self._flat(gamma_q, "gamma_q", (hd,)),
                None if gamma_k is None else self._flat(gamma_k, "gamma_k", (hd,)),
                None if not desc.rot else self._flat(pos, "pos", (n, desc.axes)),
                None if not desc.rot else self._flat(freq, "freq", (desc.rot // 2,))]
        return n, dt, qs, ks, [*qp, *kp, *rest]

    def dsmp_qk_rotate_forward(self, desc: RotateDesc, q, k, gamma_q=None, gamma_k=None, pos=None, freq=None,
                               q_out=None, k_out=None):
        """Queries [n, heads * head_dim] and keys [n, kv_heads * head_dim], each head normed and its pairs
        rotated by pos (float32 [n, axes]) times freq (float32 [rot / 2], see rotary_frequencies); returns
        (q_out, k_out).  q or k may be None; an output may be its own input."""
        n, dt, qs, ks, args = self._rotate_inputs(desc, q, k, gamma_q, gamma_k, pos, freq)
        q_out, qo, ldqo = (None, None, 0) if q is None else self._out(q_out, "q_out", qs, dt)
        k_out, ko, ldko = (None, None, 0) if k is None else self._out(k_out, "k_out", ks, dt)
        self._bind_current()
        st = self.lib.dsmp_qk_rotate_forward(self.h, desc, n, *args, qo, ldqo, ko, ldko)
        if st:
            self._check(st, self.h)
        return q_out, k_out

    def dsmp_qk_rotate_workspace(self, desc: RotateDesc, n: int) -> int:
        """Bytes of scratch that dsmp_qk_rotate_backward needs (its ws)."""
        nb = ctypes.c_size_t()
        self._check(self.lib.dsmp_qk_rotate_workspace(desc, n, ctypes.byref(nb)), None)
        return nb.value

    def dsmp_qk_rotate_backward(self, desc: RotateDesc, q, k, gamma_q, gamma_k, pos, freq, grad_q_out, grad_k_out,
                                grad_q=None, grad_k=None, grads: Optional[dict] = None, flags: int = 0, ws=None):
        """Gradients of the forward call with these inputs; returns (grad_q, grad_k, {"dgamma_q", "dgamma_k"}
        for the gammas given).  grad_q and grad_k may be the gradients that come in.  ws: scratch of the
        caller's own (uint8), needed in a capture that torch.cuda.graph does not make."""
        n, dt, qs, ks, args = self._rotate_inputs(desc, q, k, gamma_q, gamma_k, pos, freq)
        gqo = (None, 0) if q is None else self._rows(grad_q_out, "grad_q_out", qs, dt)
        gko = (None, 0) if k is None else self._rows(grad_k_out, "grad_k_out", ks, dt)
        grad_q, gq, ldgq = (None, None, 0) if q is None else self._out(grad_q, "grad_q", qs, dt)
        grad_k, gk, ldgk = (None, None, 0) if k is None else self._out(grad_k, "grad_k", ks, dt)
        out, dg = {}, []
        for name, gamma in (("dgamma_q", gamma_q), ("dgamma_k", gamma_k)):
            if gamma is None:
                dg.append(None)
                continue
            out[name] = torch.empty_like(gamma) if grads is None else grads[name]
            dg.append(self._flat(out[name], name, (desc.head_dim,)))
        size = self.dsmp_qk_rotate_workspace(desc, n) if out else 0
        wp, wb = self._scratch("rotate", size, ws)
        st = self.lib.dsmp_qk_rotate_backward(self.h, desc, n, *args, *gqo, *gko, gq, ldgq, gk, ldgk, *dg, flags, wp, wb)
        if st:
            self._check(st, self.h)
        return grad_q, grad_k, out

    def _attn_size(self, desc, qs, ks):
        key = (bytes(desc), qs.n, qs.n_seg, ks.n, ks.n_seg)   # the cuts depend on type, distance and cap too
        sizes = self._attn_sizes.get(key)
        if sizes is None:
            f, b = ctypes.c_size_t(), ctypes.c_size_t()
            self._check(self.lib.dsmp_attention_workspace(desc, qs, ks, ctypes.byref(f), ctypes.byref(b)), None)
            if len(self._attn_sizes) >= 1024:
                self._attn_sizes.clear()
            sizes = self._attn_sizes[key] = (f.value, b.value)
        return sizes

    def _attn_inputs(self, desc, q, k, v, segments, k_segments, pos, k_pos, slopes):
        nq, nk, dt, hd = q.shape[0], k.shape[0], _TORCH.get(desc.dtype), desc.head_dim
        qshape, kshape = (nq, desc.heads * hd), (nk, desc.kv_heads * hd)
        args = [*self._rows(q, "q", qshape, dt), *self._rows(k, "k", kshape, dt), *self._rows(v, "v", kshape, dt)]
        if desc.dim > 0:
            k_pos = pos if k_pos is None else k_pos
            args += [self._flat(pos, "pos", (nq, desc.dim)), self._flat(k_pos, "k_pos", (nk, desc.dim)),
                     self._flat(slopes, "slopes", (desc.heads,))]
        else:
            args += [None, None, None]
        qs = self._segments(nq, segments)
        return nq, dt, qshape, kshape, qs, self._segments(nk, segments if k_segments is None else k_segments), args

    def dsmp_attention_workspace(self, desc: AttentionDesc, n: int, n_keys: int, segments=None, k_segments=None):
        """Bytes of scratch that dsmp_attention_forward and _backward need (their ws): (forward, backward)."""
        return self._attn_size(desc, self._segments(n, segments),
                               self._segments(n_keys, segments if k_segments is None else k_segments))

    def dsmp_attention_forward(self, desc: AttentionDesc, q, k, v, segments=None, k_segments=None, pos=None, k_pos=None,
                               slopes=None, out=None, lse=None, ws=None):
        """Attention of the queries q [n, heads * head_dim] to the keys and values k, v [n_keys, kv_heads *
        head_dim] of their own segment; returns (out, lse).

        segments, k_segments: of the queries and of the keys, as for the norms (k_segments None: the
        queries'), with rows in front of the first and behind the last bound left alone.  pos, k_pos: float32
        [n, dim], [n_keys, dim] (k_pos None: pos), slopes float32 [heads], where the descriptor's dim is not
        0.  ws: scratch of the caller's own (uint8, dsmp_attention_workspace), needed in a capture that
        torch.cuda.graph does not make."""
        nq, dt, qshape, _, qs, ks, args = self._attn_inputs(desc, q, k, v, segments, k_segments, pos, k_pos, slopes)
        out, op, ldo = self._out(out, "out", qshape, dt)
        lse = torch.empty(nq, desc.heads, dtype=torch.float32, device=self.device) if lse is None else lse
        lp = self._flat(lse, "lse", (nq, desc.heads))
        wp, wb = self._scratch("attention", self._attn_size(desc, qs, ks)[0], ws)
        st = self.lib.dsmp_attention_forward(self.h, desc, qs, ks, *args, op, ldo, lp, wp, wb)
        if st:
            self._check(st, self.h)
        return out, lse

    def dsmp_attention_backward(self, desc: AttentionDesc, q, k, v, out, lse, grad_out, segments=None, k_segments=None,
                                pos=None, k_pos=None, slopes=None, grad_q=None, grad_k=None, grad_v=None, ws=None):
        """Gradients with respect to q, k and v of the forward call that returned out and lse; returns
        (grad_q, grad_k, grad_v), of the matrices' own type.  Rows of no segment are left alone here too: in
        a tensor that the call makes they are not set."""
        nq, dt, qshape, kshape, qs, ks, args = self._attn_inputs(desc, q, k, v, segments, k_segments, pos, k_pos, slopes)
        args += [*self._rows(out, "out", qshape, dt), self._flat(lse, "lse", (nq, desc.heads)),
                 *self._rows(grad_out, "grad_out", qshape, dt)]
        grad_q, gq, ldgq = self._out(grad_q, "grad_q", qshape, dt)
        grad_k, gk, ldgk = self._out(grad_k, "grad_k", kshape, dt)
        grad_v, gv, ldgv = self._out(grad_v, "grad_v", kshape, dt)
        wp, wb = self._scratch("attention", self._attn_size(desc, qs, ks)[1], ws)
        st = self.lib.dsmp_attention_backward(self.h, desc, qs, ks, *args, gq, ldgq, gk, ldgk, gv, ldgv, wp, wb)
        if st:
            self._check(st, self.h)
        return grad_q, grad_k, grad_v
