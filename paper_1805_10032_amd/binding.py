"""ctypes binding of the Zeno HIP library (include/zeno.h).

Argument marshalling only: every function takes torch tensors that already
live on the GPU, passes their device pointers and the current HIP stream to
the C entry point of the same name, and returns the output tensors.  There is
no CPU fallback: a missing library or a tensor on the wrong device raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ZENO_HIP_LIB") or os.path.join(_HERE, "lib", "libzeno_hip.so")

ZENO_MAX_LAYERS = 8
ZENO_MAX_CANDIDATES = 1024
LOSS = {"squared": 0, "softmax_ce": 1}
FWD = {"fp32": 0, "bf16": 1}
STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported size", 3: "workspace", 4: "device", 5: "host memory"}

EXPORTS = ["zeno_model_create", "zeno_cnn_model_create", "zeno_model_destroy", "zeno_model_num_params",
           "zeno_score_workspace_bytes", "zeno_score", "zeno_score_static", "zeno_aggregate", "zeno_aggregate_update", "zeno_mean",
           "zeno_median", "zeno_krum_workspace_bytes", "zeno_krum", "zeno_status_string", "zeno_profile_enable", "zeno_profile_collect",
           "zeno_score_plan_check", "zeno_logprobs_workspace_bytes", "zeno_logprobs", "zeno_logprobs_backward", "zeno_checkpoint",
           "zeno_checkpoint_values", "zeno_layer_norm", "zeno_layer_norm_workspace_bytes", "zeno_layer_norm_backward",
           "zeno_weight_gradient_workspace_bytes", "zeno_weight_gradient", "zeno_score_logprobs_workspace_bytes",
           "zeno_score_logprobs", "zeno_embedding", "zeno_embedding_workspace_bytes", "zeno_embedding_backward",
           "zeno_linear_logprobs_workspace_bytes", "zeno_linear_logprobs", "zeno_linear_logprobs_backward_workspace_bytes",
           "zeno_linear_logprobs_backward"]

KERNEL_NAMES = ["pack", "layer_base", "layer_cand", "loss", "combine", "average", "mean", "median", "average_update",
                "krum", "conv_base", "conv_cand", "aux", "logprobs", "logprobs_grad", "layer_norm", "layer_norm_grad", "checkpoint",
                "weight_grad", "score_logprobs", "embedding", "embedding_grad", "linear_logprobs",
                "linear_logprobs_grad"]
ZENO_MAX_CONV = 8
ZENO_MAX_TOP = 32
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class ZenoError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: status {status} ({STATUS.get(int(status), '?')})")


class _ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32),
                ("dims", ctypes.c_int32 * (ZENO_MAX_LAYERS + 1)),
                ("has_bias", ctypes.c_int32),
                ("loss", ctypes.c_int32),
                ("fwd", ctypes.c_int32)]


class _CnnDesc(ctypes.Structure):
    _fields_ = [("in_h", ctypes.c_int32), ("in_w", ctypes.c_int32), ("in_c", ctypes.c_int32),
                ("n_conv", ctypes.c_int32),
                ("conv_c", ctypes.c_int32 * ZENO_MAX_CONV),
                ("conv_stride", ctypes.c_int32 * ZENO_MAX_CONV),
                ("fc_out", ctypes.c_int32), ("has_bias", ctypes.c_int32), ("loss", ctypes.c_int32)]


class _ProfileRecord(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("layer", ctypes.c_int32), ("ms", ctypes.c_float),
                ("algorithmic_bytes", ctypes.c_double), ("waves", ctypes.c_int32), ("k_split", ctypes.c_int32),
                ("streaming", ctypes.c_int32), ("row_blocks", ctypes.c_int32), ("merged", ctypes.c_int32),
                ("second", ctypes.c_int32), ("k_slices", ctypes.c_int32),
                ("candidates", ctypes.c_int32),
                ("tail_candidates", ctypes.c_int32)]


class _Batch(ctypes.Structure):
    _fields_ = [("n_r", ctypes.c_int32),
                ("features", ctypes.c_void_p),
                ("labels", ctypes.c_void_p),
                ("targets", ctypes.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it with `python -m paper_1805_10032_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.zeno_model_create.argtypes = [ctypes.POINTER(_ModelDesc), ctypes.POINTER(vp)]
    lib.zeno_model_create.restype = ctypes.c_int
    lib.zeno_cnn_model_create.argtypes = [ctypes.POINTER(_CnnDesc), ctypes.POINTER(vp)]
    lib.zeno_cnn_model_create.restype = ctypes.c_int
    lib.zeno_model_destroy.argtypes = [vp]
    lib.zeno_model_destroy.restype = None
    lib.zeno_model_num_params.argtypes = [vp]
    lib.zeno_model_num_params.restype = i64
    lib.zeno_score_workspace_bytes.argtypes = [vp, i32, i32]
    lib.zeno_score_workspace_bytes.restype = ctypes.c_size_t
    lib.zeno_score.argtypes = [vp, vp, vp, i64, i32, ctypes.POINTER(_Batch), f32, f32, vp, vp,
                               ctypes.c_size_t, vp]
    lib.zeno_score.restype = ctypes.c_int
    lib.zeno_score_static.argtypes = [vp, vp, vp, i64, i32, ctypes.POINTER(_Batch), f32, f32, vp, vp]
    lib.zeno_score_static.restype = ctypes.c_int
    lib.zeno_aggregate.argtypes = [vp, i64, vp, i32, i64, i32, vp, vp, vp]
    lib.zeno_aggregate.restype = ctypes.c_int
    lib.zeno_aggregate_update.argtypes = [vp, i64, vp, i32, i64, i32, f32, vp, vp, vp, vp, vp]
    lib.zeno_aggregate_update.restype = ctypes.c_int
    lib.zeno_mean.argtypes = [vp, i64, i32, i64, vp, vp]
    lib.zeno_mean.restype = ctypes.c_int
    lib.zeno_median.argtypes = [vp, i64, i32, i64, vp, vp]
    lib.zeno_median.restype = ctypes.c_int
    lib.zeno_krum_workspace_bytes.argtypes = [i32]
    lib.zeno_krum_workspace_bytes.restype = ctypes.c_size_t
    lib.zeno_krum.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.zeno_krum.restype = ctypes.c_int
    lib.zeno_score_plan_check.argtypes = [vp, i32, i32]
    lib.zeno_score_plan_check.restype = ctypes.c_int
    size = ctypes.c_size_t
    for name, res, args in [
            ("zeno_logprobs_workspace_bytes", size, [i32, i32, i32]),
            ("zeno_logprobs", ctypes.c_int, [vp, i64, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, size, vp]),
            ("zeno_logprobs_backward", ctypes.c_int, [vp, i64, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, i64, vp]),
            ("zeno_checkpoint", ctypes.c_int, [vp, i64, i32, i32, i32, vp, vp, vp]),
            ("zeno_checkpoint_values", ctypes.c_int, [vp, vp, i32, i32, i32, vp, i64, vp]),
            ("zeno_layer_norm", ctypes.c_int, [vp, i64, i32, i32, i32, vp, vp, f32, vp, i64, vp, vp, vp, vp, vp]),
            ("zeno_layer_norm_workspace_bytes", size, [i32, i32, i32]),
            ("zeno_layer_norm_backward", ctypes.c_int,
             [vp, i64, i32, i32, i32, vp, i64, vp, vp, vp, vp, vp, i32, vp, vp, i64, vp, i64, vp, i64, vp, size, vp]),
            ("zeno_weight_gradient_workspace_bytes", size, [i32, i32, i32, i32]),
            ("zeno_weight_gradient", ctypes.c_int, [vp, i64, i32, i32, i32, vp, vp, i32, i32, vp, vp, i64, vp, i64, vp, size, vp]),
            ("zeno_score_logprobs_workspace_bytes", size, [i32, i64]),
            ("zeno_score_logprobs", ctypes.c_int, [vp, i64, i32, i64, vp, vp, i64, i32, vp, f32, vp, vp, size, vp]),
            ("zeno_embedding", ctypes.c_int, [vp, i64, i32, i32, i32, vp, i32, f32, vp, i64, i32, vp]),
            ("zeno_embedding_workspace_bytes", size, [i32, i32, i32, i32]),
            ("zeno_embedding_backward", ctypes.c_int, [vp, i64, i32, i32, i32, vp, i32, f32, i32, vp, i32, vp, i64, vp, size, vp]),
            ("zeno_linear_logprobs_workspace_bytes", size, [i32, i32, i32, i32]),
            ("zeno_linear_logprobs", ctypes.c_int, [vp, i64, vp, i64, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, size, vp]),
            ("zeno_linear_logprobs_backward_workspace_bytes", size, [i32, i32, i32, i32, i32]),
            ("zeno_linear_logprobs_backward", ctypes.c_int, [vp, i64, vp, i64, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, i64,
                                                             vp, i64, vp, i64, vp, size, vp])]:
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, res
    lib.zeno_profile_enable.argtypes = [i32]
    lib.zeno_profile_enable.restype = ctypes.c_int
    lib.zeno_profile_collect.argtypes = [ctypes.POINTER(_ProfileRecord), i32]
    lib.zeno_profile_collect.restype = i32
    lib.zeno_status_string.argtypes = [ctypes.c_int]
    lib.zeno_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


# torch.cuda.current_stream() builds a Stream object, 2.8 us of the 10 us that the host spends on a call, and the smallest calls
# are bound by the host (64 -> 1, eight candidates, score and update: 19.9 -> 14.7 us); the raw handle takes 0.2.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return int(torch.cuda.current_stream().cuda_stream)
    return int(_raw_stream(torch.cuda.current_device()))


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(G: torch.Tensor):
    """(pointer, ldg) of a candidate matrix: rows contiguous, ldg >= d floats apart
    (a column slice of a wider allocation is accepted as it is, nothing is copied)."""
    if not isinstance(G, torch.Tensor) or not G.is_cuda or G.dtype != torch.float32 or G.dim() != 2:
        raise ValueError("G must be a 2-D float32 CUDA/HIP tensor")
    m, d = G.shape
    if d > 1 and G.stride(1) != 1:
        raise ValueError("the rows of G must be contiguous")
    ldg = int(G.stride(0)) if m > 1 else int(d)
    if ldg < d:
        raise ValueError("the rows of G overlap")
    return G.data_ptr(), ldg


def candidate_pitch(d: int, align: int = 32) -> int:
    """Row pitch in floats for an [m x d] candidate matrix: d rounded up to `align` floats, and, for
    line-aligned layouts (align a multiple of 32 floats = 128 bytes), to an ODD number of 128-byte
    lines.  With an even number of lines the rows of all candidates start at the same offset modulo
    256 bytes, and the workgroups that stream the same columns of 16 candidates at the same time then
    lean on the same memory channels (measured on the 14 GB workload: 2 % slower)."""
    align = max(1, int(align))
    ldg = (int(d) + align - 1) // align * align
    if align % 32 == 0 and (ldg // 32) % 2 == 0:
        ldg += 32
    return ldg


def alloc_candidates(m: int, d: int, device=None, align: int = 32) -> torch.Tensor:
    """An [m x d] float32 view whose rows start `align`-float (128-byte) aligned, an odd number of
    128-byte lines apart: the layout the streaming kernels are fastest on."""
    buf = torch.empty((int(m), candidate_pitch(d, align)), dtype=torch.float32,
                      device=device or torch.device("cuda", torch.cuda.current_device()))
    return buf[:, :int(d)]


class ZenoModel:
    """Host-side model handle (zeno_model_create / zeno_model_destroy)."""

    def __init__(self, dims, has_bias=True, loss="softmax_ce", fwd="fp32"):
        lib = load_library()
        desc = _ModelDesc()
        if not 2 <= len(dims) <= ZENO_MAX_LAYERS + 1:
            raise ZenoError(1, "ZenoModel")
        desc.n_layers = len(dims) - 1
        for i, v in enumerate(dims):
            desc.dims[i] = int(v)
        desc.has_bias = int(bool(has_bias))
        desc.loss = LOSS[loss]
        desc.fwd = FWD[fwd]
        handle = ctypes.c_void_p()
        st = lib.zeno_model_create(ctypes.byref(desc), ctypes.byref(handle))
        if st != 0:
            raise ZenoError(st, "zeno_model_create")
        self._lib = lib
        self._h = handle
        self.dims, self.has_bias, self.loss, self.fwd = list(dims), bool(has_bias), loss, fwd

    @property
    def num_params(self) -> int:
        return int(self._lib.zeno_model_num_params(self._h))

    def workspace_bytes(self, m: int, n_r: int) -> int:
        return int(self._lib.zeno_score_workspace_bytes(self._h, int(m), int(n_r)))

    def plan_check(self, m: int, n_r: int) -> int:
        """Status of the host-side check that every launch of zeno_score stays inside its workspace slots."""
        return int(self._lib.zeno_score_plan_check(self._h, int(m), int(n_r)))

    def close(self):
        if self._h is not None and self._h.value:
            self._lib.zeno_model_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ZenoCnnModel(ZenoModel):
    """Handle of a convolutional model (zeno_cnn_model_create): desc = dict(in_h, in_w, in_c, conv_c=[...],
    conv_stride=[...], fc_out, has_bias); fp32 forward."""

    def __init__(self, desc, loss="softmax_ce"):
        lib = load_library()
        cd = _CnnDesc()
        cd.in_h, cd.in_w, cd.in_c = int(desc["in_h"]), int(desc["in_w"]), int(desc["in_c"])
        conv_c, conv_stride = list(desc["conv_c"]), list(desc["conv_stride"])
        if not (1 <= len(conv_c) <= ZENO_MAX_CONV) or len(conv_c) != len(conv_stride):
            raise ZenoError(1, "ZenoCnnModel")
        cd.n_conv = len(conv_c)
        for i, (c, s) in enumerate(zip(conv_c, conv_stride)):
            cd.conv_c[i], cd.conv_stride[i] = int(c), int(s)
        cd.fc_out = int(desc["fc_out"])
        cd.has_bias = int(bool(desc["has_bias"]))
        cd.loss = LOSS[loss]
        handle = ctypes.c_void_p()
        st = lib.zeno_cnn_model_create(ctypes.byref(cd), ctypes.byref(handle))
        if st != 0:
            raise ZenoError(st, "zeno_cnn_model_create")
        self._lib = lib
        self._h = handle
        self.desc = dict(desc)
        self.dims = [cd.in_h * cd.in_w * cd.in_c, cd.fc_out]      # input width of a sample, output width
        self.has_bias, self.loss, self.fwd = bool(desc["has_bias"]), loss, "fp32"


def alloc_workspace(model: ZenoModel, m: int, n_r: int, device=None) -> torch.Tensor:
    """A byte tensor of the size zeno_score asks for (torch's allocator returns
    at least 256-byte aligned blocks)."""
    n = model.workspace_bytes(m, n_r)
    if n == 0:
        raise ZenoError(1, "zeno_score_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device or torch.device("cuda", torch.cuda.current_device()))


def zeno_score(model: ZenoModel, x, G, features, gamma, rho, *, labels=None, targets=None,
               scores=None, workspace=None):
    """scores[i] = f_r(x) - f_r(x - gamma G[i]) - rho ||G[i]||^2  (Definition 2)."""
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if d != model.num_params or x.numel() != d:
        raise ValueError("x / G do not match the model's parameter count")
    n_r = int(features.shape[0])
    if features.shape[1] != model.dims[0]:
        raise ValueError("features do not match the model's input width")
    batch = _Batch()
    batch.n_r = n_r
    batch.features = _dev(features, torch.float32, "features")
    batch.labels = _dev(labels, torch.int32, "labels") if labels is not None else None
    batch.targets = _dev(targets, torch.float32, "targets") if targets is not None else None
    if scores is None:
        scores = torch.empty(m, dtype=torch.float32, device=G.device)
    if workspace is None:
        workspace = alloc_workspace(model, m, n_r, G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_score(model._h, _dev(x, torch.float32, "x"), g_ptr, ldg, m,
                        ctypes.byref(batch), float(gamma), float(rho),
                        _dev(scores, torch.float32, "scores"),
                        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    if st != 0:
        raise ZenoError(st, "zeno_score")
    return scores


STATIC_SCRATCH_BYTES = 32 << 20


def zeno_score_static(model: ZenoModel, x, G, features, gamma, rho, *, labels=None, targets=None, scores=None):
    """zeno_score on the library's static scratch array: no workspace, nothing allocated by the call
    (pass `scores` to keep the binding from allocating the output either)."""
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if d != model.num_params or x.numel() != d:
        raise ValueError("x / G do not match the model's parameter count")
    if features.shape[1] != model.dims[0]:
        raise ValueError("features do not match the model's input width")
    batch = _Batch()
    batch.n_r = int(features.shape[0])
    batch.features = _dev(features, torch.float32, "features")
    batch.labels = _dev(labels, torch.int32, "labels") if labels is not None else None
    batch.targets = _dev(targets, torch.float32, "targets") if targets is not None else None
    if scores is None:
        scores = torch.empty(m, dtype=torch.float32, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_score_static(model._h, _dev(x, torch.float32, "x"), g_ptr, ldg, m, ctypes.byref(batch),
                               float(gamma), float(rho), _dev(scores, torch.float32, "scores"), _stream())
    if st != 0:
        raise ZenoError(st, "zeno_score_static")
    return scores


def zeno_aggregate(G, scores, b, *, out=None, selected=None, want_selected=True):
    """Zeno_b: mean of the m-b highest-scoring rows (Definition 3).  Returns (out, selected)."""
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=G.device)
    if selected is None and want_selected and 0 <= b < m:
        selected = torch.empty(m - b, dtype=torch.int32, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_aggregate(g_ptr, ldg, _dev(scores, torch.float32, "scores"), m, d, int(b),
                            _dev(out, torch.float32, "out"),
                            _dev(selected, torch.int32, "selected") if selected is not None else None,
                            _stream())
    if st != 0:
        raise ZenoError(st, "zeno_aggregate")
    return out, selected


def zeno_aggregate_update(G, scores, b, gamma, x, *, x_next=None, out=None, want_out=True, selected=None,
                          want_selected=True):
    """Zeno_b and the server's SGD step in one pass: x_next = x - gamma * Zeno_b(G)
    (Algorithm 1, server side).  x_next=x updates in place.  Returns (x_next, out, selected)."""
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if x.numel() != d:
        raise ValueError("x does not match the width of G")
    if x_next is None:
        x_next = torch.empty(d, dtype=torch.float32, device=G.device)
    if out is None and want_out:
        out = torch.empty(d, dtype=torch.float32, device=G.device)
    if selected is None and want_selected and 0 <= b < m:
        selected = torch.empty(m - b, dtype=torch.int32, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_aggregate_update(g_ptr, ldg, _dev(scores, torch.float32, "scores"), m, d, int(b), float(gamma),
                                   _dev(x, torch.float32, "x"), _dev(x_next, torch.float32, "x_next"),
                                   _dev(out, torch.float32, "out") if out is not None else None,
                                   _dev(selected, torch.int32, "selected") if selected is not None else None,
                                   _stream())
    if st != 0:
        raise ZenoError(st, "zeno_aggregate_update")
    return x_next, out, selected


def zeno_mean(G, *, out=None):
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_mean(g_ptr, ldg, m, d, _dev(out, torch.float32, "out"), _stream())
    if st != 0:
        raise ZenoError(st, "zeno_mean")
    return out


def zeno_median(G, *, out=None):
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_median(g_ptr, ldg, m, d, _dev(out, torch.float32, "out"), _stream())
    if st != 0:
        raise ZenoError(st, "zeno_median")
    return out


def zeno_krum(G, b, *, out=None, want_scores=True, workspace=None):
    """Krum_b (Definition 5).  Returns (out, chosen index tensor [1], krum scores or None)."""
    lib = load_library()
    m, d = int(G.shape[0]), int(G.shape[1])
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=G.device)
    chosen = torch.empty(1, dtype=torch.int32, device=G.device)
    ks = torch.empty(m, dtype=torch.float32, device=G.device) if want_scores else None
    if workspace is None:
        n = int(lib.zeno_krum_workspace_bytes(m))
        workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=G.device)
    g_ptr, ldg = _rows(G)
    st = lib.zeno_krum(g_ptr, ldg, m, d, int(b), _dev(out, torch.float32, "out"), _dev(chosen, torch.int32, "chosen"),
                       _dev(ks, torch.float32, "krum_scores") if ks is not None else None,
                       _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    if st != 0:
        raise ZenoError(st, "zeno_krum")
    return out, chosen, ks


# ---- models that answer with tokens

class Checkpoint(NamedTuple):
    """Activations [rows x width] in 8 bits: e4m3 values [rows x 32 ceil(width/32)] and, for every 32 columns, the byte of a scale
    2^(byte - 127), both uint8 and contiguous."""
    values: torch.Tensor
    scales: torch.Tensor
    width: int


# Small calls are bound by the host: the current device is asked for once a call, and only tensors that the caller handed over are
# looked at.
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _elsewhere(t, name: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor")
    raise ValueError(f"{name} is on {t.device}, not on the current device")


def _current(t, name: str) -> int:
    """The current device's index, for the first tensor of a call; its others are compared with it."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _elsewhere(t, name)
    dev = _device()
    if t.get_device() != dev:
        _elsewhere(t, name)
    return dev


def _vec(t, dtype, name: str, shape, dev: int):
    """Device pointer of a contiguous tensor of the given shape on the current device, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != dev:
        _elsewhere(t, name)
    if t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# The C calls take sizes in 32 bits: a larger one would arrive there as another size.
_MOST = (1 << 31) - 1


def _size32(where: str, *sizes):
    if any(abs(n) > _MOST for n in sizes):
        raise ZenoError(2, where)
    return sizes


def _matrix(t, name: str, dev: int, shape=None, dtype=None, most=_MOST):
    """(pointer, pitch, dtype code, rows, columns) of a 2-D matrix whose rows are contiguous and do not overlap."""
    if not isinstance(t, torch.Tensor) or t.get_device() != dev:
        _elsewhere(t, name)
    code = DTYPE.get(t.dtype)
    if code is None or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must have dtype {dtype or list(DTYPE)}, got {t.dtype}")
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise ValueError(f"{name} must be a matrix of shape {tuple(shape) if shape is not None else '(rows, columns)'}, "
                         f"got {tuple(size)}")
    rows, cols = size
    if rows > _MOST or cols > most:
        raise ZenoError(2, name)
    pitch, inner = t.stride()
    if cols > 1 and inner != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    if rows <= 1:
        pitch = cols
    if pitch < cols:
        raise ValueError(f"the rows of {name} overlap")
    return t.data_ptr(), pitch, code, rows, cols


def _grad_rows(t, name: str, m: int, n: int, dev: int):
    """(pointer, pitch) of m rows of n float32 gradients: columns of G, or a tensor of its own.  (n does not go to the call: a layer may
    have more weights than 32 bits count.)"""
    if t is None:
        return None, n
    ptr, pitch, _, _, _ = _matrix(t, name, dev, (m, n), torch.float32, n)
    return ptr, pitch


def _kept(ckpt, rows: int, width: int, dev: int):
    """Device pointers of a Checkpoint of [rows x width] activations."""
    if not isinstance(ckpt, Checkpoint) or ckpt.width != width:
        raise ValueError(f"a Checkpoint of {width} columns is needed")
    if width > _MOST:
        raise ZenoError(2, "Checkpoint")
    blocks = (width + 31) // 32
    return _vec(ckpt.values, torch.uint8, "values", (rows, 32 * blocks), dev), _vec(ckpt.scales, torch.uint8, "scales", (rows, blocks), dev)


def _groups(groups, dev: int):
    """(m, device pointer) of the row offsets [m + 1] of m workers; None: one group."""
    if groups is None:
        return 1, None
    if not isinstance(groups, torch.Tensor) or groups.dim() != 1 or groups.numel() < 2:
        raise ValueError("groups must hold the m + 1 row offsets of the workers")
    if groups.numel() > _MOST:
        raise ZenoError(2, "groups")
    return groups.numel() - 1, _vec(groups, torch.int32, "groups", groups.shape, dev)


def _scratch(workspace, dev: int):
    """(pointer, bytes) of a workspace."""
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev:
        _elsewhere(workspace, "workspace")
    return _dev(workspace, torch.uint8, "workspace"), workspace.numel()


def _workspace(n: int, where: str, device=None) -> torch.Tensor:
    if n == 0:
        raise ZenoError(1, where)
    return torch.empty(n, dtype=torch.uint8, device=device or torch.device("cuda", torch.cuda.current_device()))


def alloc_logprobs_workspace(rows: int, vocab: int, top: int = 0, device=None) -> torch.Tensor:
    sizes = _size32("zeno_logprobs_workspace_bytes", int(rows), int(vocab), int(top))
    return _workspace(int(load_library().zeno_logprobs_workspace_bytes(*sizes)), "zeno_logprobs_workspace_bytes", device)


def zeno_logprobs(logits, labels=None, *, top=0, want_entropy=False, want_stats=False, logp=None, entropy=None, stats=None,
                  top_index=None, top_logp=None, workspace=None):
    """Log probabilities of the labels (int32 [rows]; -1: does not count, 0 is written), entropy and the `top` most probable
    tokens of the rows of logits.  Returns (logp, entropy, stats, top_index, top_logp), None where not wanted; `stats`
    [rows x 2] is what zeno_logprobs_backward takes."""
    lib = load_library()
    dev = _current(logits, "logits")
    ptr, pitch, code, rows, vocab = _matrix(logits, "logits", dev)
    top, f32, i32, new = int(top), torch.float32, torch.int32, logits.new_empty
    if abs(top) > _MOST:
        raise ZenoError(2, "zeno_logprobs")

    def out(t, want, shape, dtype, name):
        if t is not None:
            return t, _vec(t, dtype, name, shape, dev)
        if not want:
            return None, None
        t = new(shape, dtype=dtype)
        return t, t.data_ptr()

    logp, logp_p = out(logp, labels is not None, (rows,), f32, "logp")
    entropy, entropy_p = out(entropy, want_entropy, (rows,), f32, "entropy")
    stats, stats_p = out(stats, want_stats, (rows, 2), f32, "stats")
    if top > 0:
        top_index, index_p = out(top_index, True, (rows, top), i32, "top_index")
        top_logp, top_p = out(top_logp, True, (rows, top), f32, "top_logp")
    else:
        top_index = top_logp = index_p = top_p = None
    if workspace is None:
        workspace = alloc_logprobs_workspace(rows, vocab, top, logits.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_logprobs(ptr, pitch, code, rows, vocab, _vec(labels, i32, "labels", (rows,), dev), logp_p, entropy_p, stats_p, top,
                           index_p, top_p, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_logprobs")
    return logp, entropy, stats, top_index, top_logp


def zeno_logprobs_backward(logits, stats, *, labels=None, grad_logp=None, entropy=None, grad_entropy=None, top_index=None,
                           grad_top=None, out=None):
    """Gradient of the logits from the gradients of logp [rows], of the entropy [rows] and of top_logp [rows x top], whichever
    are given.  out=logits works in place."""
    lib = load_library()
    dev = _current(logits, "logits")
    ptr, pitch, code, rows, vocab = _matrix(logits, "logits", dev)
    if out is None:
        out = logits.new_empty((rows, vocab))
    o_ptr, o_pitch, _, _, _ = _matrix(out, "out", dev, (rows, vocab), logits.dtype)
    f32, i32, top = torch.float32, torch.int32, 0
    if grad_top is not None:
        if not isinstance(grad_top, torch.Tensor) or grad_top.dim() != 2 or grad_top.shape[1] == 0:
            raise ValueError("grad_top must have shape (rows, top)")
        top = int(grad_top.shape[1])
    st = lib.zeno_logprobs_backward(ptr, pitch, code, rows, vocab, _vec(stats, f32, "stats", (rows, 2), dev),
                                    _vec(labels, i32, "labels", (rows,), dev), _vec(grad_logp, f32, "grad_logp", (rows,), dev),
                                    _vec(entropy, f32, "entropy", (rows,), dev),
                                    _vec(grad_entropy, f32, "grad_entropy", (rows,), dev), top,
                                    _vec(top_index, i32, "top_index", (rows, top), dev) if top else None,
                                    _vec(grad_top, f32, "grad_top", (rows, top), dev), o_ptr, o_pitch, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_logprobs_backward")
    return out


def alloc_checkpoint(rows: int, width: int, device=None) -> Checkpoint:
    device = device or torch.device("cuda", torch.cuda.current_device())
    blocks = (int(width) + 31) // 32
    return Checkpoint(torch.empty((int(rows), 32 * blocks), dtype=torch.uint8, device=device),
                      torch.empty((int(rows), blocks), dtype=torch.uint8, device=device), int(width))


def _new_checkpoint(x, rows: int, width: int) -> Checkpoint:
    blocks = (width + 31) // 32
    return Checkpoint(x.new_empty((rows, 32 * blocks), dtype=torch.uint8), x.new_empty((rows, blocks), dtype=torch.uint8), width)


def zeno_checkpoint(x, *, out=None) -> Checkpoint:
    """The activations x [rows x width] in 8 bits."""
    lib = load_library()
    dev = _current(x, "x")
    ptr, pitch, code, rows, width = _matrix(x, "x", dev)
    if out is None:
        out = _new_checkpoint(x, rows, width)
    v, s = _kept(out, rows, width, dev)
    st = lib.zeno_checkpoint(ptr, pitch, code, rows, width, v, s, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_checkpoint")
    return out


def zeno_checkpoint_values(ckpt: Checkpoint, dtype=torch.float32, *, out=None):
    """The values that a checkpoint holds, [rows x width] of the given type."""
    lib = load_library()
    if not isinstance(ckpt, Checkpoint):
        raise ValueError("a Checkpoint is needed")
    dev = _current(ckpt.values, "values")
    rows, width = int(ckpt.values.shape[0]), int(ckpt.width)
    if out is None:
        out = ckpt.values.new_empty((rows, width), dtype=dtype)
    ptr, pitch, code, _, _ = _matrix(out, "out", dev, (rows, width))
    v, s = _kept(ckpt, rows, width, dev)
    st = lib.zeno_checkpoint_values(v, s, rows, width, code, ptr, pitch, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_checkpoint_values")
    return out


def zeno_layer_norm(x, weight, bias=None, eps=1e-5, *, y=None, mean=None, rstd=None, want_checkpoint=False, checkpoint=None):
    """Layer norm of the rows of x; weight and bias float32 [width].  Returns (y, mean, rstd, Checkpoint of x or None)."""
    lib = load_library()
    dev = _current(x, "x")
    ptr, pitch, code, rows, width = _matrix(x, "x", dev)
    f32 = torch.float32
    if y is None:
        y = x.new_empty((rows, width))
    y_ptr, y_pitch, _, _, _ = _matrix(y, "y", dev, (rows, width), x.dtype)
    if mean is None:
        mean = x.new_empty((rows,), dtype=f32)
    if rstd is None:
        rstd = x.new_empty((rows,), dtype=f32)
    if want_checkpoint and checkpoint is None:
        checkpoint = _new_checkpoint(x, rows, width)
    v, s = (None, None) if checkpoint is None else _kept(checkpoint, rows, width, dev)
    st = lib.zeno_layer_norm(ptr, pitch, code, rows, width, _vec(weight, f32, "weight", (width,), dev), _vec(bias, f32, "bias", (width,), dev),
                             float(eps), y_ptr, y_pitch, _vec(mean, f32, "mean", (rows,), dev), _vec(rstd, f32, "rstd", (rows,), dev), v, s,
                             _stream())
    if st != 0:
        raise ZenoError(st, "zeno_layer_norm")
    return y, mean, rstd, checkpoint


def alloc_layer_norm_workspace(rows: int, width: int, m: int = 1, device=None) -> torch.Tensor:
    sizes = _size32("zeno_layer_norm_workspace_bytes", int(rows), int(width), int(m))
    return _workspace(int(load_library().zeno_layer_norm_workspace_bytes(*sizes)), "zeno_layer_norm_workspace_bytes", device)


def zeno_layer_norm_backward(dy, x, mean, rstd, weight, *, groups=None, want_dx=True, want_weight=True, want_bias=True, dx=None,
                             dweight=None, dbias=None, workspace=None):
    """Backward pass of zeno_layer_norm; x is its input or a Checkpoint of it.  groups: int32 row offsets [m + 1] of the m
    workers (None: one group).  dweight and dbias are [m x width] float32, for instance column slices of G.  dx=dy works in
    place; rows that belong to no group keep what dx held (zeros if dx is not given).  Returns (dx, dweight, dbias)."""
    lib = load_library()
    dev = _current(dy, "dy")
    ptr, pitch, code, rows, width = _matrix(dy, "dy", dev)
    f32 = torch.float32
    m, offsets = _groups(groups, dev)
    v = s = x_ptr = None
    x_pitch = width
    if isinstance(x, Checkpoint):
        v, s = _kept(x, rows, width, dev)
    else:
        x_ptr, x_pitch, _, _, _ = _matrix(x, "x", dev, (rows, width), dy.dtype)
    if want_dx and dx is None:
        dx = dy.new_empty((rows, width)) if groups is None else dy.new_zeros((rows, width))
    if want_weight and dweight is None:
        dweight = dy.new_empty((m, width), dtype=f32)
    if want_bias and dbias is None:
        dbias = dy.new_empty((m, width), dtype=f32)
    d_ptr, d_pitch = None, width
    if dx is not None:
        d_ptr, d_pitch, _, _, _ = _matrix(dx, "dx", dev, (rows, width), dy.dtype)
    w_ptr, ldw = _grad_rows(dweight, "dweight", m, width, dev)
    b_ptr, ldb = _grad_rows(dbias, "dbias", m, width, dev)
    if workspace is None:
        workspace = alloc_layer_norm_workspace(rows, width, m, dy.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_layer_norm_backward(ptr, pitch, code, rows, width, x_ptr, x_pitch, v, s, _vec(mean, f32, "mean", (rows,), dev),
                                      _vec(rstd, f32, "rstd", (rows,), dev), _vec(weight, f32, "weight", (width,), dev), m, offsets, d_ptr,
                                      d_pitch, w_ptr, ldw, b_ptr, ldb, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_layer_norm_backward")
    return dx, dweight, dbias


def alloc_weight_gradient_workspace(rows: int, out: int, width: int, m: int = 1, device=None) -> torch.Tensor:
    sizes = _size32("zeno_weight_gradient_workspace_bytes", int(rows), int(out), int(width), int(m))
    return _workspace(int(load_library().zeno_weight_gradient_workspace_bytes(*sizes)), "zeno_weight_gradient_workspace_bytes", device)


def zeno_weight_gradient(dy, ckpt: Checkpoint, *, groups=None, want_bias=True, dweight=None, dbias=None, workspace=None):
    """Gradient of a linear layer's weights (and bias) for each of the m workers, from dy [rows x out] and a Checkpoint of the
    layer's input.  dweight [m x out * width] and dbias [m x out] are float32, for instance column slices of G."""
    lib = load_library()
    dev = _current(dy, "dy")
    ptr, pitch, code, rows, out = _matrix(dy, "dy", dev)
    m, offsets = _groups(groups, dev)
    if not isinstance(ckpt, Checkpoint):
        raise ValueError("a Checkpoint is needed")
    width = int(ckpt.width)
    v, s = _kept(ckpt, rows, width, dev)
    if dweight is None:
        dweight = dy.new_empty((m, out * width), dtype=torch.float32)
    if want_bias and dbias is None:
        dbias = dy.new_empty((m, out), dtype=torch.float32)
    w_ptr, ldw = _grad_rows(dweight, "dweight", m, out * width, dev)
    b_ptr, ldb = _grad_rows(dbias, "dbias", m, out, dev)
    if workspace is None:
        workspace = alloc_weight_gradient_workspace(rows, out, width, m, dy.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_weight_gradient(ptr, pitch, code, rows, out, v, s, width, m, offsets, w_ptr, ldw, b_ptr, ldb, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_weight_gradient")
    return dweight, dbias


def _linear_workspace(where: str, dtype, device, *sizes):
    if dtype not in DTYPE:
        raise ValueError(f"dtype must be one of {list(DTYPE)}")
    rows, vocab, width, *m = _size32(where, *(int(n) for n in sizes))
    return _workspace(int(getattr(load_library(), where)(rows, vocab, width, DTYPE[dtype], *m)), where, device)


def alloc_linear_logprobs_workspace(rows: int, vocab: int, width: int, dtype=torch.bfloat16, device=None) -> torch.Tensor:
    return _linear_workspace("zeno_linear_logprobs_workspace_bytes", dtype, device, rows, vocab, width)


def alloc_linear_logprobs_backward_workspace(rows: int, vocab: int, width: int, dtype=torch.bfloat16, m: int = 1, device=None) -> torch.Tensor:
    return _linear_workspace("zeno_linear_logprobs_backward_workspace_bytes", dtype, device, rows, vocab, width, m)


def zeno_linear_logprobs(hidden, weight, bias=None, labels=None, *, want_entropy=False, want_stats=False, logp=None, entropy=None,
                         stats=None, workspace=None):
    """zeno_logprobs of the logits hidden weight^T + bias, which are never stored.  hidden [rows x width] and weight [vocab x width] of one
    dtype, bias float32 [vocab].  Returns (logp, entropy, stats), None where not wanted; `stats` [rows x 2] is what
    zeno_linear_logprobs_backward takes."""
    lib = load_library()
    dev = _current(hidden, "hidden")
    ptr, pitch, code, rows, width = _matrix(hidden, "hidden", dev)
    w_ptr, w_pitch, _, vocab, w_width = _matrix(weight, "weight", dev, None, hidden.dtype)
    if w_width != width:
        raise ValueError(f"weight must have {width} columns, got {w_width}")
    f32, new = torch.float32, hidden.new_empty

    def out(t, want, shape, name):
        if t is not None:
            return t, _vec(t, f32, name, shape, dev)
        if not want:
            return None, None
        t = new(shape, dtype=f32)
        return t, t.data_ptr()

    logp, logp_p = out(logp, labels is not None, (rows,), "logp")
    entropy, entropy_p = out(entropy, want_entropy, (rows,), "entropy")
    stats, stats_p = out(stats, want_stats, (rows, 2), "stats")
    if workspace is None:
        workspace = alloc_linear_logprobs_workspace(rows, vocab, width, hidden.dtype, hidden.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_linear_logprobs(ptr, pitch, w_ptr, w_pitch, code, _vec(bias, f32, "bias", (vocab,), dev), rows, vocab, width,
                                  _vec(labels, torch.int32, "labels", (rows,), dev), logp_p, entropy_p, stats_p, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_linear_logprobs")
    return logp, entropy, stats


def zeno_linear_logprobs_backward(hidden, weight, bias, stats, *, labels=None, grad_logp=None, entropy=None, grad_entropy=None, groups=None,
                                  want_hidden=True, want_weight=True, want_bias=True, dhidden=None, dweight=None, dbias=None,
                                  workspace=None):
    """Gradients of the hidden states and, for each of the m workers, of the weights and the bias, from the gradients of logp [rows] and of
    the entropy [rows].  dweight [m x vocab * width] and dbias [m x vocab] are float32, for instance column slices of G; dhidden=hidden
    works in place; rows that belong to no group keep what dhidden held (zeros if it is not given).  Returns (dhidden, dweight, dbias)."""
    lib = load_library()
    dev = _current(hidden, "hidden")
    ptr, pitch, code, rows, width = _matrix(hidden, "hidden", dev)
    w_ptr, w_pitch, _, vocab, w_width = _matrix(weight, "weight", dev, None, hidden.dtype)
    if w_width != width:
        raise ValueError(f"weight must have {width} columns, got {w_width}")
    m, offsets = _groups(groups, dev)
    f32 = torch.float32
    if want_hidden and dhidden is None:
        dhidden = hidden.new_empty((rows, width)) if groups is None else hidden.new_zeros((rows, width))
    if want_weight and dweight is None:
        dweight = hidden.new_empty((m, vocab * width), dtype=f32)
    if want_bias and dbias is None:
        dbias = hidden.new_empty((m, vocab), dtype=f32)
    d_ptr, d_pitch = None, width
    if dhidden is not None:
        d_ptr, d_pitch, _, _, _ = _matrix(dhidden, "dhidden", dev, (rows, width), hidden.dtype)
    g_ptr, ldg = _grad_rows(dweight, "dweight", m, vocab * width, dev)
    b_ptr, ldb = _grad_rows(dbias, "dbias", m, vocab, dev)
    if workspace is None:
        workspace = alloc_linear_logprobs_backward_workspace(rows, vocab, width, hidden.dtype, m, hidden.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_linear_logprobs_backward(ptr, pitch, w_ptr, w_pitch, code, _vec(bias, f32, "bias", (vocab,), dev), rows, vocab, width,
                                           _vec(stats, f32, "stats", (rows, 2), dev), _vec(labels, torch.int32, "labels", (rows,), dev),
                                           _vec(grad_logp, f32, "grad_logp", (rows,), dev), _vec(entropy, f32, "entropy", (rows,), dev),
                                           _vec(grad_entropy, f32, "grad_entropy", (rows,), dev), m, offsets, d_ptr, d_pitch, g_ptr, ldg,
                                           b_ptr, ldb, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_linear_logprobs_backward")
    return dhidden, dweight, dbias


def zeno_embedding(ids, table, dtype=None, *, scale=1.0, out=None):
    """scale * table[ids] as `dtype` (default: the table's).  ids int32 [rows] (-1: a row of zeros), table [vocab x width], for instance
    a block of a parameter vector."""
    lib = load_library()
    dev = _current(ids, "ids")
    if ids.dim() != 1 or ids.numel() > _MOST:
        raise ValueError("ids must be a vector")
    rows = int(ids.numel())
    ptr, pitch, code, vocab, width = _matrix(table, "table", dev)
    if out is None:
        out = table.new_empty((rows, width), dtype=dtype or table.dtype)
    o_ptr, o_pitch, o_code, _, _ = _matrix(out, "out", dev, (rows, width), dtype)
    st = lib.zeno_embedding(ptr, pitch, code, vocab, width, _vec(ids, torch.int32, "ids", (rows,), dev), rows, float(scale), o_ptr, o_pitch,
                            o_code, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_embedding")
    return out


def alloc_embedding_workspace(rows: int, vocab: int, width: int, m: int = 1, device=None) -> torch.Tensor:
    sizes = _size32("zeno_embedding_workspace_bytes", int(rows), int(vocab), int(width), int(m))
    return _workspace(int(load_library().zeno_embedding_workspace_bytes(*sizes)), "zeno_embedding_workspace_bytes", device)


def zeno_embedding_backward(dy, ids, vocab: int, *, scale=1.0, groups=None, dtable=None, accumulate=False, workspace=None):
    """Gradient of the table of zeno_embedding for each of the m workers: dtable [m x vocab * width] float32, for instance column slices
    of G.  accumulate=True adds to what dtable holds."""
    lib = load_library()
    dev = _current(dy, "dy")
    ptr, pitch, code, rows, width = _matrix(dy, "dy", dev)
    m, offsets = _groups(groups, dev)
    vocab = int(vocab)
    _size32("zeno_embedding_backward", vocab)
    if dtable is None:
        if accumulate:
            raise ValueError("accumulate needs a dtable to add to")
        dtable = dy.new_empty((m, max(vocab, 0) * width), dtype=torch.float32)
    g_ptr, ldg = _grad_rows(dtable, "dtable", m, vocab * width, dev)
    if workspace is None:
        workspace = alloc_embedding_workspace(rows, vocab, width, m, dy.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_embedding_backward(ptr, pitch, code, rows, width, _vec(ids, torch.int32, "ids", (rows,), dev), vocab, float(scale), m,
                                     offsets, 1 if accumulate else 0, g_ptr, ldg, ws, ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_embedding_backward")
    return dtable


def alloc_score_logprobs_workspace(m: int, d: int, device=None) -> torch.Tensor:
    _size32("zeno_score_logprobs_workspace_bytes", int(m))
    return _workspace(int(load_library().zeno_score_logprobs_workspace_bytes(int(m), int(d))), "zeno_score_logprobs_workspace_bytes", device)


def zeno_score_logprobs(G, logp_x, logp, rho, *, labels=None, scores=None, workspace=None):
    """scores[i] = mean_t (logp[i][t] - logp_x[t]) - rho ||G[i]||^2  (Definition 2 for the mean of -log p); tokens with
    label -1 do not count."""
    lib = load_library()
    dev = _current(G, "G")
    g_ptr, ldg = _rows(G)
    m, d = G.shape
    if not isinstance(logp_x, torch.Tensor) or logp_x.dim() != 1:
        raise ValueError("logp_x must be a vector")
    n, f32 = int(logp_x.numel()), torch.float32
    p_ptr, ldp, _, _, _ = _matrix(logp, "logp", dev, (m, n), f32)
    if scores is None:
        scores = G.new_empty((m,))
    if workspace is None:
        workspace = alloc_score_logprobs_workspace(m, d, G.device)
    ws, ws_bytes = _scratch(workspace, dev)
    st = lib.zeno_score_logprobs(g_ptr, ldg, m, d, _vec(logp_x, f32, "logp_x", (n,), dev), p_ptr, ldp, n,
                                 _vec(labels, torch.int32, "labels", (n,), dev), float(rho), _vec(scores, f32, "scores", (m,), dev), ws,
                                 ws_bytes, _stream())
    if st != 0:
        raise ZenoError(st, "zeno_score_logprobs")
    return scores


def profile_enable(on: bool = True):
    load_library().zeno_profile_enable(1 if on else 0)


def profile_collect(max_records: int = 4096, detail: bool = False):
    """[(kernel name, layer, ms, algorithmic bytes)] of the launches since the last collect; with
    detail=True a dict per launch that also names the launch shape of the layer kernels."""
    buf = (_ProfileRecord * max_records)()
    n = load_library().zeno_profile_collect(buf, max_records)
    if detail:
        return [dict(kernel=KERNEL_NAMES[r.kernel], layer=int(r.layer), ms=float(r.ms), bytes=float(r.algorithmic_bytes),
                     waves=int(r.waves), k_split=int(r.k_split), streaming=int(r.streaming),
                     row_blocks=int(r.row_blocks), merged=int(r.merged), second=int(r.second), k_slices=int(r.k_slices),
                     candidates=int(r.candidates),
                     tail_candidates=int(r.tail_candidates))
                for r in (buf[i] for i in range(n))]
    return [(KERNEL_NAMES[buf[i].kernel], int(buf[i].layer), float(buf[i].ms), float(buf[i].algorithmic_bytes))
            for i in range(n)]
