"""ctypes binding of include/donerf.h.

Functions carry the C names and only marshal arguments: every step of the
rendering runs in libdonerf.so.  Device buffers are passed as integer device
addresses (``tensor.data_ptr()``); host arrays as numpy arrays.  A missing
library raises ``DonerfLibraryMissing``: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libdonerf.so")

OK = 0
E_INVALID_ARG = -1
E_SIZE = -2
E_NONFINITE = -3
E_DEVICE = -4
E_NOMEM = -5
E_HIP = -6
E_UNSUPPORTED = -7

FP32 = 0
BF16 = 1
FP8 = 2
SELECT_TOPN = 0
SELECT_TOPN_SOFTMAX = 1
SELECT_CDF = 2
DEPTH_ENCODED = 0
DEPTH_POSITIONS = 1
MAX_SAMPLES = 16
# donerf_type: what a matrix of the layer operators holds
TYPE_FP32 = 0
TYPE_BF16 = 1
MXFP4 = 2
MXFP8 = 3
TYPE_INT32 = 4
TYPE_INT64 = 5
MAX_COLS = 65536
MAX_TOP = 128

# Every function include/donerf.h declares.
EXPORTS = ("donerf_weight_count", "donerf_create", "donerf_destroy", "donerf_set_stream",
           "donerf_render", "donerf_render_static_scratch", "donerf_render_debug", "donerf_targets",
           "donerf_debug_plan", "donerf_debug_topn", "donerf_debug_bins", "donerf_debug_mfma_peak",
           "donerf_mx_quantize", "donerf_mx_dequantize", "donerf_mx_linear", "donerf_mx_linear_workspace",
           "donerf_train_linear", "donerf_train_linear_backward", "donerf_train_linear_backward_workspace",
           "donerf_train_norm", "donerf_train_norm_backward", "donerf_train_norm_backward_workspace",
           "donerf_train_embedding", "donerf_train_embedding_backward", "donerf_train_embedding_backward_workspace",
           "donerf_train_distill", "donerf_get_stream", "donerf_status_str", "donerf_last_error")


class DonerfLibraryMissing(RuntimeError):
    pass


class DonerfError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


class donerf_cfg(ctypes.Structure):
    _fields_ = [("near_dist", ctypes.c_float), ("far_dist", ctypes.c_float),
                ("n_bins", ctypes.c_int32), ("n_max", ctypes.c_int32),
                ("fov_x_deg", ctypes.c_float), ("centre", ctypes.c_float * 3),
                ("radius", ctypes.c_float), ("precision", ctypes.c_int32),
                ("select", ctypes.c_int32), ("depth_input", ctypes.c_int32)]


class donerf_mat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("scales", ctypes.c_void_p),
                ("ld_scales", ctypes.c_int64), ("type", ctypes.c_int32)]


@dataclass
class Config:
    near: float = 0.1
    far: float = 10.0
    n_bins: int = 128
    n_max: int = 4
    fov_x_deg: float = 60.0
    centre: tuple = (0.0, 0.0, 0.0)
    radius: float = 1.5
    precision: int = BF16
    select: int = SELECT_TOPN
    depth_input: int = DEPTH_ENCODED

    def to_c(self) -> donerf_cfg:
        c = donerf_cfg()
        c.near_dist, c.far_dist = self.near, self.far
        c.n_bins, c.n_max = self.n_bins, self.n_max
        c.fov_x_deg = self.fov_x_deg
        c.centre[:] = list(self.centre)
        c.radius = self.radius
        c.precision, c.select = self.precision, self.select
        c.depth_input = self.depth_input
        return c


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DonerfLibraryMissing(
                f"{LIB_PATH} not built; run `python -m paper_2103_03231_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz, fp = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.POINTER(ctypes.c_float)
        L.donerf_weight_count.argtypes, L.donerf_weight_count.restype = [i32, i32], sz
        L.donerf_create.argtypes = [ctypes.POINTER(donerf_cfg), fp, sz, ctypes.POINTER(vp)]
        L.donerf_create.restype = ctypes.c_int
        L.donerf_destroy.argtypes, L.donerf_destroy.restype = [vp], None
        L.donerf_set_stream.argtypes, L.donerf_set_stream.restype = [vp, vp], ctypes.c_int
        L.donerf_render.argtypes = [vp, fp, i32, i32, i32, i32, vp, vp]
        L.donerf_render.restype = ctypes.c_int
        L.donerf_render_static_scratch.argtypes = [vp, fp, i32, i32, i32, i32, vp, vp]
        L.donerf_render_static_scratch.restype = ctypes.c_int
        L.donerf_render_debug.argtypes = [vp, fp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
        L.donerf_render_debug.restype = ctypes.c_int
        L.donerf_targets.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp]
        L.donerf_targets.restype = ctypes.c_int
        L.donerf_debug_plan.argtypes = [ctypes.POINTER(donerf_cfg), i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
        L.donerf_debug_plan.restype = ctypes.c_int
        L.donerf_debug_topn.argtypes = [vp, vp, i32, i32, vp]
        L.donerf_debug_topn.restype = ctypes.c_int
        L.donerf_debug_bins.argtypes = [vp, fp, fp, fp]
        L.donerf_debug_bins.restype = ctypes.c_int
        L.donerf_debug_mfma_peak.argtypes = [vp, i32, i32, vp, ctypes.POINTER(ctypes.c_double)]
        L.donerf_debug_mfma_peak.restype = ctypes.c_int
        mat, i64 = vp, ctypes.c_int64   # a donerf_mat's bytes, or byref of one
        L.donerf_mx_quantize.argtypes, L.donerf_mx_quantize.restype = [vp, mat, mat, i64, i32], ctypes.c_int
        L.donerf_mx_dequantize.argtypes, L.donerf_mx_dequantize.restype = [vp, mat, mat, i64, i32], ctypes.c_int
        L.donerf_mx_linear.argtypes = [vp, mat, mat, vp, i32, mat, i64, i32, i32, vp, sz]
        L.donerf_mx_linear.restype = ctypes.c_int
        L.donerf_mx_linear_workspace.argtypes, L.donerf_mx_linear_workspace.restype = [i32, i64, i32], sz
        L.donerf_train_linear.argtypes = [vp, mat, mat, vp, i32, mat, mat, i64, i32, i32]
        L.donerf_train_linear.restype = ctypes.c_int
        L.donerf_train_linear_backward.argtypes = [vp, mat, mat, i32, mat, mat, mat, vp, i32, i64, i32, i32, vp, sz]
        L.donerf_train_linear_backward.restype = ctypes.c_int
        L.donerf_train_linear_backward_workspace.argtypes = [vp, i64, i32, i32]
        L.donerf_train_linear_backward_workspace.restype = sz
        f32 = ctypes.c_float
        L.donerf_train_norm.argtypes = [vp, mat, vp, vp, f32, i32, mat, mat, vp, i64, i32]
        L.donerf_train_norm.restype = ctypes.c_int
        L.donerf_train_norm_backward.argtypes = [vp, mat, mat, i32, vp, vp, mat, vp, vp, i32, i64, i32, vp, sz]
        L.donerf_train_norm_backward.restype = ctypes.c_int
        L.donerf_train_norm_backward_workspace.argtypes = [vp, i64, i32]
        L.donerf_train_norm_backward_workspace.restype = sz
        L.donerf_train_embedding.argtypes, L.donerf_train_embedding.restype = [vp, mat, mat, f32, mat, i64, i64, i32], ctypes.c_int
        L.donerf_train_embedding_backward.argtypes = [vp, mat, mat, f32, mat, i32, i64, i64, i32, vp, sz]
        L.donerf_train_embedding_backward.restype = ctypes.c_int
        L.donerf_train_embedding_backward_workspace.argtypes = [vp, i64, i64, i32]
        L.donerf_train_embedding_backward_workspace.restype = sz
        L.donerf_train_distill.argtypes = [vp, mat, mat, mat, vp, f32, vp, mat, i64, i32, i32]
        L.donerf_train_distill.restype = ctypes.c_int
        L.donerf_get_stream.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(vp)]
        L.donerf_get_stream.restype = ctypes.c_int
        L.donerf_status_str.argtypes, L.donerf_status_str.restype = [ctypes.c_int], ctypes.c_char_p
        L.donerf_last_error.argtypes, L.donerf_last_error.restype = [], ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise DonerfError(status, donerf_last_error() or donerf_status_str(status))


def _fptr(a):
    return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


def donerf_weight_count(n_bins: int, depth_input: int = DEPTH_ENCODED) -> int:
    return int(lib().donerf_weight_count(n_bins, depth_input))


def donerf_status_str(status: int) -> str:
    return lib().donerf_status_str(status).decode()


def donerf_last_error() -> str:
    return lib().donerf_last_error().decode()


def donerf_create(cfg: Config, weights) -> int:
    """Returns the handle (an integer address); raises DonerfError."""
    w = None if weights is None else np.ascontiguousarray(weights, dtype=np.float32)
    h = ctypes.c_void_p()
    c = cfg.to_c()
    _check(lib().donerf_create(ctypes.byref(c), _fptr(w), 0 if w is None else w.size, ctypes.byref(h)))
    return h.value


def donerf_destroy(h) -> None:
    lib().donerf_destroy(h)


def donerf_set_stream(h, stream: int) -> None:
    _check(lib().donerf_set_stream(h, stream))


def _poses(poses):
    return None if poses is None else np.ascontiguousarray(poses, dtype=np.float32).reshape(-1)


def donerf_render(h, poses, P, H, W, N, out_rgb_ptr, out_depth_ptr=None) -> None:
    p = _poses(poses)
    _check(lib().donerf_render(h, _fptr(p), P, H, W, N, out_rgb_ptr, out_depth_ptr))


def donerf_render_static_scratch(h, poses, P, H, W, N, out_rgb_ptr, out_depth_ptr=None) -> None:
    p = _poses(poses)
    _check(lib().donerf_render_static_scratch(h, _fptr(p), P, H, W, N, out_rgb_ptr, out_depth_ptr))


def donerf_render_debug(h, poses, P, H, W, N, out_rgb_ptr, out_depth_ptr=None,
                        out_bins_ptr=None, out_scores_ptr=None, out_samples_ptr=None) -> None:
    p = _poses(poses)
    _check(lib().donerf_render_debug(h, _fptr(p), P, H, W, N, out_rgb_ptr, out_depth_ptr,
                                     out_bins_ptr, out_scores_ptr, out_samples_ptr))


def donerf_targets(h, depth_ptr, P, H, W, K, Z, out_ptr) -> None:
    _check(lib().donerf_targets(h, depth_ptr, P, H, W, K, Z, out_ptr))


def donerf_debug_plan(cfg: Config, P, H, W, N, launch=0, n_cu=256) -> dict:
    """How a render of these sizes is cut: launch `launch`'s part, {} past the last one."""
    out = (ctypes.c_int32 * 6)()
    c = cfg.to_c()
    _check(lib().donerf_debug_plan(ctypes.byref(c), n_cu, P, H, W, N, launch, out))
    keys = ("poses", "tile_rays", "n_full", "n_split", "split", "threads")
    return dict(zip(keys, out)) if out[0] else {}


def donerf_debug_topn(h, scores_ptr, rays, N, out_idx_ptr) -> None:
    _check(lib().donerf_debug_topn(h, scores_ptr, rays, N, out_idx_ptr))


def donerf_debug_mfma_peak(h, workgroups, iters, sink_ptr) -> float:
    """Enqueue the register-fed MFMA loop; returns the launch's FLOP."""
    flop = ctypes.c_double(0.0)
    _check(lib().donerf_debug_mfma_peak(h, workgroups, iters, sink_ptr, ctypes.byref(flop)))
    return flop.value


def donerf_debug_bins(h, n_bins):
    bounds = np.empty(n_bins + 1, np.float32)
    centres = np.empty(n_bins, np.float32)
    widths = np.empty(n_bins, np.float32)
    _check(lib().donerf_debug_bins(h, _fptr(bounds), _fptr(centres), _fptr(widths)))
    return bounds, centres, widths


# A donerf_mat's bytes: a third of the time that the structure takes.
_pack_mat = struct.Struct("@PqPqi4x").pack


def _mat(m):
    """A matrix argument: None, or (data, ld, type) of rows of values, or
    (data, ld, type, scales, ld_scales) of microscaled ones, addresses as integers."""
    if m is None:
        return None
    data, ld, kind, scales, ld_scales = m if len(m) == 5 else (*m, None, 0)
    return _pack_mat(data or 0, ld, scales or 0, ld_scales, kind)


def donerf_mx_quantize(h, x, q, rows, cols) -> None:
    _check(lib().donerf_mx_quantize(h, _mat(x), _mat(q), rows, cols))


def donerf_mx_dequantize(h, q, y, rows, cols) -> None:
    _check(lib().donerf_mx_dequantize(h, _mat(q), _mat(y), rows, cols))


def donerf_mx_linear_workspace(x_type, rows, n_in) -> int:
    return lib().donerf_mx_linear_workspace(x_type, rows, n_in)


def donerf_mx_linear(h, x, w, bias_ptr, relu, y, rows, n_in, n_out, workspace_ptr=None, workspace_bytes=0) -> None:
    _check(lib().donerf_mx_linear(h, _mat(x), _mat(w), bias_ptr, relu, _mat(y), rows, n_in, n_out,
                                  workspace_ptr, workspace_bytes))


def donerf_train_linear(h, x, w, bias_ptr, relu, y, kept, rows, n_in, n_out) -> None:
    _check(lib().donerf_train_linear(h, _mat(x), _mat(w), bias_ptr, relu, _mat(y), _mat(kept), rows, n_in, n_out))


def donerf_train_linear_backward_workspace(h, rows, n_in, n_out) -> int:
    return lib().donerf_train_linear_backward_workspace(h, rows, n_in, n_out)


def donerf_train_linear_backward(h, dz, x, relu, w, dx, dw, db_ptr, accumulate, rows, n_in, n_out,
                                 workspace_ptr=None, workspace_bytes=0) -> None:
    _check(lib().donerf_train_linear_backward(h, _mat(dz), _mat(x), relu, _mat(w), _mat(dx), _mat(dw), db_ptr,
                                              accumulate, rows, n_in, n_out, workspace_ptr, workspace_bytes))


def donerf_train_norm(h, x, weight_ptr, bias_ptr, eps, relu, y, kept, stats_ptr, rows, cols) -> None:
    _check(lib().donerf_train_norm(h, _mat(x), weight_ptr, bias_ptr, eps, relu, _mat(y), _mat(kept), stats_ptr, rows, cols))


def donerf_train_norm_backward_workspace(h, rows, cols) -> int:
    return lib().donerf_train_norm_backward_workspace(h, rows, cols)


def donerf_train_norm_backward(h, dz, x, relu, weight_ptr, stats_ptr, dx, dw_ptr, db_ptr, accumulate, rows, cols,
                               workspace_ptr=None, workspace_bytes=0) -> None:
    _check(lib().donerf_train_norm_backward(h, _mat(dz), _mat(x), relu, weight_ptr, stats_ptr, _mat(dx), dw_ptr, db_ptr,
                                            accumulate, rows, cols, workspace_ptr, workspace_bytes))


def donerf_train_embedding(h, table, ids, scale, y, rows, n, cols) -> None:
    _check(lib().donerf_train_embedding(h, _mat(table), _mat(ids), scale, _mat(y), rows, n, cols))


def donerf_train_embedding_backward_workspace(h, rows, n, cols) -> int:
    return lib().donerf_train_embedding_backward_workspace(h, rows, n, cols)


def donerf_train_embedding_backward(h, dy, ids, scale, dtable, accumulate, rows, n, cols, workspace_ptr=None,
                                    workspace_bytes=0) -> None:
    _check(lib().donerf_train_embedding_backward(h, _mat(dy), _mat(ids), scale, _mat(dtable), accumulate, rows, n, cols,
                                                 workspace_ptr, workspace_bytes))


def donerf_train_distill(h, x, classes, teacher, row_weight_ptr, temperature, loss_ptr, dx, rows, cols, k) -> None:
    _check(lib().donerf_train_distill(h, _mat(x), _mat(classes), _mat(teacher), row_weight_ptr, temperature, loss_ptr,
                                      _mat(dx), rows, cols, k))


def donerf_get_stream(h):
    """(device index, stream address) that the handle's work goes to."""
    device, stream = ctypes.c_int32(), ctypes.c_void_p()
    _check(lib().donerf_get_stream(h, ctypes.byref(device), ctypes.byref(stream)))
    return device.value, stream.value or 0


@dataclass
class MxTensor:
    """A microscaled matrix on the GPU: uint8 codes (rows, bytes) and scales
    (rows, blocks rounded up to 8), as include/donerf.h lays them out; `cols`
    values a row; `format` MXFP4 or MXFP8."""

    codes: object
    scales: object
    cols: int
    format: int

    @property
    def rows(self) -> int:
        return self.codes.shape[0]


class Renderer:
    """Convenience owner of a handle; outputs are torch tensors on cuda:0
    (torch provides device memory and the stream, nothing else)."""

    def __init__(self, cfg: Config, weights):
        import torch
        self.torch = torch
        # the tensors' types as the library names them
        self._kinds = {torch.float32: TYPE_FP32, torch.bfloat16: TYPE_BF16, torch.int32: TYPE_INT32, torch.int64: TYPE_INT64}
        self.cfg = cfg
        self.h = donerf_create(cfg, weights)
        donerf_set_stream(self.h, torch.cuda.current_stream().cuda_stream)
        # where donerf_get_stream answers
        self._device, self._stream = ctypes.c_int32(), ctypes.c_void_p()
        self._device_ref, self._stream_ref = ctypes.byref(self._device), ctypes.byref(self._stream)

    def close(self):
        if self.h:
            donerf_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def targets(self, depth, K, Z):
        """Depth-oracle targets of device depth maps (P, H, W) fp32 -> (P, H, W, B)."""
        t = self.torch
        if depth.dtype != t.float32 or not depth.is_cuda or not depth.is_contiguous() or depth.dim() != 3:
            raise ValueError("depth must be a contiguous (P, H, W) float32 CUDA tensor")
        P, H, W = depth.shape
        out = t.empty((P, H, W, self.cfg.n_bins), dtype=t.float32, device=depth.device)
        donerf_targets(self.h, depth.data_ptr(), P, H, W, K, Z, out.data_ptr())
        return out

    # ---- layer operators, and those around the layers.  Matrices are 2-D tensors with
    # unit column stride (any row stride); they and the current stream must be those of
    # the handle.  Nothing is recorded for autograd, also where a tensor requires its
    # gradient: gradients come from train_linear_backward, train_norm_backward,
    # train_embedding_backward and train_distill itself.

    # Checks are written for few attribute reads: on small calls they are most
    # of the time.

    def _bind(self):
        """The handle's device, once it is certain that outputs allocated now
        belong to the stream that the kernels will run on."""
        _check(lib().donerf_get_stream(self.h, self._device_ref, self._stream_ref))
        device, c = self._device.value, self.torch._C
        if c._cuda_getDevice() != device:
            raise ValueError(f"the handle is on cuda:{device}, which is not the current device")
        # the address of torch.cuda.current_stream(), without building the object
        if c._cuda_getCurrentRawStream(device) != (self._stream.value or 0):
            raise ValueError("torch's current stream is not the handle's (donerf_set_stream)")
        return device

    def _rows(self, name, x, dtypes, shape=None, device=None):
        if not isinstance(x, self.torch.Tensor) or x.dtype not in dtypes or x.dim() != 2:
            raise ValueError(f"{name} must be a 2-D tensor of {' or '.join(str(d) for d in dtypes)}")
        if x.get_device() != device:
            raise ValueError(f"{name} must be on the handle's device")
        rows, cols = x.shape
        if shape is not None and (rows, cols) != shape:
            raise ValueError(f"{name} is {(rows, cols)}, not {shape}")
        if not 1 <= cols <= MAX_COLS:
            raise ValueError(f"{name} has {cols} columns: 1 to {MAX_COLS} are taken")
        ld, step = x.stride()
        if rows <= 1:
            ld = cols
        if step != 1 and cols > 1 or ld < cols:
            raise ValueError(f"{name}: columns must be adjacent and rows must not overlap")
        return x.data_ptr(), ld, self._kinds[x.dtype], None, 0

    def _ids(self, ids, device):
        """A vector of whole numbers, of any stride, as a matrix argument of one column."""
        t = self.torch
        if not isinstance(ids, t.Tensor) or ids.dtype not in (t.int32, t.int64) or ids.dim() != 1:
            raise ValueError("ids must be a 1-D tensor of torch.int32 or torch.int64")
        if ids.get_device() != device:
            raise ValueError("ids must be on the handle's device")
        (n,), (ld,) = ids.shape, ids.stride()
        if n <= 1:
            ld = 1
        elif ld < 1:
            raise ValueError("ids must not share memory with each other")
        return ids.data_ptr(), ld, self._kinds[ids.dtype], None, 0

    def _out(self, out, default):
        """The type of a new result."""
        t = self.torch
        out = out or default
        if out is not t.bfloat16 and out is not t.float32:
            raise ValueError("out must be torch.bfloat16 or torch.float32")
        return out

    def _mx(self, name, q, formats, shape=None, device=None):
        t = self.torch
        if not isinstance(q, MxTensor) or q.format not in formats:
            raise ValueError(f"{name} must be a microscaled tensor of format {' or '.join(str(f) for f in formats)}")
        codes, scales, cols = q.codes, q.scales, q.cols
        if not (isinstance(codes, t.Tensor) and isinstance(scales, t.Tensor) and codes.dtype is t.uint8 and scales.dtype is t.uint8
                and codes.dim() == 2 and scales.dim() == 2 and codes.get_device() == device and scales.get_device() == device):
            raise ValueError(f"{name}: codes and scales must be 2-D uint8 tensors on the handle's device")
        (rows, wide), (rows_s, wide_s) = codes.shape, scales.shape
        if shape is not None and (rows, cols) != shape:
            raise ValueError(f"{name} is {(rows, cols)}, not {shape}")
        if not 1 <= cols <= MAX_COLS:
            raise ValueError(f"{name} has {cols} columns: 1 to {MAX_COLS} are taken")
        blocks = (cols + 31) // 32
        least, least_s = blocks * (16 if q.format == MXFP4 else 32), (blocks + 7) // 8 * 8
        (ld, step), (ld_s, step_s) = codes.stride(), scales.stride()
        if rows <= 1:
            ld, ld_s = least, least_s
        if rows_s != rows or wide < least or wide_s < least_s or ld < least or ld_s < least_s or step != 1 or step_s != 1:
            raise ValueError(f"{name}: codes must hold {rows} rows of {least} bytes and scales {rows} of {least_s}")
        return codes.data_ptr(), ld, q.format, scales.data_ptr(), ld_s

    def _vector(self, name, v, n, device):
        if v is None:
            return None
        t = self.torch
        if not (isinstance(v, t.Tensor) and v.dtype is t.float32 and v.get_device() == device and v.shape == (n,)
                and v.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous float32 tensor of {n} on the handle's device")
        return v.data_ptr()

    def _new(self, rows, cols, dtype, device):
        """A new matrix and itself as an argument."""
        y = self.torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)   # cheaper than empty
        return y, (y.data_ptr(), cols, TYPE_FP32 if dtype is self.torch.float32 else TYPE_BF16, None, 0)

    def _new_vector(self, n, device):
        v = self.torch.empty_strided((n,), (1,), dtype=self.torch.float32, device=device)
        return v, v.data_ptr()

    def _mx_new(self, rows, cols, format, device):
        empty, u8 = self.torch.empty_strided, self.torch.uint8
        blocks = (cols + 31) // 32
        ld, ld_s = blocks * (16 if format == MXFP4 else 32), (blocks + 7) // 8 * 8
        q = MxTensor(empty((rows, ld), (ld, 1), dtype=u8, device=device), empty((rows, ld_s), (ld_s, 1), dtype=u8, device=device), cols, format)
        return q, (q.codes.data_ptr(), ld, format, q.scales.data_ptr(), ld_s)

    def _workspace(self, n, device):
        return self.torch.empty(n, dtype=self.torch.uint8, device=device) if n else None

    def mx_empty(self, rows, cols, format):
        """An uninitialised microscaled matrix on the handle's device."""
        if format not in (MXFP4, MXFP8) or rows < 0 or not 1 <= cols <= MAX_COLS:
            raise ValueError("no such microscaled matrix")
        return self._mx_new(rows, cols, format, self._bind())[0]

    def mx_quantize(self, x, format):
        """(rows, cols) fp32 or bf16 -> MxTensor (donerf_mx_quantize)."""
        t, dev = self.torch, self._bind()
        mx = self._rows("x", x, (t.float32, t.bfloat16), None, dev)
        if format not in (MXFP4, MXFP8):
            raise ValueError("format must be MXFP4 or MXFP8")
        rows, cols = x.shape
        q, mq = self._mx_new(rows, cols, format, dev)
        donerf_mx_quantize(self.h, mx, mq, rows, cols)
        return q

    def mx_dequantize(self, q, dtype=None):
        """MxTensor -> (rows, cols) bf16 (default) or fp32 (donerf_mx_dequantize)."""
        t, dev = self.torch, self._bind()
        mq = self._mx("q", q, (MXFP4, MXFP8), None, dev)
        dtype = dtype or t.bfloat16
        if dtype not in (t.float32, t.bfloat16):
            raise ValueError("dtype must be torch.float32 or torch.bfloat16")
        y, my = self._new(q.rows, q.cols, dtype, dev)
        donerf_mx_dequantize(self.h, mq, my, q.rows, q.cols)
        return y

    def mx_linear(self, x, w, bias=None, relu=False, out=None):
        """act(x w^T + bias) in MXFP4 (donerf_mx_linear).  x: (rows, in) fp32 or
        bf16, or MxTensor; w: MxTensor (out, in); out: torch.bfloat16 (default),
        torch.float32 or MXFP4, the result's type, or a tensor that takes it."""
        t, dev = self.torch, self._bind()
        if isinstance(x, MxTensor):
            mx = self._mx("x", x, (MXFP4,), None, dev)
            rows, n_in = x.rows, x.cols
        else:
            mx = self._rows("x", x, (t.float32, t.bfloat16), None, dev)
            rows, n_in = x.shape
        mw = self._mx("w", w, (MXFP4,), None, dev)
        if w.cols != n_in:
            raise ValueError(f"x has {n_in} columns and w {w.cols}")
        n_out = w.rows
        if not 1 <= n_out <= MAX_COLS:
            raise ValueError(f"w has {n_out} rows: 1 to {MAX_COLS} are taken")
        pb = self._vector("bias", bias, n_out, dev)
        if isinstance(out, MxTensor):
            y, my = out, self._mx("out", out, (MXFP4,), (rows, n_out), dev)
        elif isinstance(out, t.Tensor):
            y, my = out, self._rows("out", out, (t.float32, t.bfloat16), (rows, n_out), dev)
        elif out is None or out in (t.float32, t.bfloat16):
            y, my = self._new(rows, n_out, out or t.bfloat16, dev)
        elif out == MXFP4:
            y, my = self._mx_new(rows, n_out, MXFP4, dev)
        else:
            raise ValueError("out must be torch.bfloat16, torch.float32, MXFP4 or a tensor")
        need = donerf_mx_linear_workspace(mx[2], rows, n_in)
        ws = self._workspace(need, dev)
        donerf_mx_linear(self.h, mx, mw, pb, 1 if relu else 0, my, rows, n_in, n_out, ws.data_ptr() if need else None, need)
        return y

    def train_linear(self, x, w, bias=None, relu=False, keep=True):
        """A layer's forward pass (donerf_train_linear): x (rows, in) and w (out,
        in) bf16 -> (y (rows, out) bf16, the same in MXFP8 or None without keep).
        y has no autograd history: its gradient is train_linear_backward's dz."""
        t, dev = self.torch, self._bind()
        bf16 = (t.bfloat16,)
        mx, mw = self._rows("x", x, bf16, None, dev), self._rows("w", w, bf16, None, dev)
        (rows, n_in), (n_out, w_in) = x.shape, w.shape
        if w_in != n_in or not 1 <= n_out <= MAX_COLS:
            raise ValueError(f"x is {tuple(x.shape)} and w {tuple(w.shape)}")
        pb = self._vector("bias", bias, n_out, dev)
        y, my = self._new(rows, n_out, t.bfloat16, dev)
        kept, mk = self._mx_new(rows, n_out, MXFP8, dev) if keep else (None, None)
        donerf_train_linear(self.h, mx, mw, pb, 1 if relu else 0, my, mk, rows, n_in, n_out)
        return y, kept

    def train_linear_backward(self, dz, x, w, relu=False, need_dx=True, dw=None, db=None):
        """The layer's backward pass (donerf_train_linear_backward): dz (rows,
        out) bf16; x (rows, in) as MxTensor (MXFP8) or bf16, `relu` where it came
        out of a ReLU; w (out, in) bf16 -> (dx bf16 or None, dw fp32, db fp32).
        Where dw and db are given, they are added to."""
        t, dev = self.torch, self._bind()
        bf16 = (t.bfloat16,)
        mz, mw = self._rows("dz", dz, bf16, None, dev), self._rows("w", w, bf16, None, dev)
        (rows, n_out), (w_out, n_in) = dz.shape, w.shape
        if w_out != n_out:
            raise ValueError(f"dz is {tuple(dz.shape)} and w {tuple(w.shape)}")
        mx = (self._mx("x", x, (MXFP8,), (rows, n_in), dev) if isinstance(x, MxTensor)
              else self._rows("x", x, bf16, (rows, n_in), dev))
        add = dw is not None
        if add != (db is not None):
            raise ValueError("dw and db are given together or not at all")
        if add:
            mdw = self._rows("dw", dw, (t.float32,), (n_out, n_in), dev)
        else:
            dw, mdw = self._new(n_out, n_in, t.float32, dev)
            db = t.empty(n_out, dtype=t.float32, device=dev)
        pdb = self._vector("db", db, n_out, dev)
        dx, mdx = self._new(rows, n_in, t.bfloat16, dev) if need_dx else (None, None)
        need = donerf_train_linear_backward_workspace(self.h, rows, n_in, n_out)
        ws = self._workspace(need, dev)
        donerf_train_linear_backward(self.h, mz, mx, 1 if relu else 0, mw, mdx, mdw, pdb, 1 if add else 0,
                                     rows, n_in, n_out, ws.data_ptr() if need else None, need)
        return dx, dw, db

    def train_norm(self, x, weight=None, bias=None, eps=1e-5, relu=False, keep=True, out=None):
        """Layer norm's forward pass (donerf_train_norm): x (rows, cols) fp32 or
        bf16; weight and bias (cols) fp32 -> (y in torch.bfloat16 or `out`, the
        same in MXFP8 or None without keep, stats (rows, 2) for the backward pass)."""
        t, dev = self.torch, self._bind()
        mx = self._rows("x", x, (t.float32, t.bfloat16), None, dev)
        rows, cols = x.shape
        pw, pb = self._vector("weight", weight, cols, dev), self._vector("bias", bias, cols, dev)
        y, my = self._new(rows, cols, self._out(out, t.bfloat16), dev)
        kept, mk = self._mx_new(rows, cols, MXFP8, dev) if keep else (None, None)
        stats = t.empty_strided((rows, 2), (2, 1), dtype=t.float32, device=dev)
        donerf_train_norm(self.h, mx, pw, pb, eps, 1 if relu else 0, my, mk, stats.data_ptr(), rows, cols)
        return y, kept, stats

    def train_norm_backward(self, dz, x, stats, weight=None, relu=False, need_dx=True, dw=None, db=None, out=None):
        """Its backward pass (donerf_train_norm_backward): dz (rows, cols) fp32 or
        bf16; x as the forward pass had it, or in MXFP8, `relu` where it came out of a
        ReLU; stats from the forward pass -> (dx in torch.bfloat16 or `out`, or None,
        dw (cols) fp32, db (cols) fp32).  Where dw and db are given, they are added to."""
        t, dev = self.torch, self._bind()
        mz = self._rows("dz", dz, (t.float32, t.bfloat16), None, dev)
        rows, cols = dz.shape
        mx = (self._mx("x", x, (MXFP8,), (rows, cols), dev) if isinstance(x, MxTensor)
              else self._rows("x", x, (t.float32, t.bfloat16), (rows, cols), dev))
        if not (isinstance(stats, t.Tensor) and stats.dtype is t.float32 and stats.get_device() == dev
                and stats.shape == (rows, 2) and stats.is_contiguous()):
            raise ValueError(f"stats must be a contiguous float32 tensor of {(rows, 2)} on the handle's device")
        pw = self._vector("weight", weight, cols, dev)
        add = dw is not None
        if add != (db is not None):
            raise ValueError("dw and db are given together or not at all")
        if add:
            pdw, pdb = self._vector("dw", dw, cols, dev), self._vector("db", db, cols, dev)
        else:
            (dw, pdw), (db, pdb) = self._new_vector(cols, dev), self._new_vector(cols, dev)
        dx, mdx = self._new(rows, cols, self._out(out, t.bfloat16), dev) if need_dx else (None, None)
        need = donerf_train_norm_backward_workspace(self.h, rows, cols)
        ws = self._workspace(need, dev)
        donerf_train_norm_backward(self.h, mz, mx, 1 if relu else 0, pw, stats.data_ptr(), mdx, pdw, pdb, 1 if add else 0,
                                   rows, cols, ws.data_ptr() if need else None, need)
        return dx, dw, db

    def train_embedding(self, table, ids, scale=1.0, out=None):
        """scale table[ids], zeros for ids outside the table (donerf_train_embedding):
        table (n, cols) fp32 or bf16, ids (rows) int32 or int64 -> (rows, cols) in
        torch.bfloat16 or `out`."""
        t, dev = self.torch, self._bind()
        mt = self._rows("table", table, (t.float32, t.bfloat16), None, dev)
        mi = self._ids(ids, dev)
        (n, cols), rows = table.shape, ids.shape[0]
        y, my = self._new(rows, cols, self._out(out, t.bfloat16), dev)
        donerf_train_embedding(self.h, mt, mi, scale, my, rows, n, cols)
        return y

    def train_embedding_backward(self, dy, ids, n, scale=1.0, dtable=None):
        """The gradient of a table of n rows (donerf_train_embedding_backward): dy
        (rows, cols) fp32 or bf16, ids (rows) int32 or int64 -> (n, cols) fp32.  Where
        dtable is given, it is added to."""
        t, dev = self.torch, self._bind()
        md = self._rows("dy", dy, (t.float32, t.bfloat16), None, dev)
        mi = self._ids(ids, dev)
        rows, cols = dy.shape
        if ids.shape[0] != rows:
            raise ValueError(f"dy has {rows} rows and ids {ids.shape[0]}")
        add = dtable is not None
        if add:
            mt = self._rows("dtable", dtable, (t.float32,), (n, cols), dev)
        elif 1 <= n < 1 << 31:
            dtable, mt = self._new(n, cols, t.float32, dev)
        else:
            raise ValueError("n must lie in [1, 2^31)")
        need = donerf_train_embedding_backward_workspace(self.h, rows, n, cols)
        ws = self._workspace(need, dev)
        donerf_train_embedding_backward(self.h, md, mi, scale, mt, 1 if add else 0, rows, n, cols, ws.data_ptr() if need else None,
                                        need)
        return dtable

    def train_distill(self, x, classes, teacher, temperature=1.0, row_weight=None, need_dx=True, out=None):
        """Distillation from a teacher's top logits (donerf_train_distill): x (rows,
        classes) fp32 or bf16, the student's logits; classes (rows, k) int32 or int64
        and teacher (rows, k) fp32 or bf16, the teacher's entries; row_weight (rows)
        fp32 -> (each row's loss (rows) fp32, the gradient of their sum in
        torch.bfloat16 or `out`, or None)."""
        t, dev = self.torch, self._bind()
        mx = self._rows("x", x, (t.float32, t.bfloat16), None, dev)
        mc = self._rows("classes", classes, (t.int32, t.int64), None, dev)
        (rows, cols), k = x.shape, classes.shape[1]
        mt = self._rows("teacher", teacher, (t.float32, t.bfloat16), (rows, k), dev)
        if classes.shape[0] != rows:
            raise ValueError(f"x has {rows} rows and classes {classes.shape[0]}")
        pw = self._vector("row_weight", row_weight, rows, dev)
        loss, pl = self._new_vector(rows, dev)
        dx, mdx = self._new(rows, cols, self._out(out, t.bfloat16), dev) if need_dx else (None, None)
        donerf_train_distill(self.h, mx, mc, mt, pw, temperature, pl, mdx, rows, cols, k)
        return loss, dx

    def mfma_peak(self, workgroups, iters):
        """Enqueue the register-fed MFMA loop in the handle's precision;
        returns (sink, FLOP of the launch)."""
        import torch
        sink = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
        return sink, donerf_debug_mfma_peak(self.h, workgroups, iters, sink.data_ptr())

    def alloc(self, P, H, W, N, depth=False, debug=False):
        t = self.torch
        dev = "cuda"
        out = {"rgb": t.empty((P, H, W, 3), dtype=t.float32, device=dev)}
        if depth:
            out["depth"] = t.empty((P, H, W), dtype=t.float32, device=dev)
        if debug:
            out["bins"] = t.empty((P, H, W, N), dtype=t.int32, device=dev)
            out["scores"] = t.empty((P, H, W, self.cfg.n_bins), dtype=t.float32, device=dev)
            out["samples"] = t.empty((P, H, W, N, 2), dtype=t.float32, device=dev)
        return out

    def _check_out(self, P, H, W, N, out):
        """Reject output tensors the library would write out of bounds:
        each present one must be a contiguous CUDA tensor of the right dtype
        holding P x H x W x {3, 1, N, B, 2 N} values."""
        t = self.torch
        per_ray = {"rgb": 3, "depth": 1, "bins": N, "scores": self.cfg.n_bins, "samples": 2 * N}
        if "rgb" not in out:
            raise ValueError("out needs an 'rgb' tensor")
        for k, v in out.items():
            if k not in per_ray:
                raise ValueError(f"unknown output {k!r}")
            dtype = t.int32 if k == "bins" else t.float32
            if not (isinstance(v, t.Tensor) and v.is_cuda and v.is_contiguous() and v.dtype == dtype):
                raise ValueError(f"out[{k!r}] must be a contiguous CUDA {dtype} tensor")
            if v.numel() != P * H * W * per_ray[k]:
                raise ValueError(f"out[{k!r}] holds {v.numel()} values, the render writes {P * H * W * per_ray[k]}")

    def render_into(self, poses, H, W, N, out, debug=False):
        P = int(np.asarray(poses).reshape(-1, 12).shape[0])
        self._check_out(P, H, W, N, out)
        ptr = lambda k: out[k].data_ptr() if k in out else None
        if debug:
            donerf_render_debug(self.h, poses, P, H, W, N, ptr("rgb"), ptr("depth"),
                                ptr("bins"), ptr("scores"), ptr("samples"))
        else:
            donerf_render(self.h, poses, P, H, W, N, ptr("rgb"), ptr("depth"))
        return out

    def render(self, poses, H, W, N, depth=False, debug=False):
        P = int(np.asarray(poses).reshape(-1, 12).shape[0])
        out = self.alloc(P, H, W, N, depth=depth, debug=debug)
        return self.render_into(poses, H, W, N, out, debug=debug)
