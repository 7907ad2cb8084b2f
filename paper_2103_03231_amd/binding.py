"""ctypes binding of include/donerf.h.

Functions carry the C names and only marshal arguments: every step of the
rendering runs in libdonerf.so.  Device buffers are passed as integer device
addresses (``tensor.data_ptr()``); host arrays as numpy arrays.  A missing
library raises ``DonerfLibraryMissing``: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
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
MAX_COLS = 65536

# Every function include/donerf.h declares.
EXPORTS = ("donerf_weight_count", "donerf_create", "donerf_destroy", "donerf_set_stream",
           "donerf_render", "donerf_render_static_scratch", "donerf_render_debug", "donerf_targets",
           "donerf_debug_plan", "donerf_debug_topn", "donerf_debug_bins", "donerf_debug_mfma_peak",
           "donerf_mx_quantize", "donerf_mx_dequantize", "donerf_mx_linear", "donerf_mx_linear_workspace",
           "donerf_train_linear", "donerf_train_linear_backward", "donerf_train_linear_backward_workspace",
           "donerf_get_stream", "donerf_status_str", "donerf_last_error")


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
        mat, i64 = ctypes.POINTER(donerf_mat), ctypes.c_int64
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


def _mat(m):
    """A matrix argument: None, or (data, ld, type) of fp32 and bf16 rows, or
    (data, ld, type, scales, ld_scales) of microscaled ones, addresses as integers."""
    if m is None:
        return None
    data, ld, kind = m[:3]
    scales, ld_scales = m[3:] or (None, 0)
    return ctypes.byref(donerf_mat(data, ld, scales, ld_scales, kind))


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
        self.cfg = cfg
        self.h = donerf_create(cfg, weights)
        donerf_set_stream(self.h, torch.cuda.current_stream().cuda_stream)

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

    # ---- layer operators.  Matrices are 2-D tensors with unit column stride (any row
    # stride); they and the current stream must be those of the handle.

    def _bind(self):
        """The handle's device, once it is certain that outputs allocated now
        belong to the stream that the kernels will run on."""
        device, stream = donerf_get_stream(self.h)
        if self.torch.cuda.current_device() != device:
            raise ValueError(f"the handle is on cuda:{device}, which is not the current device")
        if self.torch.cuda.current_stream().cuda_stream != stream:
            raise ValueError("torch's current stream is not the handle's (donerf_set_stream)")
        return device

    def _rows(self, name, x, dtypes, shape=None, device=None):
        t = self.torch
        if not isinstance(x, t.Tensor) or x.dim() != 2 or x.dtype not in dtypes:
            raise ValueError(f"{name} must be a 2-D tensor of {' or '.join(str(d) for d in dtypes)}")
        if not x.is_cuda or x.device.index != device:
            raise ValueError(f"{name} must be on the handle's device")
        if shape is not None and tuple(x.shape) != tuple(shape):
            raise ValueError(f"{name} is {tuple(x.shape)}, not {tuple(shape)}")
        rows, cols = x.shape
        if cols < 1 or cols > MAX_COLS:
            raise ValueError(f"{name} has {cols} columns: 1 to {MAX_COLS} are taken")
        if cols > 1 and x.stride(1) != 1 or rows > 1 and x.stride(0) < cols:
            raise ValueError(f"{name}: columns must be adjacent and rows must not overlap")
        return x.data_ptr(), (x.stride(0) if rows > 1 else cols), TYPE_FP32 if x.dtype == t.float32 else TYPE_BF16

    def _mx(self, name, q, formats, shape=None, device=None):
        t = self.torch
        if not isinstance(q, MxTensor) or q.format not in formats:
            raise ValueError(f"{name} must be a microscaled tensor of format {' or '.join(str(f) for f in formats)}")
        if shape is not None and (q.rows, q.cols) != tuple(shape):
            raise ValueError(f"{name} is {(q.rows, q.cols)}, not {tuple(shape)}")
        blocks = -(-q.cols // 32)
        width = blocks * (16 if q.format == MXFP4 else 32)
        for part, x, least, unit in (("codes", q.codes, width, 16), ("scales", q.scales, -(-blocks // 8) * 8, 8)):
            if not (isinstance(x, t.Tensor) and x.dtype == t.uint8 and x.dim() == 2 and x.is_cuda and x.device.index == device):
                raise ValueError(f"{name}: {part} must be a 2-D uint8 tensor on the handle's device")
            if x.shape[0] != q.rows or x.shape[1] < least or x.stride(1) != 1 or q.rows > 1 and x.stride(0) < least:
                raise ValueError(f"{name}: {part} must hold {q.rows} rows of {least} bytes")
        pitch = lambda x, least: x.stride(0) if q.rows > 1 else least
        return (q.codes.data_ptr(), pitch(q.codes, width), q.format, q.scales.data_ptr(),
                pitch(q.scales, -(-blocks // 8) * 8))

    def _vector(self, name, v, n, device):
        if v is None:
            return None
        t = self.torch
        if not (isinstance(v, t.Tensor) and v.dtype == t.float32 and v.is_cuda and v.device.index == device
                and v.is_contiguous() and tuple(v.shape) == (n,)):
            raise ValueError(f"{name} must be a contiguous float32 tensor of {n} on the handle's device")
        return v.data_ptr()

    def mx_empty(self, rows, cols, format):
        """An uninitialised microscaled matrix on the current device."""
        t = self.torch
        if format not in (MXFP4, MXFP8) or rows < 0 or not 1 <= cols <= MAX_COLS:
            raise ValueError("no such microscaled matrix")
        blocks = -(-cols // 32)
        return MxTensor(t.empty((rows, blocks * (16 if format == MXFP4 else 32)), dtype=t.uint8, device="cuda"),
                        t.empty((rows, -(-blocks // 8) * 8), dtype=t.uint8, device="cuda"), cols, format)

    def mx_quantize(self, x, format):
        """(rows, cols) fp32 or bf16 -> MxTensor (donerf_mx_quantize)."""
        t, dev = self.torch, self._bind()
        mx = self._rows("x", x, (t.float32, t.bfloat16), device=dev)
        q = self.mx_empty(x.shape[0], x.shape[1], format)
        donerf_mx_quantize(self.h, mx, self._mx("q", q, (MXFP4, MXFP8), device=dev), *x.shape)
        return q

    def mx_dequantize(self, q, dtype=None):
        """MxTensor -> (rows, cols) bf16 (default) or fp32 (donerf_mx_dequantize)."""
        t, dev = self.torch, self._bind()
        mq = self._mx("q", q, (MXFP4, MXFP8), device=dev)
        y = t.empty((q.rows, q.cols), dtype=dtype or t.bfloat16, device="cuda")
        donerf_mx_dequantize(self.h, mq, self._rows("y", y, (t.float32, t.bfloat16), device=dev), q.rows, q.cols)
        return y

    def mx_linear(self, x, w, bias=None, relu=False, out=None):
        """act(x w^T + bias) in MXFP4 (donerf_mx_linear).  x: (rows, in) fp32 or
        bf16, or MxTensor; w: MxTensor (out, in); out: torch.bfloat16 (default),
        torch.float32 or MXFP4, the result's type, or a tensor that takes it."""
        t, dev = self.torch, self._bind()
        if isinstance(x, MxTensor):
            rows, n_in = x.rows, x.cols
            mx = self._mx("x", x, (MXFP4,), device=dev)
        else:
            mx = self._rows("x", x, (t.float32, t.bfloat16), device=dev)
            rows, n_in = x.shape
        mw = self._mx("w", w, (MXFP4,), device=dev)
        if w.cols != n_in:
            raise ValueError(f"x has {n_in} columns and w {w.cols}")
        n_out = w.rows
        pb = self._vector("bias", bias, n_out, dev)
        if isinstance(out, int):
            y = self.mx_empty(rows, n_out, out)
        else:
            y = out if isinstance(out, (t.Tensor, MxTensor)) else t.empty((rows, n_out), dtype=out or t.bfloat16, device="cuda")
        my = (self._mx("out", y, (MXFP4,), (rows, n_out), dev) if isinstance(y, MxTensor)
              else self._rows("out", y, (t.float32, t.bfloat16), (rows, n_out), dev))
        need = donerf_mx_linear_workspace(mx[2], rows, n_in)
        ws = t.empty(need, dtype=t.uint8, device="cuda") if need else None
        donerf_mx_linear(self.h, mx, mw, pb, int(bool(relu)), my, rows, n_in, n_out, ws.data_ptr() if need else None, need)
        return y

    def train_linear(self, x, w, bias=None, relu=False, keep=True):
        """A layer's forward pass (donerf_train_linear): x (rows, in) and w (out,
        in) bf16 -> (y (rows, out) bf16, the same in MXFP8 or None without keep)."""
        t, dev = self.torch, self._bind()
        mx, mw = self._rows("x", x, (t.bfloat16,), device=dev), self._rows("w", w, (t.bfloat16,), device=dev)
        (rows, n_in), n_out = x.shape, w.shape[0]
        if w.shape[1] != n_in or n_out < 1:
            raise ValueError(f"x is {tuple(x.shape)} and w {tuple(w.shape)}")
        pb = self._vector("bias", bias, n_out, dev)
        y = t.empty((rows, n_out), dtype=t.bfloat16, device="cuda")
        kept = self.mx_empty(rows, n_out, MXFP8) if keep else None
        donerf_train_linear(self.h, mx, mw, pb, int(bool(relu)), self._rows("y", y, (t.bfloat16,), device=dev),
                            self._mx("kept", kept, (MXFP8,), device=dev) if keep else None, rows, n_in, n_out)
        return y, kept

    def train_linear_backward(self, dz, x, w, relu=False, need_dx=True, dw=None, db=None):
        """The layer's backward pass (donerf_train_linear_backward): dz (rows,
        out) bf16; x (rows, in) as MxTensor (MXFP8) or bf16, `relu` where it came
        out of a ReLU; w (out, in) bf16 -> (dx bf16 or None, dw fp32, db fp32).
        Where dw and db are given, they are added to."""
        t, dev = self.torch, self._bind()
        mz, mw = self._rows("dz", dz, (t.bfloat16,), device=dev), self._rows("w", w, (t.bfloat16,), device=dev)
        (rows, n_out), n_in = dz.shape, w.shape[1]
        if w.shape[0] != n_out:
            raise ValueError(f"dz is {tuple(dz.shape)} and w {tuple(w.shape)}")
        mx = (self._mx("x", x, (MXFP8,), (rows, n_in), dev) if isinstance(x, MxTensor)
              else self._rows("x", x, (t.bfloat16,), (rows, n_in), dev))
        if (dw is None) != (db is None):
            raise ValueError("dw and db are given together or not at all")
        add = dw is not None
        if not add:
            dw = t.empty((n_out, n_in), dtype=t.float32, device="cuda")
            db = t.empty(n_out, dtype=t.float32, device="cuda")
        mdw, pdb = self._rows("dw", dw, (t.float32,), (n_out, n_in), dev), self._vector("db", db, n_out, dev)
        dx = t.empty((rows, n_in), dtype=t.bfloat16, device="cuda") if need_dx else None
        need = donerf_train_linear_backward_workspace(self.h, rows, n_in, n_out)
        ws = t.empty(need, dtype=t.uint8, device="cuda")
        donerf_train_linear_backward(self.h, mz, mx, int(bool(relu)), mw,
                                     self._rows("dx", dx, (t.bfloat16,), device=dev) if need_dx else None, mdw, pdb,
                                     int(add), rows, n_in, n_out, ws.data_ptr(), need)
        return dx, dw, db

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
