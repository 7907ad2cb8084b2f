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
    data, ld, kind, scales, ld_scales = m if len(m) == 5 else (*m, None, 0)
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

    # ---- layer operators.  Matrices are 2-D tensors with unit column stride (any row
    # stride); they and the current stream must be those of the handle.  Nothing is
    # recorded for autograd, also where a tensor requires its gradient: gradients come
    # from train_linear_backward.

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
        t = self.torch
        if not isinstance(x, t.Tensor) or x.dtype not in dtypes or x.dim() != 2:
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
        return x.data_ptr(), ld, TYPE_FP32 if x.dtype is t.float32 else TYPE_BF16, None, 0

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
        if not (isinstance(v, t.Tensor) and v.dtype is t.float32 and v.get_device() == device and v.dim() == 1
                and v.shape[0] == n and v.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous float32 tensor of {n} on the handle's device")
        return v.data_ptr()

    def _new(self, rows, cols, dtype, device):
        """A new matrix and itself as an argument."""
        y = self.torch.empty((rows, cols), dtype=dtype, device=device)
        return y, (y.data_ptr(), cols, TYPE_FP32 if dtype is self.torch.float32 else TYPE_BF16, None, 0)

    def _mx_new(self, rows, cols, format, device):
        empty, u8 = self.torch.empty, self.torch.uint8
        blocks = (cols + 31) // 32
        ld, ld_s = blocks * (16 if format == MXFP4 else 32), (blocks + 7) // 8 * 8
        q = MxTensor(empty((rows, ld), dtype=u8, device=device), empty((rows, ld_s), dtype=u8, device=device), cols, format)
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
