"""Thin ctypes binding over libmpcnn.so (the C ABI declared in include/mpcnn.h).

Argument marshalling only: every step of the whole-image forward / backward
runs in the library's HIP kernels.  PyTorch supplies device memory (tensors'
`data_ptr()`) and the stream.  There is no fallback: if the library has not
been built, or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from functools import lru_cache
from typing import Optional, Sequence, Tuple

import numpy as np


class _Torch:
    """Stands for torch until something of it is wanted, and puts it in its own place then: names and constants can be read without it."""

    def __getattr__(self, name):
        import torch as module
        globals()["torch"] = module
        return getattr(module, name)


torch = _Torch()

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmpcnn.so")

KIND_C, KIND_MP, KIND_FC = 0, 1, 2
STATIC_WORKSPACE_BYTES = 64 * 1024 * 1024   # MPCNN_STATIC_WORKSPACE_BYTES
F32, BF16 = 0, 1
I8, E4M3 = 2, 3   # mpcnn_packing: kinds of rows in 8 bits

STATUS = {0: "MPCNN_OK", 1: "MPCNN_EINVAL", 2: "MPCNN_ESHAPE", 3: "MPCNN_EWORKSPACE",
          4: "MPCNN_EUNSUPPORTED", 5: "MPCNN_EHIP", 6: "MPCNN_ENOMEM"}

# every symbol include/mpcnn.h declares
SYMBOLS = [
    "mpcnn_net_create", "mpcnn_net_destroy", "mpcnn_net_patch", "mpcnn_net_classes",
    "mpcnn_param_count", "mpcnn_layer_shape", "mpcnn_set_params", "mpcnn_get_params",
    "mpcnn_get_grads", "mpcnn_workspace_bytes", "mpcnn_seg_forward", "mpcnn_seg_backward",
    "mpcnn_sgd_step", "mpcnn_get_activation", "mpcnn_get_argmax", "mpcnn_last_error",
    "mpcnn_profile_enable", "mpcnn_profile_read", "mpcnn_workspace_bytes_same", "mpcnn_seg_forward_same",
    "mpcnn_set_loss", "mpcnn_class_balance_weights", "mpcnn_seg_loss", "mpcnn_armijo_step",
    "mpcnn_lbfgs_step", "mpcnn_lbfgs_reset", "mpcnn_set_activation", "mpcnn_set_conv_tiling",
    "mpcnn_workspace_bytes_banded", "mpcnn_seg_backward_banded", "mpcnn_seg_forward_static",
    "mpcnn_plan_describe", "mpcnn_sgd_step_clipped", "mpcnn_grad_list_create", "mpcnn_grad_list_destroy",
    "mpcnn_grad_norm", "mpcnn_grad_clip", "mpcnn_sgd_step_list",
    "mpcnn_workspace_bytes_class", "mpcnn_workspace_bytes_class_call", "mpcnn_class_loss", "mpcnn_class_backward",
    "mpcnn_rows_pack", "mpcnn_rows_unpack", "mpcnn_rows_norm", "mpcnn_workspace_bytes_norm", "mpcnn_rows_norm_backward",
    "mpcnn_workspace_bytes_weight_grad", "mpcnn_rows_weight_grad",
    "mpcnn_workspace_bytes_beam", "mpcnn_beam_select", "mpcnn_workspace_bytes_class_beam", "mpcnn_class_beam",
    "mpcnn_beam_states_create", "mpcnn_beam_states_destroy", "mpcnn_beam_reorder",
]


class MpcnnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS.get(status, status), message))
        self.status = status


class _LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int), ("maps", C.c_int), ("k", C.c_int), ("k2", C.c_int)]


class KernelStat(C.Structure):
    """mpcnn_kernel_stat: one launch site (kernel x layer) of the profiled calls."""
    _fields_ = [("name", C.c_char * 48), ("layer", C.c_int), ("step", C.c_int),
                ("launches", C.c_int), ("ms_total", C.c_double), ("flops", C.c_double),
                ("bytes", C.c_double)]


class _Tensor(C.Structure):
    """mpcnn_tensor: a gradient and the parameters it belongs to."""
    _fields_ = [("grad", C.c_void_p), ("param", C.c_void_p), ("n", C.c_int64), ("grad_dtype", C.c_int),
                ("param_dtype", C.c_int)]


class _Packed(C.Structure):
    """mpcnn_packed: a matrix in 8 bits."""
    _fields_ = [("values", C.c_void_p), ("scales", C.c_void_p), ("kind", C.c_int)]


class _BeamState(C.Structure):
    """mpcnn_beam_state: a tensor of beams' states."""
    _fields_ = [("data", C.c_void_p), ("row_pitch", C.c_int64), ("segment_pitch", C.c_int64), ("unit_bytes", C.c_int64), ("units", C.c_int64),
                ("segments", C.c_int64)]


_lib = None


def lib():
    """Load libmpcnn.so (built by `python -m paper_1302_1690_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libmpcnn.so is not built: run `python -m paper_1302_1690_amd.build` "
                              "(there is no fallback path)")
        # torch ships its own copy of the HIP runtime (same soname as the system one):
        # it must be loaded first so that the library binds to it and both share one
        # runtime, hence one set of device allocations and streams.
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        vp, sz, i = C.c_void_p, C.c_size_t, C.c_int
        L.mpcnn_net_create.argtypes = [C.POINTER(_LayerDesc), i, i, i, i, C.POINTER(vp)]
        L.mpcnn_net_destroy.argtypes = [vp]
        L.mpcnn_net_destroy.restype = None
        L.mpcnn_net_patch.argtypes = [vp]
        L.mpcnn_net_classes.argtypes = [vp]
        L.mpcnn_param_count.argtypes = [vp]
        L.mpcnn_param_count.restype = sz
        L.mpcnn_layer_shape.argtypes = [vp, i, i, i] + [C.POINTER(i)] * 4
        L.mpcnn_plan_describe.argtypes = [vp, i, i, i, i, C.c_char_p, sz]
        L.mpcnn_set_params.argtypes = [vp, vp, sz]
        L.mpcnn_get_params.argtypes = [vp, vp, sz]
        L.mpcnn_get_grads.argtypes = [vp, vp, sz]
        L.mpcnn_workspace_bytes.argtypes = [vp, i, i, i, i]
        L.mpcnn_workspace_bytes.restype = sz
        L.mpcnn_seg_forward.argtypes = [vp, vp, i, i, i, vp, vp, sz, vp]
        L.mpcnn_seg_forward_static.argtypes = [vp, vp, i, i, i, vp, vp]
        L.mpcnn_workspace_bytes_same.argtypes = [vp, i, i, i]
        L.mpcnn_workspace_bytes_same.restype = sz
        L.mpcnn_seg_forward_same.argtypes = [vp, vp, i, i, i, vp, vp, sz, vp]
        L.mpcnn_seg_loss.argtypes = [vp, vp, vp, vp, i, i, i, vp, vp, sz, vp]
        L.mpcnn_armijo_step.argtypes = [vp, vp, vp, vp, i, i, i, C.c_double, C.c_float, C.c_float, C.c_float,
                                        C.c_float, i, vp, sz, vp, C.POINTER(C.c_float), C.POINTER(C.c_double),
                                        C.POINTER(i)]
        L.mpcnn_lbfgs_step.argtypes = [vp, vp, vp, vp, i, i, i, C.c_double, i, C.c_float, C.c_float, C.c_float,
                                       i, vp, sz, vp, C.POINTER(C.c_float), C.POINTER(C.c_double),
                                       C.POINTER(i), C.POINTER(i)]
        L.mpcnn_lbfgs_reset.argtypes = [vp]
        L.mpcnn_set_loss.argtypes = [vp, i]
        L.mpcnn_workspace_bytes_banded.argtypes = [vp, i, i, i]
        L.mpcnn_workspace_bytes_banded.restype = sz
        L.mpcnn_seg_backward_banded.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, vp, sz, vp]
        L.mpcnn_set_activation.argtypes = [vp, i]
        L.mpcnn_set_conv_tiling.argtypes = [vp, i, i]
        L.mpcnn_class_balance_weights.argtypes = [vp, vp, i, i, i, vp, vp, vp]
        L.mpcnn_seg_backward.argtypes = [vp, vp, vp, vp, i, i, i, vp, vp, vp, sz, vp]
        L.mpcnn_sgd_step.argtypes = [vp, C.c_float, C.c_float, vp]
        L.mpcnn_sgd_step_clipped.argtypes = [vp, C.c_double, C.c_double, C.c_double, vp, vp]
        L.mpcnn_grad_list_create.argtypes = [C.POINTER(_Tensor), i, C.POINTER(vp)]
        L.mpcnn_grad_list_destroy.argtypes = [vp]
        L.mpcnn_grad_list_destroy.restype = None
        L.mpcnn_grad_norm.argtypes = [vp, C.c_double, vp, vp]
        L.mpcnn_grad_clip.argtypes = [vp, C.c_double, vp, vp]
        L.mpcnn_sgd_step_list.argtypes = [vp, C.c_double, C.c_double, C.c_double, vp, vp]
        l = C.c_int64
        for f in (L.mpcnn_workspace_bytes_class, L.mpcnn_workspace_bytes_class_call):
            f.argtypes = [l, l, l, i, i]
            f.restype = sz
        L.mpcnn_class_loss.argtypes = [vp, l, vp, l, vp, vp, vp, l, l, l, i, vp, vp, vp, vp, sz, vp]
        L.mpcnn_class_backward.argtypes = [vp, l, vp, l, vp, vp, vp, l, l, l, i, vp, vp, vp, l, vp, vp, vp, sz, vp]
        pk = C.POINTER(_Packed)
        L.mpcnn_rows_pack.argtypes = [vp, l, l, l, i, pk, vp]
        L.mpcnn_rows_unpack.argtypes = [pk, l, l, i, vp, l, vp]
        L.mpcnn_rows_norm.argtypes = [vp, l, vp, l, vp, l, l, i, C.c_double, vp, l, pk, vp, l, pk, vp, vp]
        L.mpcnn_workspace_bytes_norm.argtypes = [l, l]
        L.mpcnn_workspace_bytes_norm.restype = sz
        L.mpcnn_rows_norm_backward.argtypes = [vp, l, vp, l, pk, vp, vp, vp, l, l, l, i, vp, l, vp, vp, sz, vp]
        L.mpcnn_workspace_bytes_weight_grad.argtypes = [l, l, l, i]
        L.mpcnn_workspace_bytes_weight_grad.restype = sz
        L.mpcnn_rows_weight_grad.argtypes = [vp, l, pk, l, l, l, i, vp, i, vp, sz, vp]
        L.mpcnn_workspace_bytes_beam.argtypes = [l, l, l]
        L.mpcnn_workspace_bytes_beam.restype = sz
        L.mpcnn_beam_select.argtypes = [vp, l, vp, vp, vp, l, l, l, l, l, i, vp, vp, vp, vp, vp, sz, vp]
        L.mpcnn_workspace_bytes_class_beam.argtypes = [l, l, l, l, i]
        L.mpcnn_workspace_bytes_class_beam.restype = sz
        L.mpcnn_class_beam.argtypes = [vp, l, vp, l, vp, vp, vp, l, l, l, l, l, l, i, vp, vp, vp, vp, vp, sz, vp]
        L.mpcnn_beam_states_create.argtypes = [C.POINTER(_BeamState), i, l, l, C.POINTER(vp)]
        L.mpcnn_beam_states_destroy.argtypes = [vp]
        L.mpcnn_beam_states_destroy.restype = None
        L.mpcnn_beam_reorder.argtypes = [vp, vp, l, vp]
        L.mpcnn_get_activation.argtypes = [vp, i, vp, sz]
        L.mpcnn_get_argmax.argtypes = [vp, i, vp, sz]
        L.mpcnn_last_error.restype = C.c_char_p
        L.mpcnn_profile_enable.argtypes = [vp, i]
        L.mpcnn_profile_read.argtypes = [vp, C.POINTER(KernelStat), i, C.POINTER(i)]
        _lib = L
    return _lib


def _check(st: int):
    if st != 0:
        raise MpcnnError(st, lib().mpcnn_last_error().decode())


def _stream_handle(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(getattr(stream, "cuda_stream", stream))


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class Net:
    """mpcnn_net handle.  `layers`: (kind, maps, k) triples; see include/mpcnn.h."""

    def __init__(self, layers: Sequence[Tuple[int, int, int]], in_channels: int, patch: int,
                 dtype: int = F32):
        arr = (_LayerDesc * len(layers))(*[_LayerDesc(int(l[0]), int(l[1]), int(l[2]), int(l[3]) if len(l) > 3 else 0)
                                           for l in layers])
        h = C.c_void_p()
        _check(lib().mpcnn_net_create(arr, len(layers), in_channels, patch, dtype, C.byref(h)))
        self._h = h
        self.layers = [tuple(int(v) for v in l) for l in layers]
        self.in_channels = in_channels
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            lib().mpcnn_net_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except TypeError:     # interpreter shutdown: the module's globals are already gone
            pass

    # ---- host-only queries
    @property
    def patch(self) -> int:
        return lib().mpcnn_net_patch(self._h)

    @property
    def n_classes(self) -> int:
        return lib().mpcnn_net_classes(self._h)

    @property
    def param_count(self) -> int:
        return lib().mpcnn_param_count(self._h)

    def layer_shape(self, H: int, W: int, layer: int):
        r, c, ch, sp = C.c_int(), C.c_int(), C.c_int(), C.c_int()
        _check(lib().mpcnn_layer_shape(self._h, H, W, layer, C.byref(r), C.byref(c), C.byref(ch),
                                       C.byref(sp)))
        return r.value, c.value, ch.value, sp.value

    def workspace_bytes(self, B: int, H: int, W: int, training: bool) -> int:
        return lib().mpcnn_workspace_bytes(self._h, B, H, W, 1 if training else 0)

    def plan_describe(self, B: int, H: int, W: int, training: bool) -> str:
        """Text: the kernel, tiling and launch shape of every layer for a call of these sizes."""
        buf = C.create_string_buffer(1 << 16)
        _check(lib().mpcnn_plan_describe(self._h, B, H, W, 1 if training else 0, buf, len(buf)))
        return buf.value.decode()

    # ---- parameters
    def set_params(self, params: np.ndarray):
        p = np.ascontiguousarray(params, dtype=np.float32)
        _check(lib().mpcnn_set_params(self._h, p.ctypes.data, p.size))

    def get_params(self) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.float32)
        _check(lib().mpcnn_get_params(self._h, out.ctypes.data, out.size))
        return out

    def get_grads(self) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.float32)
        _check(lib().mpcnn_get_grads(self._h, out.ctypes.data, out.size))
        return out

    # ---- device calls (torch tensors carry the memory)
    def alloc_workspace(self, B: int, H: int, W: int, training: bool):
        need = self.workspace_bytes(B, H, W, training)
        if need == 0:
            raise MpcnnError(2, "image %dx%d does not fit the net" % (H, W))
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._ws

    def seg_forward(self, image, probs=None, ws=None, stream=None):
        """image [B,C0,H,W] fp32 cuda tensor -> probs [B,n_cls,H-P+1,W-P+1]."""
        B, _, H, W = image.shape
        assert image.is_cuda and image.dtype == torch.float32 and image.is_contiguous()
        if ws is None:
            ws = self.alloc_workspace(B, H, W, False)
        if probs is None:
            probs = torch.empty((B, self.n_classes, H - self.patch + 1, W - self.patch + 1),
                                dtype=torch.float32, device=image.device)
        _check(lib().mpcnn_seg_forward(self._h, _ptr(image), B, H, W, _ptr(probs), _ptr(ws),
                                       ws.numel(), _stream_handle(stream)))
        return probs

    def seg_forward_static(self, image, probs, stream=None):
        """seg_forward on the library's fixed device workspace: no allocation anywhere in the
        call (the caller supplies `probs`)."""
        B, _, H, W = image.shape
        _check(lib().mpcnn_seg_forward_static(self._h, _ptr(image), B, H, W, _ptr(probs), _stream_handle(stream)))
        return probs

    def seg_loss(self, image, labels, pixw=None, ws=None, stream=None) -> float:
        """Summed loss at the current parameters (forward only, nothing kept)."""
        B, _, H, W = image.shape
        if ws is None:
            ws = self.alloc_workspace(B, H, W, False)
        loss = torch.zeros(1, dtype=torch.float64, device=image.device)
        _check(lib().mpcnn_seg_loss(self._h, _ptr(image), _ptr(labels), _ptr(pixw), B, H, W, _ptr(loss),
                                    _ptr(ws), ws.numel(), _stream_handle(stream)))
        return float(loss.item())

    def armijo_step(self, image, labels, f0, alpha0, pixw=None, grad_scale=1.0, c=1e-4, beta=0.5,
                    max_trials=20, ws=None, stream=None):
        """Safeguarded gradient step after seg_backward on the same inputs -> (alpha, loss, trials)."""
        B, _, H, W = image.shape
        if ws is None:
            ws = self.alloc_workspace(B, H, W, False)
        a, f, t = C.c_float(0), C.c_double(0), C.c_int(0)
        _check(lib().mpcnn_armijo_step(self._h, _ptr(image), _ptr(labels), _ptr(pixw), B, H, W, f0, alpha0,
                                       grad_scale, c, beta, max_trials, _ptr(ws), ws.numel(),
                                       _stream_handle(stream), C.byref(a), C.byref(f), C.byref(t)))
        return a.value, f.value, t.value

    def lbfgs_step(self, image, labels, f0, history=8, alpha0=1.0, pixw=None, c=1e-4, beta=0.5,
                   max_trials=20, ws=None, stream=None):
        """Limited-memory BFGS iteration after seg_backward on the same inputs
        -> (alpha, loss, trials, pairs used)."""
        B, _, H, W = image.shape
        if ws is None:
            ws = self.alloc_workspace(B, H, W, False)
        a, f, t, m = C.c_float(0), C.c_double(0), C.c_int(0), C.c_int(0)
        _check(lib().mpcnn_lbfgs_step(self._h, _ptr(image), _ptr(labels), _ptr(pixw), B, H, W, f0, history,
                                      alpha0, c, beta, max_trials, _ptr(ws), ws.numel(),
                                      _stream_handle(stream), C.byref(a), C.byref(f), C.byref(t), C.byref(m)))
        return a.value, f.value, t.value, m.value

    def lbfgs_reset(self):
        _check(lib().mpcnn_lbfgs_reset(self._h))

    def set_loss(self, kind: str):
        """"mcce": softmax + cross-entropy (default); "mse": linear outputs, half the squared error."""
        _check(lib().mpcnn_set_loss(self._h, {"mcce": 0, "mse": 1}.get(kind, -1)))

    def seg_backward_banded(self, image, labels, band_rows, pixw=None, probs=None, loss=None, stream=None):
        """Forward + backward with the image taken in bands of `band_rows` output rows; the
        workspace (allocated here) is one band's.  Gradients stay in the net."""
        B, _, H, W = image.shape
        assert image.is_cuda and image.dtype == torch.float32 and image.is_contiguous()
        assert labels.dtype == torch.int32 and labels.is_contiguous() and tuple(labels.shape) == (B, H, W)
        n = lib().mpcnn_workspace_bytes_banded(self._h, B, W, band_rows)
        if n == 0:
            raise MpcnnError(2, "no plan for bands of %d rows" % band_rows)
        ws = torch.empty(n, dtype=torch.uint8, device=image.device)
        _check(lib().mpcnn_seg_backward_banded(self._h, _ptr(image), _ptr(labels), _ptr(pixw), B, H, W, band_rows,
                                               _ptr(probs), _ptr(loss), _ptr(ws), ws.numel(),
                                               _stream_handle(stream)))
        return probs, loss

    def set_activation(self, kind: str):
        """"tanh" (default) or "logistic": the squashing function of C and hidden FC layers."""
        _check(lib().mpcnn_set_activation(self._h, {"tanh": 0, "logistic": 1}.get(kind, -1)))

    def set_conv_tiling(self, position_tiles: int = 0, tiles_per_wave: int = 0):
        """Restrict the matrix-core convolution kernel's tiling (0 = the planner's choice)."""
        _check(lib().mpcnn_set_conv_tiling(self._h, position_tiles, tiles_per_wave))

    def class_balance_weights(self, labels, stream=None):
        """labels [B,H,W] int32 cuda -> pixw [B,H,W] fp32 cuda, 1/N_k at output pixels of class k."""
        B, H, W = labels.shape
        assert labels.is_cuda and labels.dtype == torch.int32 and labels.is_contiguous()
        pixw = torch.empty((B, H, W), dtype=torch.float32, device=labels.device)
        counts = torch.empty(16, dtype=torch.int32, device=labels.device)
        _check(lib().mpcnn_class_balance_weights(self._h, _ptr(labels), B, H, W, _ptr(pixw), _ptr(counts),
                                                 _stream_handle(stream)))
        return pixw, counts

    def seg_forward_same(self, image, probs=None, ws=None, stream=None):
        """Deployment forward with mirrored borders: image [B,C0,H,W] -> probs [B,n_cls,H,W]."""
        B, _, H, W = image.shape
        assert image.is_cuda and image.dtype == torch.float32 and image.is_contiguous()
        if ws is None:
            need = lib().mpcnn_workspace_bytes_same(self._h, B, H, W)
            if need == 0:
                raise MpcnnError(2, "image %dx%d does not fit the net" % (H, W))
            if self._ws is None or self._ws.numel() < need:
                self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            ws = self._ws
        if probs is None:
            probs = torch.empty((B, self.n_classes, H, W), dtype=torch.float32, device=image.device)
        _check(lib().mpcnn_seg_forward_same(self._h, _ptr(image), B, H, W, _ptr(probs), _ptr(ws),
                                            ws.numel(), _stream_handle(stream)))
        return probs

    def seg_backward(self, image, labels, pixw=None, probs=None, loss=None, ws=None, stream=None):
        """Forward + backward; gradients stay in the net.  Returns (probs, loss) as given."""
        B, _, H, W = image.shape
        assert image.is_cuda and image.dtype == torch.float32 and image.is_contiguous()
        assert labels.dtype == torch.int32 and labels.is_contiguous() and tuple(labels.shape) == (B, H, W)
        if pixw is not None:
            assert pixw.dtype == torch.float32 and pixw.is_contiguous() and tuple(pixw.shape) == (B, H, W)
        if loss is not None:
            assert loss.dtype == torch.float64 and loss.numel() == 1
        if ws is None:
            ws = self.alloc_workspace(B, H, W, True)
        _check(lib().mpcnn_seg_backward(self._h, _ptr(image), _ptr(labels), _ptr(pixw), B, H, W,
                                        _ptr(probs), _ptr(loss), _ptr(ws), ws.numel(),
                                        _stream_handle(stream)))
        return probs, loss

    def sgd_step(self, lr: float, grad_scale: float = 1.0, stream=None):
        _check(lib().mpcnn_sgd_step(self._h, lr, grad_scale, _stream_handle(stream)))

    def sgd_step_clipped(self, lr: float, max_norm: float, grad_scale: float = 1.0, norm=None, stream=None):
        """sgd_step with the scaled gradient's norm bounded by max_norm; that norm is put into `norm` (one
        fp64 on the GPU) if it is given."""
        if norm is not None:
            _check_norm(norm, None)
        _check(lib().mpcnn_sgd_step_clipped(self._h, lr, grad_scale, max_norm, _ptr(norm), _stream_handle(stream)))
        return norm

    # ---- per-kernel timing
    def profile_enable(self, on: bool):
        _check(lib().mpcnn_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        """List of dicts (name, layer, step, launches, ms_total, flops, bytes), waits for the GPU."""
        cap = 256
        arr = (KernelStat * cap)()
        n = C.c_int(0)
        _check(lib().mpcnn_profile_read(self._h, arr, cap, C.byref(n)))
        return [dict(name=arr[k].name.decode(), layer=arr[k].layer, step=arr[k].step,
                     launches=arr[k].launches, ms_total=arr[k].ms_total, flops=arr[k].flops,
                     bytes=arr[k].bytes) for k in range(min(n.value, cap))]

    # ---- test hooks
    def get_activation(self, B: int, H: int, W: int, layer: int) -> np.ndarray:
        r, c, ch, _ = self.layer_shape(H, W, layer)
        out = np.empty((B, r, c, ch), dtype=np.float32)
        _check(lib().mpcnn_get_activation(self._h, layer, out.ctypes.data, out.size))
        return out

    def get_argmax(self, B: int, H: int, W: int, layer: int) -> np.ndarray:
        r, c, ch, _ = self.layer_shape(H, W, layer)
        out = np.empty((B, r, c, ch), dtype=np.uint8)
        _check(lib().mpcnn_get_argmax(self._h, layer, out.ctypes.data, out.size))
        return out


# ---- tensors of the caller's own: no net needed

def _refuse(text: str):
    raise MpcnnError(1, text)


def _check_norm(norm, device):
    if norm.dtype != torch.float64 or norm.numel() != 1 or not norm.is_cuda or (device is not None and norm.device != device):
        _refuse("norm: one fp64 on the tensors' GPU")


class _On:
    """The tensors' GPU and the stream a call goes to (None: that GPU's current one), made current: memory that
    is allocated inside belongs to that stream, as the work on it does."""
    __slots__ = ("handle", "ctx")

    def __init__(self, device, stream):
        self.ctx = None
        if stream is None:
            self.handle = torch._C._cuda_getCurrentRawStream(device.index)
            if device.index != torch.cuda.current_device():
                self.ctx = torch.cuda.device(device)
        else:
            self.handle = int(getattr(stream, "cuda_stream", stream))
            if not hasattr(stream, "cuda_stream"):
                stream = torch.cuda.ExternalStream(self.handle, device=device)
            if stream.device != device:
                _refuse("the stream belongs to %s, the tensors to %s" % (stream.device, device))
            self.ctx = torch.cuda.stream(stream)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self.handle

    def __exit__(self, *error):
        if self.ctx is not None:
            self.ctx.__exit__(*error)


_STORAGE = {}


def _dtype_of(t) -> int:
    kind = _STORAGE.get(t.dtype)
    if kind is None:
        _STORAGE.update({torch.float32: F32, torch.bfloat16: BF16})        # (the first time)
        kind = _STORAGE.get(t.dtype)
        if kind is None:
            _refuse("%s: fp32 and bf16 are supported" % t.dtype)
    return kind


class GradList:
    """mpcnn_grad_list handle: gradients (dense tensors on one GPU, fp32 or bf16, of any shape) and, for
    sgd_step, the parameters they belong to.  The list keeps the tensors alive and works on their memory."""

    def __init__(self, grads, params=None):
        self._h = None
        self.grads = list(grads)
        self.params = None if params is None else list(params)
        if self.params is not None and len(self.params) != len(self.grads):
            _refuse("%d gradients, %d parameters" % (len(self.grads), len(self.params)))
        every = self.grads + (self.params or [])
        self.device = every[0].device if every else torch.device("cuda", torch.cuda.current_device())
        for t in every:
            if not t.is_cuda or t.device != self.device:
                _refuse("every tensor has to be on one GPU: %s, %s" % (t.device, self.device))
            if not t.is_contiguous():
                _refuse("tensors have to be contiguous: strides %s of %s" % (tuple(t.stride()), tuple(t.shape)))
        arr = (_Tensor * max(1, len(self.grads)))()
        for k, g in enumerate(self.grads):
            arr[k].grad, arr[k].n, arr[k].grad_dtype = g.data_ptr(), g.numel(), _dtype_of(g)
            if self.params is not None:
                p = self.params[k]
                if p.numel() != g.numel():
                    _refuse("tensor %d: %d gradients, %d parameters" % (k, g.numel(), p.numel()))
                arr[k].param, arr[k].param_dtype = p.data_ptr(), _dtype_of(p)
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().mpcnn_grad_list_create(arr, len(self.grads), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().mpcnn_grad_list_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except TypeError:     # interpreter shutdown: the module's globals are already gone
            pass

    def _norm(self, norm):
        if norm is None:
            return torch.empty(1, dtype=torch.float64, device=self.device)
        _check_norm(norm, self.device)
        return norm

    def norm(self, grad_scale: float = 1.0, norm=None, stream=None):
        """|grad_scale| times the 2-norm over all gradients: one fp64 on the GPU."""
        with _On(self.device, stream) as st:
            norm = self._norm(norm)
            _check(lib().mpcnn_grad_norm(self._h, grad_scale, norm.data_ptr(), st))
        return norm

    def clip(self, max_norm: float, norm=None, stream=None):
        """Scale the gradients down to a norm of at most max_norm -> their norm before."""
        with _On(self.device, stream) as st:
            norm = self._norm(norm)
            _check(lib().mpcnn_grad_clip(self._h, max_norm, norm.data_ptr(), st))
        return norm

    def sgd_step(self, lr: float, grad_scale: float = 1.0, max_norm: float = float("inf"), norm=None, stream=None):
        """parameters -= lr * grad_scale * gradients, the scaled gradients' norm bounded by max_norm -> that
        norm before the bound."""
        with _On(self.device, stream) as st:
            norm = self._norm(norm)
            _check(lib().mpcnn_sgd_step_list(self._h, lr, grad_scale, max_norm, norm.data_ptr(), st))
        return norm


def class_workspace_bytes(rows: int, features: int, classes: int, dtype: int, training: bool) -> int:
    """Bytes of workspace that are enough for class_loss (training: class_backward) on so many rows or fewer."""
    return lib().mpcnn_workspace_bytes_class(rows, features, classes, dtype, 1 if training else 0)


def _rows_of(name, t, device, dtype):
    """A matrix whose rows are dense -> its rows, columns and pitch in elements."""
    if t.dtype is not dtype or t.dim() != 2 or t.device != device:
        _refuse("%s: a %s matrix on %s is wanted" % (name, dtype, device))
    rows, columns = t.shape
    if t.is_contiguous():
        return rows, columns, columns
    stride = t.stride()
    if columns > 1 and stride[1] != 1:
        _refuse("%s: the numbers of a row have to be consecutive" % name)
    return rows, columns, stride[0] if rows > 1 else max(columns, stride[0])


def _vector(name, t, n, dtype, device):
    if t is None:
        return None
    if t.dtype != dtype or t.shape != (n,) or t.device != device or not t.is_contiguous():
        _refuse("%s: %d numbers %s on %s are wanted, consecutive" % (name, n, dtype, device))
    return t.data_ptr()


def _class_call(x, w, labels, bias, roww):
    """The arguments that class_loss and class_backward share, checked; and the tensors' GPU."""
    device, dtype = x.device, x.dtype
    if device.type != "cuda":
        _refuse("x: a tensor on a GPU is wanted")
    kind = _dtype_of(x)
    rows, features, x_pitch = _rows_of("x", x, device, dtype)
    classes, columns, w_pitch = _rows_of("w", w, device, dtype)
    if columns != features:
        _refuse("x has %d features, w %d" % (features, columns))
    f32 = torch.float32
    return device, (x.data_ptr(), x_pitch, w.data_ptr(), w_pitch, _vector("bias", bias, classes, f32, device),
                    _vector("labels", labels, rows, torch.int32, device), _vector("roww", roww, rows, f32, device),
                    rows, features, classes, kind)


def _new(shape, dtype, device):
    """A new tensor of one or two dimensions, dense (strides given: it takes three quarters of the time)."""
    return torch.empty_strided(shape, (1,) if len(shape) == 1 else (shape[1], 1), dtype=dtype, device=device)


def _output(name, given, shape, dtype, device):
    """Given (checked), allocated (None) or not asked for (False) -> the tensor or None."""
    if given is None:
        return _new(shape, dtype, device)
    if given is False:
        return None
    if given.dtype != dtype or given.device != device or given.shape != shape:
        _refuse("%s: %s of shape %s on %s is wanted" % (name, dtype, shape, device))
    if name != "dx" and not given.is_contiguous():
        _refuse("%s has to be contiguous" % name)
    return given


def _class_workspace(ws, args, training, device):
    """Address and bytes of the workspace, and what keeps it."""
    if ws is None:
        ws = torch.empty(max(256, lib().mpcnn_workspace_bytes_class_call(*args[7:], training)), dtype=torch.uint8, device=device)
    elif ws.device != device or not ws.is_contiguous():
        _refuse("ws: contiguous memory on %s is wanted" % device)
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def class_loss(x, w, labels, bias=None, roww=None, rowloss=None, lse=None, loss=None, ws=None, stream=None):
    """Softmax cross-entropy of a class layer on rows of features, for any number of classes (the scores are not kept).

    x [rows, features] and w [classes, features], fp32 or bf16, rows dense; labels [rows] int32; bias [classes]
    and roww [rows] fp32 or None.  -> (loss, rowloss, lse): the summed loss (one fp64), w * -log p[label] and
    log sum exp of the scores per row (fp32), put into the tensors given, allocated for None, left out for False."""
    device, args = _class_call(x, w, labels, bias, roww)
    with _On(device, stream) as st:
        loss = _output("loss", loss, (1,), torch.float64, device)
        rowloss = _output("rowloss", rowloss, (args[7],), torch.float32, device)
        lse = _output("lse", lse, (args[7],), torch.float32, device)
        at, size, _kept = _class_workspace(ws, args, 0, device)
        _check(lib().mpcnn_class_loss(*args, _ptr(rowloss), _ptr(lse), _ptr(loss), at, size, st))
    return loss, rowloss, lse


def class_backward(x, w, labels, bias=None, roww=None, rowloss=None, loss=None, dx=None, dw=None, db=None, ws=None, stream=None):
    """class_loss and its gradients -> (loss, rowloss, dx, dw, db); dx and dw have x's type, db (None without
    a bias) is fp32.  Each is put into the tensor given (dx: its rows dense), allocated for None, left out for False.
    Its losses can differ from class_loss's in the last bits."""
    device, args = _class_call(x, w, labels, bias, roww)
    rows, features, classes = args[7:10]
    with _On(device, stream) as st:
        loss = _output("loss", loss, (1,), torch.float64, device)
        rowloss = _output("rowloss", rowloss, (rows,), torch.float32, device)
        pitch = features
        if dx is None:
            dx = torch.empty(rows, features, dtype=x.dtype, device=device)
        else:
            dx = _output("dx", dx, (rows, features), x.dtype, device)
            if dx is not None:
                pitch = _rows_of("dx", dx, device, x.dtype)[2]
        dw = _output("dw", dw, (classes, features), x.dtype, device)
        db = _output("db", False if bias is None and db is None else db, (classes,), torch.float32, device)
        at, size, _kept = _class_workspace(ws, args, 1, device)
        _check(lib().mpcnn_class_backward(*args, _ptr(rowloss), _ptr(loss), _ptr(dx), pitch, _ptr(dw), _ptr(db), at, size, st))
    return loss, rowloss, dx, dw, db


# ---- rows beside the class layer: in 8 bits, and their norm

class PackedRows:
    """Rows of features in 8 bits (mpcnn_packed): `values` [rows, features rounded up to 32], int8 or float8_e4m3fn, zeros behind the
    last feature, and `scales` [rows, blocks of 32 features] uint8: 127 + the exponent of the block's power of two, 255 for a block that is not finite.
    Their contents may be written, the tensors not be replaced."""
    __slots__ = ("_values", "_scales", "_features", "_kind", "_c")
    values, scales, features, kind = (property(operator.attrgetter(name)) for name in __slots__[:4])

    def __init__(self, values, scales, features: int):
        kind = {torch.int8: I8, torch.float8_e4m3fn: E4M3}.get(values.dtype)
        if kind is None:
            _refuse("values: %s: int8 and float8_e4m3fn are supported" % values.dtype)
        blocks = (features + 31) // 32
        if features < 1 or values.dim() != 2 or values.shape[1] != 32 * blocks or not values.is_contiguous() or not values.is_cuda:
            _refuse("values: a contiguous matrix of %d columns on a GPU is wanted" % (32 * blocks))
        if scales.dtype != torch.uint8 or scales.shape != (values.shape[0], blocks) or not scales.is_contiguous() or scales.device != values.device:
            _refuse("scales: [%d, %d] uint8 on %s are wanted, contiguous" % (values.shape[0], blocks, values.device))
        self._values, self._scales, self._features, self._kind = values, scales, features, kind
        self._c = _Packed(values.data_ptr(), scales.data_ptr(), kind)

    @classmethod
    def empty(cls, rows: int, features: int, kind: int, device):
        if kind not in (I8, E4M3) or isinstance(kind, bool):
            _refuse("unknown kind %r of rows in 8 bits" % (kind,))
        if rows < 0 or features < 1:
            _refuse("%d rows of %d features in 8 bits" % (rows, features))
        blocks = (features + 31) // 32
        self = cls.__new__(cls)            # (nothing to check)
        self._values = _new((rows, 32 * blocks), torch.int8 if kind == I8 else torch.float8_e4m3fn, device)
        self._scales = _new((rows, blocks), torch.uint8, device)
        self._features, self._kind = features, kind
        self._c = _Packed(self._values.data_ptr(), self._scales.data_ptr(), kind)
        return self

    @property
    def rows(self) -> int:
        return self._values.shape[0]

    @property
    def device(self):
        return self._values.device


def _here(device, stream):
    """The handle of the current stream, where a call goes there and its tensors' GPU is the current one; else None: the call is made inside _On."""
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None and device.index == torch._C._cuda_getDevice() else None


def _on_gpu(name, x):
    """A matrix of rows on a GPU -> (device, kind, rows, features, pitch)."""
    device = x.device
    if device.type != "cuda":
        _refuse("%s: a tensor on a GPU is wanted" % name)
    return (device, _dtype_of(x)) + _rows_of(name, x, device, x.dtype)


def _matrix_out(name, given, rows, features, dtype, device):
    """A matrix to write, given (its rows dense), allocated (None) or left out (False) -> the tensor or None, its address, its pitch."""
    if given is None:
        given = _new((rows, features), dtype, device)
        return given, given.data_ptr(), features
    if given is False:
        return None, None, features
    if given.shape != (rows, features):
        _refuse("%s: %d rows of %d features are wanted" % (name, rows, features))
    return given, given.data_ptr(), _rows_of(name, given, device, dtype)[2]


def _packed_out(name, given, rows, features, device):
    """PackedRows, given or a kind to allocate them in."""
    if not isinstance(given, PackedRows):
        return PackedRows.empty(rows, features, given, device)
    if given._values.shape[0] != rows or given._features != features or given._values.device != device:
        _refuse("%s: %d rows of %d features in 8 bits on %s are wanted" % (name, rows, features, device))
    return given


def _is_kind(v) -> bool:
    return isinstance(v, PackedRows) or (isinstance(v, int) and not isinstance(v, bool))


def _like(name, t, rows, features, dtype, device):
    """Another input of the same shape, or None -> its address and pitch."""
    if t is None:
        return None, features
    got = _rows_of(name, t, device, dtype)
    if got[:2] != (rows, features):
        _refuse("%s: %d rows of %d features are wanted" % (name, rows, features))
    return t.data_ptr(), got[2]


def rows_pack(x, kind=I8, stream=None) -> PackedRows:
    """Rows of features (fp32 or bf16) into 8 bits, I8 or E4M3, blocks of 32 features with a power of two each; `kind` may be the PackedRows to
    write into."""
    device, dtype, rows, features, pitch = _on_gpu("x", x)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return rows_pack(x, kind)
    out = _packed_out("kind", kind, rows, features, device)
    _check(lib().mpcnn_rows_pack(x.data_ptr(), pitch, rows, features, dtype, C.byref(out._c), st))
    return out


def rows_unpack(packed: PackedRows, out=None, stream=None):
    """What rows in 8 bits stand for, into `out` (fp32 or bf16, exact in both; None: a new bf16 tensor)."""
    device, rows, features = packed.device, packed.rows, packed.features
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return rows_unpack(packed, out)
    dtype = torch.bfloat16 if out is None else out.dtype
    out, at, pitch = _matrix_out("out", out, rows, features, dtype, device)
    _check(lib().mpcnn_rows_unpack(C.byref(packed._c), rows, features, _dtype_of(out), at, pitch, st))
    return out


def rows_norm(x, gain, residual=None, eps: float = 1e-6, y=None, h=None, kept=False, rstd=None, stream=None):
    """Root-mean-square norm of rows, with the residual's addition: h = x + residual, y = h / sqrt(mean h^2 + eps) * gain.

    x [rows, features] fp32 or bf16, rows dense, residual likewise or None; gain [features] fp32.  -> (y, h, kept, rstd).
    y: a tensor of x's type, or in 8 bits: a kind (I8, E4M3) or PackedRows to write into.  h: the sum in x's type (without a residual only if asked
    for by a tensor); kept: the sum in 8 bits, a kind or PackedRows.  rstd [rows] fp32.  Each is put into what is given, allocated for None, left out
    for False.  y and h may be x or residual itself."""
    device, dtype, rows, features, x_pitch = _on_gpu("x", x)
    res, res_pitch = _like("residual", residual, rows, features, x.dtype, device)
    g = _vector("gain", gain, features, torch.float32, device)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return rows_norm(x, gain, residual, eps, y, h, kept, rstd)
    y_at, y_pitch, y8, h8 = None, features, None, None
    if _is_kind(y):
        y = _packed_out("y", y, rows, features, device)
        y8 = C.byref(y._c)
    else:
        y, y_at, y_pitch = _matrix_out("y", y, rows, features, x.dtype, device)
    h, h_at, h_pitch = _matrix_out("h", False if h is None and residual is None else h, rows, features, x.dtype, device)
    if kept is not False:
        kept = _packed_out("kept", I8 if kept is None else kept, rows, features, device)
        h8 = C.byref(kept._c)
    else:
        kept = None
    rstd = _output("rstd", rstd, (rows,), torch.float32, device)
    _check(lib().mpcnn_rows_norm(x.data_ptr(), x_pitch, res, res_pitch, g, rows, features, dtype, eps, y_at, y_pitch, y8, h_at, h_pitch, h8,
                                 _ptr(rstd), st))
    return y, h, kept, rstd


@lru_cache(maxsize=4096)
def norm_workspace_bytes(rows: int, features: int) -> int:
    """Bytes of workspace that are enough for rows_norm_backward on so many rows or fewer."""
    return lib().mpcnn_workspace_bytes_norm(rows, features)


def _workspace(ws, size, device):
    """The workspace's address and bytes, and what keeps it."""
    if ws is None:
        size = max(256, size)
        ws = _new((size,), torch.uint8, device)
        return ws.data_ptr(), size, ws
    if ws.device != device or not ws.is_contiguous():
        _refuse("ws: contiguous memory on %s is wanted" % device)
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def rows_norm_backward(dy, h, gain, rstd, dh=None, dx=None, dgain=None, ws=None, stream=None):
    """Gradients of rows_norm -> (dx, dgain), from the gradients dy of y and dh of h (or None), and h as a tensor or as the PackedRows that were kept.
    dx (x's gradient and the residual's, dy's type) may be dy, dh or h itself; dgain is fp32.  Each is put into the tensor given, allocated for
    None, left out for False.  A row of dy that is zero throughout adds nothing, whatever h holds there."""
    device, dtype, rows, features, dy_pitch = _on_gpu("dy", dy)
    h_at, h_pitch, h8 = None, features, None
    if isinstance(h, PackedRows):
        _packed_out("h", h, rows, features, device)
        h8 = C.byref(h._c)
    else:
        h_at, h_pitch = _like("h", h, rows, features, dy.dtype, device)
    more, more_pitch = _like("dh", dh, rows, features, dy.dtype, device)
    g, r = _vector("gain", gain, features, torch.float32, device), _vector("rstd", rstd, rows, torch.float32, device)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return rows_norm_backward(dy, h, gain, rstd, dh, dx, dgain, ws)
    dx, dx_at, dx_pitch = _matrix_out("dx", dx, rows, features, dy.dtype, device)
    dgain = _output("dgain", dgain, (features,), torch.float32, device)
    at, size, _kept = _workspace(ws, norm_workspace_bytes(rows, features) if ws is None else 0, device)
    _check(lib().mpcnn_rows_norm_backward(dy.data_ptr(), dy_pitch, h_at, h_pitch, h8, g, r, more, more_pitch, rows, features, dtype, dx_at, dx_pitch,
                                          _ptr(dgain), at, size, st))
    return dx, dgain


@lru_cache(maxsize=4096)
def weight_grad_workspace_bytes(rows: int, outs: int, features: int, dtype: int) -> int:
    """Bytes of workspace that are enough for rows_weight_grad on so many rows or fewer."""
    return lib().mpcnn_workspace_bytes_weight_grad(rows, outs, features, dtype)


def rows_weight_grad(dy, x: PackedRows, dw=None, ws=None, stream=None):
    """The gradient of a linear layer's weights, dw[o, f] = sum over the rows of dy[n, o] x[n, f], from the layer's input rows in 8 bits.

    dy [rows, outs] fp32 or bf16, rows dense; dw [outs, features]: given (fp32 or bf16) or allocated in dy's type."""
    device, dtype, rows, outs, pitch = _on_gpu("dy", dy)
    if not isinstance(x, PackedRows):
        _refuse("x: PackedRows are wanted")
    features = x.features
    _packed_out("x", x, rows, features, device)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return rows_weight_grad(dy, x, dw, ws)
    if dw is None:
        dw = _new((outs, features), dy.dtype, device)
    else:
        _output("dw", dw, (outs, features), dw.dtype, device)
    at, size, _kept = _workspace(ws, weight_grad_workspace_bytes(rows, outs, features, dtype) if ws is None else 0, device)
    _check(lib().mpcnn_rows_weight_grad(dy.data_ptr(), pitch, C.byref(x._c), rows, outs, features, dtype, dw.data_ptr(), _dtype_of(dw), at, size, st))
    return dw


# ---- beam search over a class layer's classes

@lru_cache(maxsize=4096)
def beam_workspace_bytes(sequences: int, beams: int, classes: int) -> int:
    """Bytes of workspace that are enough for beam_select on so many sequences or fewer."""
    return lib().mpcnn_workspace_bytes_beam(sequences, beams, classes)


def _beams(totals, done, device):
    """Sequences and beams, and the addresses of what is known of the beams."""
    if totals.dim() != 2 or totals.dtype != torch.float32 or totals.device != device or not totals.is_contiguous():
        _refuse("totals: [sequences, beams] fp32 on %s are wanted, consecutive" % device)
    if done is not None and (done.dtype not in (torch.bool, torch.uint8) or done.shape != totals.shape or done.device != device or not done.is_contiguous()):
        _refuse("done: %s bool on %s are wanted, consecutive" % (tuple(totals.shape), device))
    return totals.shape[0], totals.shape[1]


def _beam_outputs(out, sequences, width, device):
    """What a selection writes: given as (totals, parents, classes, done), or allocated."""
    if not 0 < width < 1 << 16:
        _refuse("width = %r" % (width,))
    if out is None:
        shape = (sequences, width)
        return (_new(shape, torch.float32, device), _new(shape, torch.int32, device), _new(shape, torch.int32, device), _new(shape, torch.bool, device))
    totals, parents, classes, done = out
    for name, t, dtype in (("totals", totals, torch.float32), ("parents", parents, torch.int32), ("classes", classes, torch.int32), ("done", done, torch.bool)):
        _output(name, t, (sequences, width), dtype, device)
    return out


def beam_select(scores, totals, width=None, bias=None, done=None, end: int = -1, out=None, ws=None, stream=None):
    """The continuations of every sequence's beams that go on -> (totals, parents, classes, done), each [sequences, width], best first.

    scores [sequences * beams, classes] fp32 or bf16, rows dense; totals [sequences, beams] fp32: the beams' log-probabilities so far (minus infinity: dead);
    bias [classes] fp32 or None (minus infinity: off); done [sequences, beams] bool or None: finished beams, which offer class `end` at their total; width:
    how many go on (None: as many as there are).  totals fp32, parents (beams of the sequence) and classes int32, done bool; minus infinity, -1, -1
    and True where there is no candidate.  `out`: four such tensors to write into."""
    device, kind, rows, classes, pitch = _on_gpu("scores", scores)
    sequences, beams = _beams(totals, done, device)
    if rows != sequences * beams:
        _refuse("scores: %d rows of %d sequences of %d beams" % (rows, sequences, beams))
    width = beams if width is None else width
    b = _vector("bias", bias, classes, torch.float32, device)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return beam_select(scores, totals, width, bias, done, end, out, ws)
    out = _beam_outputs(out, sequences, width, device)
    at, size, _kept = _workspace(ws, beam_workspace_bytes(sequences, beams, classes) if ws is None else 0, device)
    _check(lib().mpcnn_beam_select(scores.data_ptr(), pitch, b, totals.data_ptr(), _ptr(done), end, sequences, beams, width, classes, kind,
                                   out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(), at, size, st))
    return out


@lru_cache(maxsize=4096)
def class_beam_workspace_bytes(sequences: int, beams: int, features: int, classes: int, dtype: int) -> int:
    """Bytes of workspace that are enough for class_beam on so many sequences or fewer."""
    return lib().mpcnn_workspace_bytes_class_beam(sequences, beams, features, classes, dtype)


def class_beam(x, w, totals, width=None, bias=None, done=None, end: int = -1, out=None, ws=None, stream=None):
    """beam_select on the scores of a class layer: x [sequences * beams, features] and w [classes, features], fp32 or bf16, rows dense; the rest as there."""
    device, kind, rows, features, x_pitch = _on_gpu("x", x)
    classes, columns, w_pitch = _rows_of("w", w, device, x.dtype)
    if columns != features:
        _refuse("x has %d features, w %d" % (features, columns))
    sequences, beams = _beams(totals, done, device)
    if rows != sequences * beams:
        _refuse("x: %d rows of %d sequences of %d beams" % (rows, sequences, beams))
    width = beams if width is None else width
    b = _vector("bias", bias, classes, torch.float32, device)
    st = _here(device, stream)
    if st is None:
        with _On(device, stream):
            return class_beam(x, w, totals, width, bias, done, end, out, ws)
    out = _beam_outputs(out, sequences, width, device)
    at, size, _kept = _workspace(ws, class_beam_workspace_bytes(sequences, beams, features, classes, kind) if ws is None else 0, device)
    _check(lib().mpcnn_class_beam(x.data_ptr(), x_pitch, w.data_ptr(), w_pitch, b, totals.data_ptr(), _ptr(done), end, sequences, beams, width, features,
                                  classes, kind, out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(), at, size, st))
    return out


class BeamStates:
    """mpcnn_beam_states handle: tensors [sequences * beams, ...] on one GPU, of any types, each row dense, that follow the beams.  With `axis`, reorder can be
    told to move the first positions along that axis only.  The list keeps the tensors alive and works on their memory."""

    def __init__(self, tensors, sequences: int, beams: int, axis: Optional[int] = None):
        self._h = None
        self.tensors, self.sequences, self.beams = list(tensors), sequences, beams
        self.device = self.tensors[0].device if self.tensors else torch.device("cuda", torch.cuda.current_device())
        arr = (_BeamState * max(1, len(self.tensors)))()
        for k, t in enumerate(self.tensors):
            if not t.is_cuda or t.device != self.device:
                _refuse("every state has to be on one GPU: %s, %s" % (t.device, self.device))
            if t.dim() < 1 or t.shape[0] != sequences * beams:
                _refuse("state %d: %d rows are wanted, the shape is %s" % (k, sequences * beams, tuple(t.shape)))
            if axis is not None and not 1 <= axis < t.dim():
                _refuse("state %d: no axis %d in %s" % (k, axis, tuple(t.shape)))
            if t.numel() and not t[0].is_contiguous():
                _refuse("state %d: rows have to be dense: strides %s of %s" % (k, tuple(t.stride()), tuple(t.shape)))
            size = t.element_size()
            s = arr[k]
            s.data, s.row_pitch = t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else 0) * size
            s.segments = 1 if axis is None else int(np.prod(t.shape[1:axis], dtype=np.int64))
            s.units = 1 if axis is None else t.shape[axis]
            s.unit_bytes = int(np.prod(t.shape[1:] if axis is None else t.shape[axis + 1:], dtype=np.int64)) * size
            s.segment_pitch = s.units * s.unit_bytes
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().mpcnn_beam_states_create(arr, len(self.tensors), sequences, beams, C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().mpcnn_beam_states_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except TypeError:     # interpreter shutdown: the module's globals are already gone
            pass

    def reorder(self, parents, length: Optional[int] = None, stream=None):
        """Row b * beams + k of every tensor becomes what row b * beams + parents[b, k] was (int32, -1: it stays); with `length`, in the first `length`
        positions only."""
        if parents.dtype != torch.int32 or parents.shape != (self.sequences, self.beams) or parents.device != self.device or not parents.is_contiguous():
            _refuse("parents: [%d, %d] int32 on %s are wanted, consecutive" % (self.sequences, self.beams, self.device))
        if length is not None and length < 0:
            _refuse("length = %d" % length)
        with _On(self.device, stream) as st:
            _check(lib().mpcnn_beam_reorder(self._h, parents.data_ptr(), -1 if length is None else length, st))
