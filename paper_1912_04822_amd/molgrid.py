"""Thin ctypes binding over the C-ABI HIP library (``include/molgrid_hip.h``).

Argument marshalling only: every step of the path runs in the library's
kernels.  PyTorch supplies device memory and the stream.  There is no CPU
fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmolgrid_hip.so")

MG_OK = 0
MG_ESHAPE = -2
MG_EWORKSPACE = -4
EXPORTS = [
    "mg_gridmaker_create", "mg_gridmaker_create_subgrids", "mg_gridmaker_subgrids_per_side",
    "mg_gridmaker_destroy", "mg_gridmaker_points_per_side",
    "mg_workspace_bytes", "mg_transform_forward", "mg_transform_backward", "mg_draw_transforms",
    "mg_forward_index", "mg_forward_index_static", "mg_forward_vector", "mg_forward_index_f64", "mg_forward_vector_f64",
    "mg_backward_index_f64", "mg_backward_vector_f64",
    "mg_backward_index", "mg_backward_vector", "mg_strerror", "mg_last_hip_error",
    "mg_prepare", "mg_forward_index_prepared", "mg_forward_vector_prepared",
    "mg_backward_index_prepared", "mg_backward_vector_prepared",
    "mg_set_option", "mg_time_next_kernel",
    "mg_mx_pack", "mg_mx_unpack", "mg_mx8_weight_gradient", "mg_mx8_weight_gradient_workspace",
    "mg_mx4_product", "mg_mx4_linear", "mg_mx4_linear_workspace",
]

BINDING_PATH = os.path.join(_HERE, "_binding.so")

_lib: Optional[ctypes.CDLL] = None
_binding = None         # the C++ side of the microscaled-format calls, loaded with the library
_no_binding = None      # why it was not, until the first such call has said so


class MolgridError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (code %d)" % (where, strerror(code), code))


def lib(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libmolgrid_hip.so (built by ``paper_1912_04822_amd.build``); raise if absent.
    ``path`` (first call only) names another build of the same library, e.g. the measurement
    build with the timing aids."""
    global _lib, _no_binding
    if _lib is None:
        path = path or LIB_PATH
        if not os.path.exists(path):
            raise FileNotFoundError(
                "HIP library not built: %s (run python -m paper_1912_04822_amd.build)" % path)
        L = ctypes.CDLL(path)
        vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.mg_gridmaker_create.restype = ci
        L.mg_gridmaker_create.argtypes = [ctypes.POINTER(vp), cf, cf, ci, ci, cf, cf]
        L.mg_gridmaker_create_subgrids.restype = ci
        L.mg_gridmaker_create_subgrids.argtypes = [ctypes.POINTER(vp), cf, cf, ci, ci, ci, cf, cf]
        L.mg_gridmaker_subgrids_per_side.restype = ci
        L.mg_gridmaker_subgrids_per_side.argtypes = [vp, ctypes.POINTER(ci)]
        L.mg_gridmaker_destroy.restype = None
        L.mg_gridmaker_destroy.argtypes = [vp]
        L.mg_gridmaker_points_per_side.restype = ci
        L.mg_gridmaker_points_per_side.argtypes = [vp, ctypes.POINTER(ci)]
        L.mg_workspace_bytes.restype = ci
        L.mg_workspace_bytes.argtypes = [vp, ci, ci, ci, ctypes.POINTER(sz)]
        L.mg_transform_forward.restype = ci
        L.mg_transform_forward.argtypes = [ci, ci, vp, vp, vp, vp, vp, vp]
        L.mg_transform_backward.restype = ci
        L.mg_transform_backward.argtypes = [ci, ci, vp, vp, vp, vp, vp, vp]
        L.mg_draw_transforms.restype = ci
        L.mg_draw_transforms.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ci, ci, cf, vp, vp, vp]
        L.mg_forward_index.restype = ci
        L.mg_forward_index.argtypes = [vp, ci, ci, ci] + [vp] * 8 + [vp, sz, vp]
        L.mg_forward_index_static.restype = ci
        L.mg_forward_index_static.argtypes = [vp, ci, ci, ci] + [vp] * 8 + [vp]
        L.mg_forward_vector.restype = ci
        L.mg_forward_vector.argtypes = [vp, ci, ci, ci] + [vp] * 8 + [vp, sz, vp]
        for name, src in (("mg_forward_index_f64", "mg_forward_index"),
                          ("mg_forward_vector_f64", "mg_forward_vector")):
            getattr(L, name).restype = ci
            getattr(L, name).argtypes = [vp, ci, ci, ci] + [vp] * 8 + [vp, sz, vp]
        L.mg_backward_index_f64.restype = ci
        L.mg_backward_index_f64.argtypes = [vp, ci, ci, ci] + [vp] * 9 + [vp, sz, vp]
        L.mg_backward_vector_f64.restype = ci
        L.mg_backward_vector_f64.argtypes = [vp, ci, ci, ci] + [vp] * 10 + [vp, sz, vp]
        L.mg_backward_index.restype = ci
        L.mg_backward_index.argtypes = [vp, ci, ci, ci] + [vp] * 9 + [vp, sz, vp]
        L.mg_backward_vector.restype = ci
        L.mg_backward_vector.argtypes = [vp, ci, ci, ci] + [vp] * 10 + [vp, sz, vp]
        L.mg_prepare.restype = ci
        L.mg_prepare.argtypes = [vp, ci, ci, ci] + [vp] * 7 + [vp, sz, vp]
        L.mg_forward_index_prepared.restype = ci
        L.mg_forward_index_prepared.argtypes = [vp, ci, ci, ci, vp, vp, sz, vp]
        L.mg_forward_vector_prepared.restype = ci
        L.mg_forward_vector_prepared.argtypes = [vp, ci, ci, ci, vp, vp, vp, vp, sz, vp]
        L.mg_backward_index_prepared.restype = ci
        L.mg_backward_index_prepared.argtypes = [vp, ci, ci, ci, vp, vp, vp, sz, vp]
        L.mg_backward_vector_prepared.restype = ci
        L.mg_backward_vector_prepared.argtypes = [vp, ci, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
        i64 = ctypes.c_int64
        for name, args in (
                ("mg_mx_pack", [ci, ci, i64, i64, vp, i64, vp, vp, vp]),
                ("mg_mx_unpack", [ci, ci, i64, i64, vp, vp, vp, i64, vp]),
                ("mg_mx8_weight_gradient_workspace", [ci] * 4 + [ctypes.POINTER(sz)]),
                ("mg_mx8_weight_gradient", [ci] * 6 + [vp, i64] + [vp] * 6 + [sz, vp]),
                ("mg_mx4_product", [ci] * 4 + [vp] * 6 + [i64, vp]),
                ("mg_mx4_linear_workspace", [ci] * 3 + [ctypes.POINTER(sz)]),
                ("mg_mx4_linear", [ci] * 4 + [vp, i64] + [vp] * 4 + [i64, vp, sz, vp])):
            getattr(L, name).restype = ci
            getattr(L, name).argtypes = args
        L.mg_strerror.restype = ctypes.c_char_p
        L.mg_strerror.argtypes = [ci]
        L.mg_last_hip_error.restype = ci
        L.mg_last_hip_error.argtypes = []
        L.mg_set_option.restype = ci
        L.mg_set_option.argtypes = [ctypes.c_char_p, ci]
        L.mg_time_next_kernel.restype = ci
        L.mg_time_next_kernel.argtypes = [vp, vp]
        _lib = L
        try:
            _load_binding(L)
        except (ImportError, OSError) as e:
            _no_binding = str(e)
    return _lib


def _load_binding(L) -> None:
    """Load the C++ side of the binding and hand it the addresses of the library's functions.  It is built against
    one version of torch; without it every call goes through ctypes to the same kernels."""
    global _binding
    if not os.path.exists(BINDING_PATH):
        raise FileNotFoundError(
            "binding not built: %s (run python -m paper_1912_04822_amd.build)" % BINDING_PATH)
    name = __package__ + "._binding"
    spec = importlib.util.spec_from_file_location(name, BINDING_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.bind(*(ctypes.cast(getattr(L, f), ctypes.c_void_p).value for f in (
        "mg_mx_pack", "mg_mx_unpack", "mg_mx8_weight_gradient_workspace", "mg_mx8_weight_gradient",
        "mg_mx4_product", "mg_mx4_linear_workspace", "mg_mx4_linear")))
    _binding = module


def strerror(code: int) -> str:
    return lib().mg_strerror(int(code)).decode()


def set_option(key: str, value: int) -> None:
    rc = lib().mg_set_option(key.encode(), int(value))
    if rc != MG_OK:
        raise MolgridError(rc, "mg_set_option")


def mg_time_next_kernel(start_event: Optional[int], stop_event: Optional[int]) -> None:
    """Have the next forward/backward call record these hipEvent_t handles around its main kernel."""
    lib().mg_time_next_kernel(ctypes.c_void_p(start_event), ctypes.c_void_p(stop_event))


def _ptr(t: Optional[torch.Tensor], dtype, name: str, shape=None):
    """Address of a device tensor after its checks (an int, or None for a missing array)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t.data_ptr()


# torch's own short way to the current stream's handle, without building a Stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def mg_transform_forward(coords, centers=None, quats=None, translations=None, out=None):
    """x' = R(q)(x - c) + c + t per example; [B,N,3] float32 device tensors."""
    B, N, _ = coords.shape
    if out is None:
        out = torch.empty_like(coords)
    rc = lib().mg_transform_forward(
        B, N, _ptr(coords, torch.float32, "coords", (B, N, 3)),
        _ptr(centers, torch.float32, "centers", (B, 3)), _ptr(quats, torch.float32, "quats", (B, 4)),
        _ptr(translations, torch.float32, "translations", (B, 3)),
        _ptr(out, torch.float32, "out", (B, N, 3)), _stream())
    if rc != MG_OK:
        raise MolgridError(rc, "mg_transform_forward")
    return out


def mg_transform_backward(coords, centers=None, quats=None, translations=None, out=None):
    """x = R(q)^T ((x' - t) - c) + c per example; [B,N,3] float32 device tensors."""
    B, N, _ = coords.shape
    if out is None:
        out = torch.empty_like(coords)
    rc = lib().mg_transform_backward(
        B, N, _ptr(coords, torch.float32, "coords", (B, N, 3)),
        _ptr(centers, torch.float32, "centers", (B, 3)), _ptr(quats, torch.float32, "quats", (B, 4)),
        _ptr(translations, torch.float32, "translations", (B, 3)),
        _ptr(out, torch.float32, "out", (B, N, 3)), _stream())
    if rc != MG_OK:
        raise MolgridError(rc, "mg_transform_backward")
    return out


def mg_draw_transforms(seed: int, draw: int, B: int, random_rotation: bool = True,
                       max_translation: float = 0.0, quats=None, translations=None, device=None):
    """Per-example random quaternions [B,4] and translations [B,3] drawn on the device."""
    if quats is None:
        quats = torch.empty((B, 4), dtype=torch.float32, device=device or "cuda")
    if translations is None:
        translations = torch.empty((B, 3), dtype=torch.float32, device=quats.device)
    rc = lib().mg_draw_transforms(
        int(seed) & (2 ** 64 - 1), int(draw) & (2 ** 64 - 1), B, 1 if random_rotation else 0,
        float(max_translation), _ptr(quats, torch.float32, "quats", (B, 4)),
        _ptr(translations, torch.float32, "translations", (B, 3)), _stream())
    if rc != MG_OK:
        raise MolgridError(rc, "mg_draw_transforms")
    return quats, translations


class GridMaker:
    """Handle over ``mg_gridmaker`` (GridMaker constructor listing of the paper)."""

    def __init__(self, resolution=0.5, dimension=23.5, binary=False, radius_type_indexed=False,
                 radius_scale=1.0, gaussian_radius_multiple=1.0, subgrids_per_side=1):
        self._h = ctypes.c_void_p()
        if subgrids_per_side == 1:
            rc = lib().mg_gridmaker_create(ctypes.byref(self._h), resolution, dimension,
                                           int(binary), int(radius_type_indexed), radius_scale,
                                           gaussian_radius_multiple)
        else:
            rc = lib().mg_gridmaker_create_subgrids(
                ctypes.byref(self._h), resolution, dimension, int(subgrids_per_side), int(binary),
                int(radius_type_indexed), radius_scale, gaussian_radius_multiple)
        if rc != MG_OK:
            self._h = ctypes.c_void_p()
            raise MolgridError(rc, "mg_gridmaker_create")
        sps = ctypes.c_int()
        lib().mg_gridmaker_subgrids_per_side(self._h, ctypes.byref(sps))
        self.S = sps.value
        d = ctypes.c_int()
        lib().mg_gridmaker_points_per_side(self._h, ctypes.byref(d))
        self.D = d.value
        self.binary = bool(binary)
        self.radius_type_indexed = bool(radius_type_indexed)
        # workspaces the binding allocated, one per (device, stream): calls on different
        # streams may run at the same time and must not share tables
        self._ws = {}
        self._need = (None, 0)      # the last (B, N, T) asked for and its workspace size

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.mg_gridmaker_destroy(h)
            self._h = ctypes.c_void_p()

    def workspace_bytes(self, B: int, N: int, T: int) -> int:
        n = ctypes.c_size_t()
        rc = lib().mg_workspace_bytes(self._h, B, N, T, ctypes.byref(n))
        if rc != MG_OK:
            raise MolgridError(rc, "mg_workspace_bytes")
        return n.value

    def grid_shape(self, B: int, T: int):
        """[B,T,D,D,D], or [B,S,S,S,T,D,D,D] for a GridMaker with S > 1 subgrids per side."""
        D, S = self.D, self.S
        return (B, T, D, D, D) if S == 1 else (B, S, S, S, T, D, D, D)

    def _workspace(self, B, N, T, device, workspace, stream):
        """The caller's workspace or this GridMaker's for the stream (the caller of this holds the
        tensor until its kernels are enqueued: another thread may put a larger one in its place)."""
        if workspace is not None:
            self.workspace_bytes(B, N, T)       # raises for shapes no call takes
            return workspace, workspace.numel() * workspace.element_size()
        last, need = self._need
        if last != (B, N, T):
            need = self.workspace_bytes(B, N, T)
            self._need = ((B, N, T), need)
        key = (device, stream)
        ws = self._ws.get(key)
        if ws is None or ws.numel() < need:
            ws = torch.empty(need, dtype=torch.uint8, device=device)
            self._ws[key] = ws
        return ws, ws.numel()

    def _common(self, coords, natoms, centers, quats, translations):
        B, N, _ = coords.shape
        if centers is None and quats is None and translations is None and natoms is None:
            return B, N, _ptr(coords, torch.float32, "coords", (B, N, 3)), None, None, None, None
        return (B, N, _ptr(coords, torch.float32, "coords", (B, N, 3)),
                _ptr(natoms, torch.int32, "natoms", (B,)),
                _ptr(centers, torch.float32, "centers", (B, 3)),
                _ptr(quats, torch.float32, "quats", (B, 4)),
                _ptr(translations, torch.float32, "translations", (B, 3)))

    def mg_forward_index(self, coords, types, radii, T, natoms=None, centers=None, quats=None,
                         translations=None, out=None, workspace=None, dtype=torch.float32):
        """``dtype`` (or ``out.dtype``) torch.float64 calls ``mg_forward_index_f64``."""
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        if out is None:
            out = torch.empty(self.grid_shape(B, T), dtype=dtype, device=coords.device)
        st = _stream()
        ws, wsb = self._workspace(B, N, T, coords.device, workspace, st)
        rshape = (T,) if self.radius_type_indexed else (B, N)
        fn = lib().mg_forward_index_f64 if out.dtype == torch.float64 else lib().mg_forward_index
        rc = fn(
            self._h, B, N, T, pc, _ptr(types, torch.int32, "types", (B, N)),
            _ptr(radii, torch.float32, "radii", rshape), pn, pce, pq, pt,
            _ptr(out, out.dtype, "out", self.grid_shape(B, T)), ws.data_ptr(), wsb, st)
        if rc != MG_OK:
            raise MolgridError(rc, "mg_forward_index")
        return out

    def mg_forward_index_static(self, coords, types, radii, T, out, natoms=None, centers=None,
                                quats=None, translations=None):
        """``mg_forward_index`` with the workspace in the library's static device array: the
        call allocates nothing, so ``out`` is required."""
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        rshape = (T,) if self.radius_type_indexed else (B, N)
        rc = lib().mg_forward_index_static(
            self._h, B, N, T, pc, _ptr(types, torch.int32, "types", (B, N)),
            _ptr(radii, torch.float32, "radii", rshape), pn, pce, pq, pt,
            _ptr(out, torch.float32, "out", self.grid_shape(B, T)), _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_forward_index_static")
        return out

    def mg_forward_vector(self, coords, weights, radii, natoms=None, centers=None, quats=None,
                          translations=None, out=None, workspace=None, dtype=torch.float32):
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        T = weights.shape[2]
        if out is None:
            out = torch.empty(self.grid_shape(B, T), dtype=dtype, device=coords.device)
        st = _stream()
        ws, wsb = self._workspace(B, N, T, coords.device, workspace, st)
        fn = lib().mg_forward_vector_f64 if out.dtype == torch.float64 else lib().mg_forward_vector
        rc = fn(
            self._h, B, N, T, pc, _ptr(weights, torch.float32, "weights", (B, N, T)),
            _ptr(radii, torch.float32, "radii", (T,)), pn, pce, pq, pt,
            _ptr(out, out.dtype, "out", self.grid_shape(B, T)), ws.data_ptr(), wsb, st)
        if rc != MG_OK:
            raise MolgridError(rc, "mg_forward_vector")
        return out

    def mg_backward_index(self, coords, types, radii, T, grad_out, natoms=None, centers=None,
                          quats=None, translations=None, grad_coords=None, workspace=None):
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        if grad_coords is None:
            grad_coords = torch.empty((B, N, 3), dtype=torch.float32, device=coords.device)
        st = _stream()
        ws, wsb = self._workspace(B, N, T, coords.device, workspace, st)
        rshape = (T,) if self.radius_type_indexed else (B, N)
        fn = (lib().mg_backward_index_f64 if grad_out.dtype == torch.float64
              else lib().mg_backward_index)
        rc = fn(
            self._h, B, N, T, pc, _ptr(types, torch.int32, "types", (B, N)),
            _ptr(radii, torch.float32, "radii", rshape), pn, pce, pq, pt,
            _ptr(grad_out, grad_out.dtype, "grad_out", self.grid_shape(B, T)),
            _ptr(grad_coords, torch.float32, "grad_coords", (B, N, 3)),
            ws.data_ptr(), wsb, st)
        if rc != MG_OK:
            raise MolgridError(rc, "mg_backward_index")
        return grad_coords

    def mg_backward_vector(self, coords, weights, radii, grad_out, natoms=None, centers=None,
                           quats=None, translations=None, grad_coords=None, grad_weights=None,
                           want_coords=True, want_weights=True, workspace=None):
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        T = weights.shape[2]
        if grad_coords is None and want_coords:
            grad_coords = torch.empty((B, N, 3), dtype=torch.float32, device=coords.device)
        if grad_weights is None and want_weights:
            grad_weights = torch.empty((B, N, T), dtype=torch.float32, device=coords.device)
        st = _stream()
        ws, wsb = self._workspace(B, N, T, coords.device, workspace, st)
        fn = (lib().mg_backward_vector_f64 if grad_out.dtype == torch.float64
              else lib().mg_backward_vector)
        rc = fn(
            self._h, B, N, T, pc, _ptr(weights, torch.float32, "weights", (B, N, T)),
            _ptr(radii, torch.float32, "radii", (T,)), pn, pce, pq, pt,
            _ptr(grad_out, grad_out.dtype, "grad_out", self.grid_shape(B, T)),
            _ptr(grad_coords, torch.float32, "grad_coords", (B, N, 3)),
            _ptr(grad_weights, torch.float32, "grad_weights", (B, N, T)),
            ws.data_ptr(), wsb, st)
        if rc != MG_OK:
            raise MolgridError(rc, "mg_backward_vector")
        return grad_coords, grad_weights

    # ---- tables once, calls many (mg_prepare + the *_prepared calls) ----

    def mg_prepare(self, coords, types, radii, T, natoms=None, centers=None, quats=None,
                   translations=None, workspace=None):
        """Build the workspace's tables for these atoms and poses (``types=None``: the tables
        of vector types) and return the workspace tensor the ``*_prepared`` calls then take."""
        B, N, pc, pn, pce, pq, pt = self._common(coords, natoms, centers, quats, translations)
        if workspace is None:
            workspace = torch.empty(self.workspace_bytes(B, N, T), dtype=torch.uint8,
                                    device=coords.device)
        rshape = (T,) if (self.radius_type_indexed or types is None) else (B, N)
        rc = lib().mg_prepare(
            self._h, B, N, T, pc, _ptr(types, torch.int32, "types", (B, N)),
            _ptr(radii, torch.float32, "radii", rshape), pn, pce, pq, pt,
            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_prepare")
        return workspace

    def mg_forward_index_prepared(self, B, N, T, workspace, out=None):
        if out is None:
            out = torch.empty(self.grid_shape(B, T), dtype=torch.float32, device=workspace.device)
        rc = lib().mg_forward_index_prepared(
            self._h, B, N, T, _ptr(out, torch.float32, "out", self.grid_shape(B, T)),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_forward_index_prepared")
        return out

    def mg_forward_vector_prepared(self, weights, radii, workspace, out=None):
        B, N, T = weights.shape
        if out is None:
            out = torch.empty(self.grid_shape(B, T), dtype=torch.float32, device=weights.device)
        rc = lib().mg_forward_vector_prepared(
            self._h, B, N, T, _ptr(weights, torch.float32, "weights", (B, N, T)),
            _ptr(radii, torch.float32, "radii", (T,)),
            _ptr(out, torch.float32, "out", self.grid_shape(B, T)),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_forward_vector_prepared")
        return out

    def mg_backward_index_prepared(self, B, N, T, grad_out, workspace, grad_coords=None):
        if grad_coords is None:
            grad_coords = torch.empty((B, N, 3), dtype=torch.float32, device=grad_out.device)
        rc = lib().mg_backward_index_prepared(
            self._h, B, N, T,
            _ptr(grad_out, torch.float32, "grad_out", self.grid_shape(B, T)),
            _ptr(grad_coords, torch.float32, "grad_coords", (B, N, 3)),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_backward_index_prepared")
        return grad_coords

    def mg_backward_vector_prepared(self, weights, radii, grad_out, workspace, grad_coords=None,
                                    grad_weights=None, want_coords=True, want_weights=True):
        B, N, T = weights.shape
        if grad_coords is None and want_coords:
            grad_coords = torch.empty((B, N, 3), dtype=torch.float32, device=weights.device)
        if grad_weights is None and want_weights:
            grad_weights = torch.empty((B, N, T), dtype=torch.float32, device=weights.device)
        rc = lib().mg_backward_vector_prepared(
            self._h, B, N, T, _ptr(weights, torch.float32, "weights", (B, N, T)),
            _ptr(radii, torch.float32, "radii", (T,)),
            _ptr(grad_out, torch.float32, "grad_out", self.grid_shape(B, T)),
            _ptr(grad_coords, torch.float32, "grad_coords", (B, N, 3)),
            _ptr(grad_weights, torch.float32, "grad_weights", (B, N, T)),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            _stream())
        if rc != MG_OK:
            raise MolgridError(rc, "mg_backward_vector_prepared")
        return grad_coords, grad_weights


# ---- microscaled formats: numbers in 8 or 4 bits ----
#
# Like the GridMaker's, these calls record nothing for autograd: what they return has no history, also where
# their arguments require gradients (AtomTyper and saved_in_8_bits are what differentiates).

MX_FORMATS = {"int8": 0, "e4m3": 1, "e2m1": 2}          # MG_MX_INT8, MG_MX_E4M3, MG_MX_E2M1
NUMBERS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}     # MG_F32, MG_F16, MG_BF16


class MXTensor:
    """A tensor in a microscaled format: ``codes`` and ``scales`` (uint8 device tensors laid out as
    include/molgrid_hip.h says, one row for every index but the last), the ``shape`` it stands for,
    the ``format`` ("int8", "e4m3" or "e2m1") and the ``dtype`` ``mg_mx_unpack`` gives back."""

    __slots__ = ("codes", "scales", "shape", "format", "dtype")

    def __init__(self, codes, scales, shape, format, dtype=torch.float32):
        self.codes, self.scales, self.shape = codes, scales, tuple(shape)
        self.format, self.dtype = format, dtype

    @property
    def rows(self):
        n = 1
        for d in self.shape[:-1]:
            n *= d
        return n

    def __repr__(self):
        return "MXTensor(%s, %s)" % (self.format, list(self.shape))


def _mx_layout(shape, format):
    """(rows, columns), shapes of codes and scales."""
    per_block = _BLOCK_BYTES.get(format)
    if per_block is None:
        raise ValueError("format must be one of %s, got %r" % (", ".join(MX_FORMATS), format))
    if len(shape) == 2:
        rows, cols = shape
    elif len(shape) == 0:
        raise ValueError("a tensor in a microscaled format has at least one dimension")
    else:
        rows, cols = 1, shape[-1]
        for d in shape[:-1]:
            rows *= d
    blocks = (cols + 31) >> 5
    return rows, cols, (rows, blocks * per_block), (rows, (blocks + 3) & ~3)


_BLOCK_BYTES = {"int8": 32, "e4m3": 32, "e2m1": 16}


def _is_packed(t, name):
    if not isinstance(t, MXTensor):
        raise TypeError("%s must be an MXTensor, got %s" % (name, type(t).__name__))


def _mx_pointers(t, name, formats, dev):
    """Checks an MXTensor; (rows, columns, codes, scales)."""
    _is_packed(t, name)
    if t.format not in formats:
        raise ValueError("%s must be in %s, got %s" % (name, " or ".join(formats), t.format))
    rows, cols, cshape, sshape = _mx_layout(t.shape, t.format)
    codes, scales = t.codes, t.scales
    if codes.get_device() != dev or scales.get_device() != dev:
        _refuse_device(dev, **{name + ".codes": codes, name + ".scales": scales})
    if (dev >= 0 and codes.dtype is scales.dtype is torch.uint8 and codes.shape == cshape and scales.shape == sshape
            and codes.is_contiguous() and scales.is_contiguous()):
        return rows, cols, codes.data_ptr(), scales.data_ptr()
    return (rows, cols, _ptr(codes, torch.uint8, name + ".codes", cshape),      # says what is wrong
            _ptr(scales, torch.uint8, name + ".scales", sshape))


def _device(t, name):
    """Number of the device a tensor is on."""
    dev = t.get_device()
    if dev < 0 or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    return dev


def _refuse_device(dev, **tensors):
    for name, t in tensors.items():
        if t.get_device() != dev:
            if not t.is_cuda:
                raise ValueError("%s must be a device tensor" % name)
            raise ValueError("%s is on device %d, not on %d" % (name, t.get_device(), dev))


def _optional(t, dtype, name, shape, dev):
    """Address of an array that may be missing, on the call's device."""
    if t is None:
        return None
    if t.get_device() != dev:
        _refuse_device(dev, **{name: t})
    return _ptr(t, dtype, name, shape)


def _number(dtype, name):
    code = NUMBERS.get(dtype)
    if code is None:
        raise TypeError("%s must be float32, float16 or bfloat16, got %s" % (name, dtype))
    return code


def row_stride(t):
    """Elements from row to row of a tensor (a row: its last dimension), or None where rows are not
    contiguous, not equally far apart, or overlap."""
    if t.is_contiguous():
        return t.size(-1)
    cols = t.size(-1)
    if cols > 1 and t.stride(-1) != 1:
        return None
    step = unit = None
    for d in range(t.dim() - 2, -1, -1):        # the innermost dimension that has a step fixes it
        if t.shape[d] == 1:
            continue
        if step is None:
            step = unit = t.stride(d)
        elif t.stride(d) != unit:
            return None
        unit *= t.shape[d]
    if step is None:
        return cols
    return step if step >= cols else None


def _row_stride(t, name):
    if t.is_neg():                              # its memory holds the numbers with the other sign
        raise ValueError("%s is a view that negates: give %s.resolve_neg()" % (name, name))
    step = row_stride(t)
    if step is None:
        raise ValueError("the rows of %s must be contiguous and equally far apart" % name)
    return step


def _fits(name, *sizes):
    """Refuses sizes that the C side's int does not hold (ctypes would cut them)."""
    if max(sizes) > 0x7fffffff:
        raise MolgridError(MG_ESHAPE, name)


# torch's own short way to the number of the current device
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(fn, dev, *args):
    """One library call on the current stream of the tensors' device, whichever device is current."""
    if dev == _current_device() and _raw_stream is not None:
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _stream())
    if rc != MG_OK:
        raise MolgridError(rc, fn.__name__)


def _native(dev):
    """The C++ side of the binding, which takes calls on the current device in their common form (dense
    tensors, new results) and returns None for any other, or None."""
    global _no_binding
    if dev < 0 or _raw_stream is None or dev != _current_device():
        return None
    if _binding is None:
        lib()
        if _no_binding is not None:
            why, _no_binding = _no_binding, None
            warnings.warn("calls on microscaled formats take 4 us more host time each: " + why)
    return _binding


def _taken(r, name):
    """Whether the C++ side took a call; raises the library's error."""
    if r is None:
        return False
    if type(r) is int:
        raise MolgridError(r, name)
    return True


def _workspace_of(fn, like, *sizes):
    """The workspace a call of these sizes needs (bytes from ``fn``), and its size.  A new one for
    every call: calls on several streams, or captured in several graphs, share none."""
    n = ctypes.c_size_t()
    rc = fn(*sizes, ctypes.byref(n))
    if rc != MG_OK:
        raise MolgridError(rc, fn.__name__)
    return (like.new_empty(n.value, dtype=torch.uint8) if n.value else None), n.value


def mg_mx_pack(x, format="int8", out: Optional[MXTensor] = None) -> MXTensor:
    """``x`` (float32, float16 or bfloat16; rows along the last dimension, equally far apart) in
    blocks of 32 numbers that share a power of two."""
    if out is None and format in MX_FORMATS:
        dev = x.get_device()
        native = _native(dev)
        if native is not None:
            r = native.pack(x, MX_FORMATS[format], dev, _raw_stream(dev))
            if _taken(r, "mg_mx_pack"):
                return MXTensor(r[0], r[1], x.shape, format, x.dtype)
    shape = x.shape
    rows, cols, cshape, sshape = _mx_layout(shape, format)
    dtype, stride, dev = _number(x.dtype, "x"), _row_stride(x, "x"), _device(x, "x")
    if out is None:
        out = MXTensor(x.new_empty(cshape, dtype=torch.uint8), x.new_empty(sshape, dtype=torch.uint8), shape,
                       format, x.dtype)
        codes, scales = out.codes.data_ptr(), out.scales.data_ptr()
    else:
        if out.shape != tuple(shape):
            raise ValueError("out must have shape %s, got %s" % (tuple(shape), out.shape))
        _, _, codes, scales = _mx_pointers(out, "out", (format,), dev)
        out.dtype = x.dtype
    _launch(lib().mg_mx_pack, dev, MX_FORMATS[format], dtype, rows, cols, x.data_ptr(), stride, codes, scales)
    return out


def mg_mx_unpack(packed: MXTensor, dtype=None, out=None):
    """The numbers ``packed`` stands for, as a tensor of its shape (``dtype``: default its own)."""
    _is_packed(packed, "packed")
    dev = _device(packed.codes, "packed.codes")
    if out is None:
        native = _native(dev)
        if native is not None:
            r = native.unpack(packed.codes, packed.scales, packed.shape, MX_FORMATS.get(packed.format),
                              NUMBERS.get(dtype or packed.dtype), dev, _raw_stream(dev))
            if _taken(r, "mg_mx_unpack"):
                return r
    rows, cols, codes, scales = _mx_pointers(packed, "packed", MX_FORMATS, dev)
    if out is None:
        out = packed.codes.new_empty(packed.shape, dtype=dtype or packed.dtype)
    elif tuple(out.shape) != packed.shape:
        raise ValueError("out must have shape %s, got %s" % (packed.shape, tuple(out.shape)))
    number, stride = _number(out.dtype, "out"), _row_stride(out, "out")
    if out.get_device() != dev:
        _refuse_device(dev, out=out)
    _launch(lib().mg_mx_unpack, dev, MX_FORMATS[packed.format], number, rows, cols, codes, scales, out.data_ptr(),
            stride)
    return out


def mg_mx8_weight_gradient(grad, packed: MXTensor, natoms=None, grad_weight=None, grad_bias=None):
    """(``grad_weight`` [T,E], ``grad_bias`` [T]) in float32 of y = x W^T + b, from ``grad`` [...,T]
    on y and the 8-bit codes of x [...,E].  ``natoms`` [B] (x of shape [B,N,E]): atoms past it
    count for nothing, whatever their rows hold."""
    dev = grad.get_device()
    if (grad_weight is None and grad_bias is None and isinstance(packed, MXTensor)
            and packed.format in ("int8", "e4m3")):
        native = _native(dev)
        if native is not None:
            r = native.gradient(grad, packed.codes, packed.scales, packed.shape, MX_FORMATS[packed.format], natoms,
                                dev, _raw_stream(dev))
            if _taken(r, "mg_mx8_weight_gradient"):
                return r
    rows, E, codes, scales = _mx_pointers(packed, "packed", ("int8", "e4m3"), dev)
    T = grad.shape[-1]
    if tuple(grad.shape[:-1]) != packed.shape[:-1]:
        raise ValueError("grad must have shape %s, got %s" % (packed.shape[:-1] + (T,), tuple(grad.shape)))
    B, N = (packed.shape[0], packed.shape[1]) if len(packed.shape) == 3 else (1, rows)
    if natoms is not None and len(packed.shape) != 3:
        raise ValueError("natoms needs x of shape [B,N,E], got %s" % (packed.shape,))
    number, stride = _number(grad.dtype, "grad"), _row_stride(grad, "grad")
    _fits("mg_mx8_weight_gradient", B, N, T, E)
    L = lib()
    ws, size = _workspace_of(L.mg_mx8_weight_gradient_workspace, grad, B, N, T, E)
    if grad_weight is None:
        grad_weight = grad.new_empty((T, E), dtype=torch.float32)
    if grad_bias is None:
        grad_bias = grad.new_empty((T,), dtype=torch.float32)
    _launch(L.mg_mx8_weight_gradient, dev, MX_FORMATS[packed.format], number, B, N, T, E, grad.data_ptr(), stride,
            codes, scales, _optional(natoms, torch.int32, "natoms", (B,), dev),
            _optional(grad_weight, torch.float32, "grad_weight", (T, E), dev),
            _optional(grad_bias, torch.float32, "grad_bias", (T,), dev), None if ws is None else ws.data_ptr(), size)
    return grad_weight, grad_bias


def _product_out(out, shape, dtype, like, dev):
    """The result's tensor and the stride of its rows."""
    if out is None:
        return like.new_empty(shape, dtype=dtype), shape[-1]
    if tuple(out.shape) != tuple(shape):
        raise ValueError("out must have shape %s, got %s" % (tuple(shape), tuple(out.shape)))
    if out.dtype != dtype:
        raise TypeError("out must be %s, got %s" % (dtype, out.dtype))
    if out.get_device() != dev:
        _refuse_device(dev, out=out)
    return out, _row_stride(out, "out")


def mg_mx4_product(a: MXTensor, b: MXTensor, bias=None, dtype=torch.float32, out=None):
    """``a`` [...,K] times ``b`` [N,K] transposed, plus ``bias`` [N] (float32): [...,N] of ``dtype``."""
    _is_packed(a, "a")
    _is_packed(b, "b")
    dev = _device(a.codes, "a.codes")
    if out is None and a.format == "e2m1" and b.format == "e2m1":
        native = _native(dev)
        if native is not None:
            r = native.product(a.codes, a.scales, a.shape, b.codes, b.scales, b.shape, bias, NUMBERS.get(dtype), dev,
                               _raw_stream(dev))
            if _taken(r, "mg_mx4_product"):
                return r
    M, K, ac, asc = _mx_pointers(a, "a", ("e2m1",), dev)
    N, Kb, bc, bsc = _mx_pointers(b, "b", ("e2m1",), dev)
    if K != Kb:
        raise ValueError("rows of a have %d numbers, rows of b %d" % (K, Kb))
    dtype = out.dtype if out is not None else dtype
    number = _number(dtype, "dtype")
    _fits("mg_mx4_product", M, N, K)
    out, stride = _product_out(out, a.shape[:-1] + (N,), dtype, a.codes, dev)
    _launch(lib().mg_mx4_product, dev, number, M, N, K, ac, asc, bc, bsc,
            _optional(bias, torch.float32, "bias", (N,), dev), out.data_ptr(), stride)
    return out


def mg_mx4_linear(x, weight: MXTensor, bias=None, out=None):
    """``x`` [...,K] (plain numbers, taken to "e2m1" by the call) times ``weight`` [N,K] transposed,
    plus ``bias`` [N] (float32): [...,N] in the type of ``x``."""
    dev = x.get_device()
    if out is None and isinstance(weight, MXTensor) and weight.format == "e2m1":
        native = _native(dev)
        if native is not None:
            r = native.linear(x, weight.codes, weight.scales, weight.shape, bias, dev, _raw_stream(dev))
            if _taken(r, "mg_mx4_linear"):
                return r
    N, K, wc, wsc = _mx_pointers(weight, "weight", ("e2m1",), dev)
    shape = x.shape
    if shape[-1] != K:
        raise ValueError("rows of x have %d numbers, rows of weight %d" % (shape[-1], K))
    number, stride = _number(x.dtype, "x"), _row_stride(x, "x")
    M = shape[0] if len(shape) == 2 else shape[:-1].numel()
    _fits("mg_mx4_linear", M, N, K)
    out, ostride = _product_out(out, shape[:-1] + (N,), x.dtype, x, dev)
    fn = lib().mg_mx4_linear
    args = (number, M, N, K, x.data_ptr(), stride, wc, wsc, _optional(bias, torch.float32, "bias", (N,), dev),
            out.data_ptr(), ostride)
    try:                                        # most calls need no workspace: ask only where one does
        _launch(fn, dev, *args, None, 0)
    except MolgridError as e:
        if e.code != MG_EWORKSPACE:
            raise
        ws, size = _workspace_of(lib().mg_mx4_linear_workspace, x, M, N, K)
        _launch(fn, dev, *args, ws.data_ptr(), size)
    return out
