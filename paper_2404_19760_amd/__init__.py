"""Python binding of the MI355X Lightplane Renderer library (`liblightplane.so`).

Argument marshalling only: every step of the Renderer runs in the library's HIP
kernels.  PyTorch supplies device memory (tensors) and streams.  The functions carry
the names of the C entry points declared in `include/lightplane.h`.

There is no CPU fallback: importing this package without a built library, or calling
it without a GPU tensor, raises.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
import struct
from typing import List, Optional, Sequence

import numpy as np
import torch
from torch.autograd.graph import increment_version

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("LP_LIB_PATH", os.path.join(_HERE, "liblightplane.so"))

LP_MAX_LAYERS = 8
LP_OK, LP_ERR_INVALID_ARG, LP_ERR_UNSUPPORTED, LP_ERR_HIP, LP_ERR_WORKSPACE = range(5)
LP_GRID_VOXEL, LP_GRID_TRIPLANE, LP_GRID_HASH, LP_GRID_HEXPLANE = 0, 1, 2, 3
LP_MATH_DEFAULT, LP_MATH_GENERIC, LP_MATH_BF16X3 = 0, 1, 2
LP_FEAT_SIGMOID, LP_FEAT_IDENTITY = 0, 1
LP_F32, LP_BF16, LP_F16 = 0, 1, 2
LP_ACT_NONE, LP_ACT_RELU, LP_ACT_SILU, LP_ACT_GELU = 0, 1, 2, 3
LP_NORM_RMS, LP_NORM_LAYER = 0, 1
LP_RESIDUAL_NORM_MAX_CHANNELS = 8192
LP_ORTH_MAX_STEPS = 16
LP_MUON_SCALE_NONE, LP_MUON_SCALE_ASPECT, LP_MUON_SCALE_RMS = 0, 1, 2


class LightplaneError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"lightplane status {status}: {message}")
        self.status = status


class _Grid(C.Structure):
    _fields_ = [("kind", C.c_int32), ("B", C.c_int32), ("C", C.c_int32),
                ("NX", C.c_int32), ("NY", C.c_int32), ("NZ", C.c_int32),
                ("data", C.c_void_p * 3),
                ("aabb_min", C.c_float * 3), ("aabb_max", C.c_float * 3), ("contract_a", C.c_float),
                ("dtype", C.c_int32), ("hash_size", C.c_int64),
                ("data_t", C.c_void_p * 3), ("NT", C.c_int32), ("t_min", C.c_float), ("t_max", C.c_float)]


class _Mlp(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("dims", C.c_int32 * (LP_MAX_LAYERS + 1)),
                ("W", C.c_void_p * LP_MAX_LAYERS), ("b", C.c_void_p * LP_MAX_LAYERS)]


class _Decoder(C.Structure):
    _fields_ = [("opacity", _Mlp), ("feature", _Mlp), ("n_freq", C.c_int32), ("n_feat", C.c_int32),
                ("feat_act", C.c_int32)]


class _Splat(C.Structure):
    _fields_ = [("n_in", C.c_int32), ("n_freq", C.c_int32), ("feats", C.c_void_p),
                ("prior", C.POINTER(_Grid)), ("mlp", C.POINTER(_Mlp))]


class _Rays(C.Structure):
    _fields_ = [("M", C.c_int64), ("S", C.c_int32),
                ("origins", C.c_void_p), ("dirs", C.c_void_p),
                ("near", C.c_void_p), ("far", C.c_void_p), ("scene", C.c_void_p), ("time", C.c_void_p)]


class _GroupNorm(C.Structure):
    _fields_ = [("N", C.c_int64), ("P", C.c_int64), ("C", C.c_int32), ("G", C.c_int32), ("act", C.c_int32), ("eps", C.c_float),
                ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("x_stride", C.c_int64), ("y_stride", C.c_int64),
                ("gamma", C.c_void_p), ("beta", C.c_void_p), ("occupancy", C.c_void_p)]


class _Linear(C.Structure):
    _fields_ = [("P", C.c_int64), ("K", C.c_int32), ("N", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32), ("x_stride", C.c_int64),
                ("y_stride", C.c_int64), ("r_stride", C.c_int64), ("weight", C.c_void_p), ("bias", C.c_void_p), ("residual", C.c_void_p)]


class _ResidualNorm(C.Structure):
    _fields_ = [("N", C.c_int64), ("P", C.c_int64), ("C", C.c_int32), ("kind", C.c_int32), ("post_norm", C.c_int32),
                ("gate_per_sample", C.c_int32), ("alpha", C.c_float), ("eps", C.c_float), ("h_dtype", C.c_int32), ("f_dtype", C.c_int32),
                ("h_stride", C.c_int64), ("f_stride", C.c_int64), ("y_stride", C.c_int64), ("post_gamma", C.c_void_p),
                ("gate", C.c_void_p), ("gamma", C.c_void_p), ("beta", C.c_void_p)]


class _Gradient(C.Structure):
    _fields_ = [("size", C.c_int64), ("input", C.c_void_p), ("out", C.c_void_p), ("dtype", C.c_int32)]


class _Orth(C.Structure):
    _fields_ = [("steps", C.c_int32), ("coeffs", C.POINTER(C.c_float)), ("eps", C.c_float)]


class _Matrices(C.Structure):
    _fields_ = [("count", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("input", C.c_void_p), ("out", C.c_void_p),
                ("dtype", C.c_int32)]


class _Muon(C.Structure):
    _fields_ = [("lr", C.c_float), ("momentum", C.c_float), ("weight_decay", C.c_float), ("nesterov", C.c_int32),
                ("scale", C.c_int32), ("orth", _Orth)]


class _MuonWeights(C.Structure):
    _fields_ = [("count", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("weight", C.c_void_p), ("grad", C.c_void_p),
                ("momentum", C.c_void_p)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python paper_2404_19760_amd/build.py` "
                          "(there is no fallback implementation)")
    lib = C.CDLL(LIB_PATH)
    lib.lp_last_error.restype = C.c_char_p
    lib.lp_version.restype = C.c_int32
    lib.lp_diag_coexecution.restype = C.c_int
    lib.lp_diag_coexecution.argtypes = [C.POINTER(C.c_float), C.c_void_p]
    lib.lp_diag_atomic_rate.restype = C.c_int
    lib.lp_diag_atomic_rate.argtypes = [C.POINTER(C.c_float), C.c_void_p]
    lib.lp_diag_ws_phases.restype = C.c_int
    lib.lp_diag_ws_phases.argtypes = [C.POINTER(C.c_ulonglong)]
    lib.lp_has_fast_path.restype = C.c_int32
    lib.lp_has_fast_path.argtypes = [C.POINTER(_Grid), C.POINTER(_Mlp)]
    lib.lp_render_fwd.restype = C.c_int
    lib.lp_render_fwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Mlp), C.POINTER(_Rays),
                                  C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_int32, C.c_void_p]
    lib.lp_render_bwd.restype = C.c_int
    lib.lp_render_bwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Mlp), C.POINTER(_Rays),
                                  C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                  C.POINTER(C.c_void_p), C.c_void_p, C.c_size_t, C.c_int32,
                                  C.c_void_p]
    lib.lp_render_bwd_static.restype = C.c_int
    lib.lp_render_bwd_static.argtypes = [C.POINTER(_Grid), C.POINTER(_Mlp), C.POINTER(_Rays),
                                         C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                         C.POINTER(C.c_void_p), C.c_int32, C.c_void_p]
    lib.lp_bwd_workspace_bytes.restype = C.c_int
    lib.lp_bwd_workspace_bytes.argtypes = [C.POINTER(_Grid), C.POINTER(_Mlp), C.POINTER(_Rays),
                                           C.c_int32, C.POINTER(C.c_size_t)]
    lib.lp_dec_has_fast_path.restype = C.c_int32
    lib.lp_dec_has_fast_path.argtypes = [C.POINTER(_Grid), C.POINTER(_Decoder)]
    lib.lp_dec_workspace_bytes.restype = C.c_int
    lib.lp_dec_workspace_bytes.argtypes = [C.POINTER(_Grid), C.POINTER(_Decoder), C.POINTER(_Rays), C.c_int32,
                                           C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.lp_render_dec_fwd.restype = C.c_int
    lib.lp_render_dec_fwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Decoder), C.POINTER(_Rays),
                                      C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p]
    lib.lp_render_dec_bwd.restype = C.c_int
    lib.lp_render_dec_bwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Decoder), C.POINTER(_Rays),
                                      C.POINTER(C.c_float), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                      C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_void_p, C.c_size_t,
                                      C.c_int32, C.c_void_p]
    lib.lp_splat_fwd.restype = C.c_int
    lib.lp_splat_fwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Rays), C.POINTER(_Splat), C.POINTER(C.c_void_p),
                                 C.POINTER(C.c_void_p), C.c_void_p]
    lib.lp_splat_has_fast_path.restype = C.c_int32
    lib.lp_splat_has_fast_path.argtypes = [C.POINTER(_Grid), C.POINTER(_Splat)]
    lib.lp_splat_bwd_workspace_bytes.restype = C.c_int
    lib.lp_splat_bwd_workspace_bytes.argtypes = [C.POINTER(_Grid), C.POINTER(_Rays), C.POINTER(_Splat),
                                                 C.POINTER(C.c_size_t)]
    lib.lp_splat_bwd.restype = C.c_int
    lib.lp_splat_bwd.argtypes = [C.POINTER(_Grid), C.POINTER(_Rays), C.POINTER(_Splat), C.POINTER(C.c_void_p),
                                 C.POINTER(C.c_void_p), C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                 C.POINTER(C.c_void_p), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_group_norm_workspace_bytes.restype = C.c_int
    lib.lp_group_norm_workspace_bytes.argtypes = [C.POINTER(_GroupNorm), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.lp_group_norm_fwd.restype = C.c_int
    lib.lp_group_norm_fwd.argtypes = [C.POINTER(_GroupNorm), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_group_norm_bwd.restype = C.c_int
    lib.lp_group_norm_bwd.argtypes = [C.POINTER(_GroupNorm), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_linear_workspace_bytes.restype = C.c_int
    lib.lp_linear_workspace_bytes.argtypes = [C.POINTER(_Linear), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.lp_linear_fwd.restype = C.c_int
    lib.lp_linear_fwd.argtypes = [C.POINTER(_Linear), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_linear_bwd.restype = C.c_int
    lib.lp_linear_bwd.argtypes = [C.POINTER(_Linear), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_residual_norm_workspace_bytes.restype = C.c_int
    lib.lp_residual_norm_workspace_bytes.argtypes = [C.POINTER(_ResidualNorm), C.POINTER(C.c_size_t)]
    lib.lp_residual_norm_fwd.restype = C.c_int
    lib.lp_residual_norm_fwd.argtypes = [C.POINTER(_ResidualNorm), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.lp_residual_norm_bwd.restype = C.c_int
    lib.lp_residual_norm_bwd.argtypes = [C.POINTER(_ResidualNorm), *[C.c_void_p] * 11, C.c_size_t, C.c_void_p]
    lib.lp_grad_norm_workspace_bytes.restype = C.c_int
    lib.lp_grad_norm_workspace_bytes.argtypes = [C.c_int32, C.POINTER(_Gradient), C.POINTER(C.c_size_t)]
    lib.lp_grad_norm.restype = C.c_int
    lib.lp_grad_norm.argtypes = [C.c_int32, C.POINTER(_Gradient), C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_clip_grad_norm.restype = C.c_int
    lib.lp_clip_grad_norm.argtypes = [C.c_int32, C.POINTER(_Gradient), C.c_float, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_orthogonalize_workspace_bytes.restype = C.c_int
    lib.lp_orthogonalize_workspace_bytes.argtypes = [C.c_int32, C.POINTER(_Matrices), C.POINTER(C.c_size_t)]
    lib.lp_orthogonalize.restype = C.c_int
    lib.lp_orthogonalize.argtypes = [C.c_int32, C.POINTER(_Matrices), C.POINTER(_Orth), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lp_muon_workspace_bytes.restype = C.c_int
    lib.lp_muon_workspace_bytes.argtypes = [C.c_int32, C.POINTER(_MuonWeights), C.POINTER(C.c_size_t)]
    lib.lp_muon_step.restype = C.c_int
    lib.lp_muon_step.argtypes = [C.c_int32, C.POINTER(_MuonWeights), C.POINTER(_Muon), C.c_void_p, C.c_size_t, C.c_void_p]
    return lib


_lib = _load()


def _check(status: int):
    if status != LP_OK:
        raise LightplaneError(status, _lib.lp_last_error().decode())


def _dev_f32(t: Optional[torch.Tensor], name: str, shape=None, index=None) -> Optional[int]:
    if t is None:
        return None
    # (one test in the common case, and the name put together only for an error: a call marshals some twenty tensors, and
    # small launches wait for that)
    if t.is_cuda and t.dtype is torch.float32 and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    if index is not None:
        name = f"{name}[{index}]"
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous float32 tensor on the GPU")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


_GRID_DTYPES = {torch.float32: LP_F32, torch.bfloat16: LP_BF16, torch.float16: LP_F16}


@dataclasses.dataclass
class Grid:
    """Voxel grid [B][NX][NY][NZ][C] (one tensor), triplane (three tensors [B][NX][NY][C],
    [B][NY][NZ][C], [B][NZ][NX][C]) or hash table [B][T][C] (one tensor; res = the virtual lattice
    whose corners are hashed into it) or HexPlane (six tensors: the triplane's three, then the
    space-time planes [B][NZ][NT][C], [B][NX][NT][C], [B][NY][NT][C]; t_range = the times of the first
    and last index of the time axis); float32, bfloat16 or float16 (all tensors alike), on the GPU."""
    kind: int
    data: List[torch.Tensor]
    res: Sequence[int]
    aabb_min: Sequence[float] = (-1.0, -1.0, -1.0)
    aabb_max: Sequence[float] = (1.0, 1.0, 1.0)
    contract_a: float = 0.0
    t_range: Sequence[float] = (0.0, 1.0)

    @property
    def n_scenes(self) -> int:
        return int(self.data[0].shape[0])

    @property
    def channels(self) -> int:
        return int(self.data[0].shape[-1])

    def shapes(self):
        first = self.data[0].shape
        b, c = first[0], first[-1]
        nx, ny, nz = self.res
        if self.kind == LP_GRID_VOXEL:
            return [(b, nx, ny, nz, c)]
        if self.kind == LP_GRID_HASH:
            return [(b, first[1], c)]
        planes = [(b, nx, ny, c), (b, ny, nz, c), (b, nz, nx, c)]
        if self.kind == LP_GRID_HEXPLANE:
            if len(self.data) != 6:
                raise ValueError("a HexPlane has six tensors")
            nt = int(self.data[3].shape[2])
            planes += [(b, nz, nt, c), (b, nx, nt, c), (b, ny, nt, c)]
        return planes

    def c_struct(self, shapes=None) -> _Grid:
        """`shapes`: self.shapes(), if the caller has it."""
        data = self.data
        if shapes is None:
            shapes = self.shapes()
        nx, ny, nz = self.res
        if len(data) != len(shapes):
            raise ValueError("wrong number of grid tensors for this kind")
        dt = data[0].dtype
        if dt not in _GRID_DTYPES:
            raise ValueError("grid tensors must be float32, bfloat16 or float16")
        ptr = [None] * 6
        for p, (t, s) in enumerate(zip(data, shapes)):
            if not (t.is_cuda and t.dtype is dt and t.is_contiguous() and t.shape == s):
                raise ValueError(f"grid.data[{p}] must be a contiguous GPU tensor of shape {tuple(s)} and the "
                                 "dtype of grid.data[0]")
            ptr[p] = t.data_ptr()
        lo, hi = self.aabb_min, self.aabb_max
        hexplane = self.kind == LP_GRID_HEXPLANE
        return _Grid(self.kind, shapes[0][0], shapes[0][-1], int(nx), int(ny), int(nz), tuple(ptr[:3]),
                     (float(lo[0]), float(lo[1]), float(lo[2])), (float(hi[0]), float(hi[1]), float(hi[2])),
                     float(self.contract_a), _GRID_DTYPES[dt], shapes[0][1] if self.kind == LP_GRID_HASH else 0, tuple(ptr[3:]),
                     shapes[3][2] if hexplane else 0, float(self.t_range[0]) if hexplane else 0.0,
                     float(self.t_range[1]) if hexplane else 0.0)


@dataclasses.dataclass
class Mlp:
    """weights[l] = [out][in], biases[l] = [out]; float32, on the GPU."""
    weights: List[torch.Tensor]
    biases: List[torch.Tensor]

    @property
    def dims(self):
        return [self.weights[0].shape[1], *[w.shape[0] for w in self.weights]]

    def c_struct(self) -> _Mlp:
        weights, biases = self.weights, self.biases
        if len(weights) != len(biases) or not 1 <= len(weights) <= LP_MAX_LAYERS:
            raise ValueError("MLP needs 1..8 layers with one bias per weight matrix")
        dims = self.dims
        return _Mlp(len(weights), tuple(dims),
                    tuple([_dev_f32(w, "weights", (dims[l + 1], dims[l]), l) for l, w in enumerate(weights)]),
                    tuple([_dev_f32(b, "biases", (dims[l + 1],), l) for l, b in enumerate(biases)]))


@dataclasses.dataclass
class Decoder:
    """The two-MLP decoder: opacity MLP (C -> ... -> 1) and feature MLP
    (C + 3 + 6 n_freq -> ... -> n_feat); feat_act LP_FEAT_SIGMOID or LP_FEAT_IDENTITY."""
    opacity: Mlp
    feature: Mlp
    n_freq: int
    n_feat: int
    feat_act: int = 0

    def c_struct(self) -> _Decoder:
        d = _Decoder()
        d.opacity, d.feature = self.opacity.c_struct(), self.feature.c_struct()
        d.n_freq, d.n_feat, d.feat_act = int(self.n_freq), int(self.n_feat), int(self.feat_act)
        return d


@dataclasses.dataclass
class Rays:
    origins: torch.Tensor          # [M][3]
    dirs: torch.Tensor             # [M][3] unit
    near: torch.Tensor             # [M]
    far: torch.Tensor              # [M]
    samples: int                   # S
    scene: Optional[torch.Tensor] = None  # [M] int32
    time: Optional[torch.Tensor] = None   # [M] float32, the time of every ray (read by a HexPlane only)

    @property
    def n_rays(self) -> int:
        return self.origins.shape[0]

    def c_struct(self) -> _Rays:
        m = self.n_rays
        scene = self.scene
        if scene is not None:
            if not (scene.is_cuda and scene.dtype is torch.int32 and scene.is_contiguous() and scene.shape == (m,)):
                raise ValueError("scene must be a contiguous int32 GPU tensor of shape [M]")
            scene = scene.data_ptr()
        return _Rays(m, int(self.samples), _dev_f32(self.origins, "origins", (m, 3)), _dev_f32(self.dirs, "dirs", (m, 3)),
                     _dev_f32(self.near, "near", (m,)), _dev_f32(self.far, "far", (m,)), scene,
                     _dev_f32(self.time, "time", (m,)))


# the current stream's handle without a Stream object around it, where torch has it (a private name: else the public one)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return C.c_void_p(_raw_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


_Float3, _Pointers6, _PointersL = C.c_float * 3, C.c_void_p * 6, C.c_void_p * LP_MAX_LAYERS


def _bg(bg) -> C.Array:
    return _Float3(*[float(v) for v in bg])


def lp_version() -> int:
    return int(_lib.lp_version())


def lp_diag_coexecution(stream=None):
    """Nanoseconds per loop iteration of the ten measurements the header describes."""
    out = (C.c_float * 10)()
    _check(_lib.lp_diag_coexecution(out, _stream_ptr(stream)))
    return [float(v) for v in out]


def lp_diag_atomic_rate(stream=None):
    """64-byte lines of fp32 atomic adds per second in the six settings the header describes."""
    out = (C.c_float * 6)()
    _check(_lib.lp_diag_atomic_rate(out, _stream_ptr(stream)))
    return [float(v) for v in out]


def lp_diag_ws_phases():
    """Cycle sums per phase of the two-wave backward (measurement builds only; see the header)."""
    out = (C.c_ulonglong * 32)()
    _check(_lib.lp_diag_ws_phases(out))
    return [int(v) for v in out]


def lp_has_fast_path(grid: Grid, mlp: Mlp) -> bool:
    g, m = grid.c_struct(), mlp.c_struct()
    return bool(_lib.lp_has_fast_path(C.byref(g), C.byref(m)))


def lp_render_fwd(grid: Grid, mlp: Mlp, rays: Rays, bg, rgb: torch.Tensor,
                  alpha: Optional[torch.Tensor], depth: Optional[torch.Tensor],
                  ray_cache: Optional[torch.Tensor], math_mode: int = LP_MATH_DEFAULT,
                  stream=None) -> None:
    """Enqueue the forward on `stream` (default: torch's current stream); outputs are
    caller-allocated GPU tensors rgb [M][3], alpha [M], depth [M], ray_cache [M]."""
    m = rays.n_rays
    g, ml, r = grid.c_struct(), mlp.c_struct(), rays.c_struct()
    _check(_lib.lp_render_fwd(C.byref(g), C.byref(ml), C.byref(r), _bg(bg),
                              _dev_f32(rgb, "rgb", (m, 3)), _dev_f32(alpha, "alpha", (m,)),
                              _dev_f32(depth, "depth", (m,)), _dev_f32(ray_cache, "ray_cache", (m,)),
                              int(math_mode), _stream_ptr(stream)))


def lp_bwd_workspace_bytes(grid: Grid, mlp: Mlp, rays: Rays, math_mode: int = LP_MATH_DEFAULT) -> int:
    g, ml, r = grid.c_struct(), mlp.c_struct(), rays.c_struct()
    n = C.c_size_t(0)
    _check(_lib.lp_bwd_workspace_bytes(C.byref(g), C.byref(ml), C.byref(r), int(math_mode), C.byref(n)))
    return int(n.value)


LP_STATIC_SCRATCH_BYTES = 32 * 1024 * 1024


def lp_render_bwd_static(grid: Grid, mlp: Mlp, rays: Rays, bg, d_rgb: torch.Tensor,
                         d_alpha: Optional[torch.Tensor], d_depth: Optional[torch.Tensor],
                         ray_cache: torch.Tensor, d_grid: List[torch.Tensor], dW: List[torch.Tensor],
                         db: List[torch.Tensor], math_mode: int = LP_MATH_DEFAULT, stream=None) -> None:
    """lp_render_bwd without a workspace: the library's static device scratch holds the records
    (nothing is allocated; shapes that need more than LP_STATIC_SCRATCH_BYTES are refused)."""
    _render_bwd(grid, mlp, rays, bg, d_rgb, d_alpha, d_depth, ray_cache, d_grid, dW, db, None, math_mode, stream)


def lp_render_bwd(grid: Grid, mlp: Mlp, rays: Rays, bg, d_rgb: torch.Tensor,
                  d_alpha: Optional[torch.Tensor], d_depth: Optional[torch.Tensor],
                  ray_cache: torch.Tensor, d_grid: List[torch.Tensor], dW: List[torch.Tensor],
                  db: List[torch.Tensor], workspace: torch.Tensor,
                  math_mode: int = LP_MATH_DEFAULT, stream=None) -> None:
    """Enqueue the backward; d_grid / dW / db are ACCUMULATED into (same shapes as the
    grid tensors, weights and biases); `workspace` is a GPU byte tensor of at least
    lp_bwd_workspace_bytes(...) bytes."""
    if workspace is None:
        raise ValueError("workspace must be a contiguous GPU tensor")
    _render_bwd(grid, mlp, rays, bg, d_rgb, d_alpha, d_depth, ray_cache, d_grid, dW, db, workspace, math_mode, stream)


def _render_bwd(grid, mlp, rays, bg, d_rgb, d_alpha, d_depth, ray_cache, d_grid, dW, db, workspace, math_mode, stream):
    m = rays.n_rays
    shapes = grid.shapes()
    g, ml, r = grid.c_struct(shapes), mlp.c_struct(), rays.c_struct()
    dims = ml.dims   # (of an MLP that c_struct has found to be one)
    if len(d_grid) != len(shapes):
        raise ValueError("d_grid needs one tensor per grid tensor")
    dg = _Pointers6(*[_dev_f32(t, "d_grid", s, p) for p, (t, s) in enumerate(zip(d_grid, shapes))])
    if len(dW) != len(mlp.weights) or len(db) != len(mlp.weights):
        raise ValueError("dW / db need one tensor per layer")
    dWp = _PointersL(*[_dev_f32(w, "dW", (dims[l + 1], dims[l]), l) for l, w in enumerate(dW)])
    dbp = _PointersL(*[_dev_f32(b, "db", (dims[l + 1],), l) for l, b in enumerate(db)])
    common = (C.byref(g), C.byref(ml), C.byref(r), _bg(bg),
              _dev_f32(d_rgb, "d_rgb", (m, 3)), _dev_f32(d_alpha, "d_alpha", (m,)),
              _dev_f32(d_depth, "d_depth", (m,)), _dev_f32(ray_cache, "ray_cache", (m,)), dg, dWp, dbp)
    if workspace is None:
        _check(_lib.lp_render_bwd_static(*common, int(math_mode), _stream_ptr(stream)))
        return
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous GPU tensor")
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.lp_render_bwd(*common, C.c_void_p(workspace.data_ptr()), C.c_size_t(ws_bytes),
                              int(math_mode), _stream_ptr(stream)))


def lp_dec_has_fast_path(grid: Grid, dec: Decoder) -> bool:
    g, d = grid.c_struct(), dec.c_struct()
    return bool(_lib.lp_dec_has_fast_path(C.byref(g), C.byref(d)))


def lp_dec_workspace_bytes(grid: Grid, dec: Decoder, rays: Rays, math_mode: int = LP_MATH_DEFAULT):
    """(forward bytes, backward bytes) of workspace for the two-MLP decoder calls."""
    g, d, r = grid.c_struct(), dec.c_struct(), rays.c_struct()
    nf, nb = C.c_size_t(0), C.c_size_t(0)
    _check(_lib.lp_dec_workspace_bytes(C.byref(g), C.byref(d), C.byref(r), int(math_mode), C.byref(nf), C.byref(nb)))
    return int(nf.value), int(nb.value)


def _workspace(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, C.c_size_t(0)
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous GPU tensor")
    return C.c_void_p(workspace.data_ptr()), C.c_size_t(workspace.numel() * workspace.element_size())


def lp_render_dec_fwd(grid: Grid, dec: Decoder, rays: Rays, bg, out: torch.Tensor,
                      alpha: Optional[torch.Tensor], depth: Optional[torch.Tensor],
                      ray_cache: Optional[torch.Tensor], workspace: torch.Tensor,
                      math_mode: int = LP_MATH_DEFAULT, stream=None) -> None:
    """Forward with the two-MLP decoder; out [M][n_feat]; bg has n_feat entries."""
    m, f = rays.n_rays, int(dec.n_feat)
    g, d, r = grid.c_struct(), dec.c_struct(), rays.c_struct()
    wp, wn = _workspace(workspace)
    _check(_lib.lp_render_dec_fwd(C.byref(g), C.byref(d), C.byref(r), (C.c_float * f)(*[float(v) for v in bg]),
                                  _dev_f32(out, "out", (m, f)), _dev_f32(alpha, "alpha", (m,)),
                                  _dev_f32(depth, "depth", (m,)), _dev_f32(ray_cache, "ray_cache", (m,)),
                                  wp, wn, int(math_mode), _stream_ptr(stream)))


def lp_render_dec_bwd(grid: Grid, dec: Decoder, rays: Rays, bg, d_out: torch.Tensor,
                      d_alpha: Optional[torch.Tensor], d_depth: Optional[torch.Tensor],
                      ray_cache: torch.Tensor, d_grid: List[torch.Tensor],
                      dW_opacity: List[torch.Tensor], db_opacity: List[torch.Tensor],
                      dW_feature: List[torch.Tensor], db_feature: List[torch.Tensor],
                      workspace: torch.Tensor, math_mode: int = LP_MATH_DEFAULT, stream=None) -> None:
    """Backward with the two-MLP decoder; all gradient tensors are ACCUMULATED into."""
    m, f = rays.n_rays, int(dec.n_feat)
    g, d, r = grid.c_struct(), dec.c_struct(), rays.c_struct()
    shapes = grid.shapes()
    if len(d_grid) != len(shapes):
        raise ValueError("d_grid needs one tensor per grid tensor")
    dg = (C.c_void_p * 6)(*[_dev_f32(d_grid[p], f"d_grid[{p}]", shapes[p]) if p < len(shapes) else None
                            for p in range(6)])

    def lists(mlp, dW, db, name):
        dims = mlp.dims
        if len(dW) != len(mlp.weights) or len(db) != len(mlp.weights):
            raise ValueError(f"dW_{name} / db_{name} need one tensor per layer")
        return ((C.c_void_p * LP_MAX_LAYERS)(*[_dev_f32(w, f"dW_{name}[{l}]", (dims[l + 1], dims[l]))
                                               for l, w in enumerate(dW)]),
                (C.c_void_p * LP_MAX_LAYERS)(*[_dev_f32(b, f"db_{name}[{l}]", (dims[l + 1],))
                                               for l, b in enumerate(db)]))
    dWs, dbs = lists(dec.opacity, dW_opacity, db_opacity, "opacity")
    dWv, dbv = lists(dec.feature, dW_feature, db_feature, "feature")
    wp, wn = _workspace(workspace)
    _check(_lib.lp_render_dec_bwd(C.byref(g), C.byref(d), C.byref(r), (C.c_float * f)(*[float(v) for v in bg]),
                                  _dev_f32(d_out, "d_out", (m, f)), _dev_f32(d_alpha, "d_alpha", (m,)),
                                  _dev_f32(d_depth, "d_depth", (m,)), _dev_f32(ray_cache, "ray_cache", (m,)),
                                  dg, dWs, dbs, dWv, dbv, wp, wn, int(math_mode), _stream_ptr(stream)))


@dataclasses.dataclass
class Splat:
    """Arguments of the Splatter besides target and rays: pixel features [M][n_in], optional
    prior structure (a Grid of the target's kind) and MLP, octaves of the direction encoding."""
    feats: torch.Tensor
    prior: Optional[Grid] = None
    mlp: Optional[Mlp] = None
    n_freq: int = -1

    def c_struct(self):
        """Returns (struct, keep-alive objects)."""
        s = _Splat()
        m, n_in = int(self.feats.shape[0]), int(self.feats.shape[1])
        s.n_in, s.n_freq = n_in, int(self.n_freq)
        s.feats = _dev_f32(self.feats, "feats", (m, n_in))
        keep = []
        if self.prior is not None:
            g = self.prior.c_struct()
            keep.append(g)
            s.prior = C.pointer(g)
        if self.mlp is not None:
            ml = self.mlp.c_struct()
            keep.append(ml)
            s.mlp = C.pointer(ml)
        return s, keep


def target_struct(kind: int, n_scenes: int, channels: int, res, aabb_min=(-1.0, -1.0, -1.0),
                  aabb_max=(1.0, 1.0, 1.0), contract_a: float = 0.0, hash_size: int = 0) -> _Grid:
    """lp_grid describing the structure a Splatter call builds (no data pointers; hash_size: the
    entries per scene of a hash-table target)."""
    g = _Grid()
    g.hash_size = int(hash_size) if int(kind) == LP_GRID_HASH else 0
    g.kind, g.B, g.C = int(kind), int(n_scenes), int(channels)
    g.NX, g.NY, g.NZ = [int(v) for v in res]
    for a in range(3):
        g.aabb_min[a] = float(aabb_min[a])
        g.aabb_max[a] = float(aabb_max[a])
    g.contract_a = float(contract_a)
    return g


def _target_shapes(t: _Grid, channels: Optional[int]):
    b, nx, ny, nz = t.B, t.NX, t.NY, t.NZ
    c = () if channels is None else (channels,)
    if t.kind == LP_GRID_VOXEL:
        return [(b, nx, ny, nz) + c]
    if t.kind == LP_GRID_HASH:
        return [(b, int(t.hash_size)) + c]
    return [(b, nx, ny) + c, (b, ny, nz) + c, (b, nz, nx) + c]


def _ptr3(tensors, shapes, name):
    if len(tensors) != len(shapes):
        raise ValueError(f"{name} needs {len(shapes)} tensors")
    return (C.c_void_p * 3)(*[_dev_f32(tensors[p], f"{name}[{p}]", shapes[p]) if p < len(shapes) else None
                              for p in range(3)])


def lp_splat_fwd(target: _Grid, rays: Rays, splat: Splat, theta: List[torch.Tensor],
                 theta_w: List[torch.Tensor], stream=None) -> None:
    """Enqueue the Splatter forward: theta (shapes of the target's tensors) and theta_w (same
    without the channel axis) are written."""
    r = rays.c_struct()
    s, keep = splat.c_struct()
    _check(_lib.lp_splat_fwd(C.byref(target), C.byref(r), C.byref(s),
                             _ptr3(theta, _target_shapes(target, target.C), "theta"),
                             _ptr3(theta_w, _target_shapes(target, None), "theta_w"), _stream_ptr(stream)))
    del keep


def lp_splat_has_fast_path(target: _Grid, splat: Splat) -> bool:
    s, keep = splat.c_struct()
    fast = bool(_lib.lp_splat_has_fast_path(C.byref(target), C.byref(s)))
    del keep
    return fast


def lp_splat_bwd_workspace_bytes(target: _Grid, rays: Rays, splat: Splat) -> int:
    r = rays.c_struct()
    s, keep = splat.c_struct()
    n = C.c_size_t(0)
    _check(_lib.lp_splat_bwd_workspace_bytes(C.byref(target), C.byref(r), C.byref(s), C.byref(n)))
    del keep
    return int(n.value)


def lp_splat_bwd(target: _Grid, rays: Rays, splat: Splat, theta_w: List[torch.Tensor],
                 d_theta: List[torch.Tensor], d_feats: torch.Tensor, d_prior: Optional[List[torch.Tensor]],
                 dW: Optional[List[torch.Tensor]], db: Optional[List[torch.Tensor]], workspace: torch.Tensor,
                 stream=None) -> None:
    """Enqueue the Splatter backward: d_feats is written; d_prior, dW, db are accumulated into."""
    r = rays.c_struct()
    s, keep = splat.c_struct()
    m, n_in = int(splat.feats.shape[0]), int(splat.feats.shape[1])
    dp = (C.c_void_p * 3)()
    if splat.prior is not None:
        dp = _ptr3(d_prior, splat.prior.shapes(), "d_prior")
    dWp, dbp = (C.c_void_p * LP_MAX_LAYERS)(), (C.c_void_p * LP_MAX_LAYERS)()
    if splat.mlp is not None:
        dims = splat.mlp.dims
        dWp = (C.c_void_p * LP_MAX_LAYERS)(*[_dev_f32(w, "dW", (dims[l + 1], dims[l]), l) for l, w in enumerate(dW)])
        dbp = (C.c_void_p * LP_MAX_LAYERS)(*[_dev_f32(b, "db", (dims[l + 1],), l) for l, b in enumerate(db)])
    wp, wn = _workspace(workspace)
    _check(_lib.lp_splat_bwd(C.byref(target), C.byref(r), C.byref(s),
                             _ptr3(theta_w, _target_shapes(target, None), "theta_w"),
                             _ptr3(d_theta, _target_shapes(target, target.C), "d_theta"),
                             _dev_f32(d_feats, "d_feats", (m, n_in)), dp, dWp, dbp, wp, wn, _stream_ptr(stream)))
    del keep


def _written(*tensors: Optional[torch.Tensor]) -> None:
    """Moves the versions of tensors that a call wrote through their addresses: a graph that has saved one of them notices.
    (None: not wanted.)"""
    increment_version([t for t in tensors if t is not None])


def _int32(value, name: str) -> int:
    value = int(value)
    if not -1 << 31 <= value < 1 << 31:   # (ctypes would cut it off)
        raise ValueError(f"{name} does not fit 32 bits")
    return value


@dataclasses.dataclass
class GroupNorm:
    """Group norm with an activation over channel-last tensors [N][...][C] (a voxel grid [B][NX][NY][NZ][C], a plane
    [B][NX][NY][C], ...): everything between the first and the last axis is normalised together with the channels of a
    group.  gamma, beta: float32 [C] or None; occupancy: float32 [N][...] or None, positions whose value is not above zero
    do not take part (the weight sums `theta_w` of a Splatter)."""
    groups: int
    gamma: Optional[torch.Tensor] = None
    beta: Optional[torch.Tensor] = None
    act: int = LP_ACT_NONE
    eps: float = 1e-5
    occupancy: Optional[torch.Tensor] = None

    def c_struct(self, x: torch.Tensor, y_dtype=None, y_stride: int = 0) -> _GroupNorm:
        y_dtype = x.dtype if y_dtype is None else y_dtype
        if x.dtype not in _GRID_DTYPES or y_dtype not in _GRID_DTYPES:
            raise ValueError("x and y must be float32, bfloat16 or float16")
        shape = x.shape
        if len(shape) < 2:
            raise ValueError("x must have a first axis of samples and a last axis of channels")
        n, c = shape[0], shape[-1]
        return _GroupNorm(n, x.numel() // (n * c) if n and c else 0, _int32(c, "the number of channels"), _int32(self.groups, "groups"),
                          _int32(self.act, "act"), float(self.eps),
                          _GRID_DTYPES[x.dtype], _GRID_DTYPES[y_dtype], _position_stride(x, "x"), y_stride,
                          _dev_f32(self.gamma, "gamma", (c,)), _dev_f32(self.beta, "beta", (c,)),
                          _dev_f32(self.occupancy, "occupancy", shape[:-1]))


def _position_stride(t: torch.Tensor, name: str) -> int:
    """Elements from position to position of a channel-last tensor: dense, or a slice of the channels of a dense one."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    c = t.shape[-1]
    if t.is_contiguous() or t.numel() == 0:
        return c
    strides, shape = t.stride(), t.shape
    step, want = None, None
    for k in range(t.dim() - 2, -1, -1):
        if shape[k] == 1:
            continue
        if step is None:
            step, want = strides[k], strides[k]
        if strides[k] != want:
            step = 0
            break
        want *= shape[k]
    if not step or step < c or (c > 1 and strides[-1] != 1):
        raise ValueError(f"{name} must be channel-last: dense, or a slice of the channels of a dense tensor")
    return step


def _channel_last(t: torch.Tensor, name: str, shape, dtype):
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must have shape {tuple(shape)} and type {dtype}")
    return _position_stride(t, name)


def _no_overlap(written: torch.Tensor, written_step: int, read: torch.Tensor, read_step: int, written_name: str, read_name: str) -> None:
    """A tensor that is written is the one that is read or shares no value with it (channels of a wider tensor may lie between
    another one's).  The steps are those from position to position."""
    if written.numel() == 0:
        return
    a, b, c, count = written.data_ptr(), read.data_ptr(), written.shape[-1], written.numel() // written.shape[-1]
    if a == b and written_step == read_step and written.dtype == read.dtype:
        return
    a_size, b_size = written.element_size(), read.element_size()
    a_step, b_step, a_width, b_width = written_step * a_size, read_step * b_size, c * a_size, c * b_size
    if a + (count - 1) * a_step + a_width <= b or b + (count - 1) * b_step + b_width <= a:
        return
    if a_step == b_step:   # position j of `read` starts `behind` bytes behind position j + rows of `written`
        rows, behind = divmod(b - a, a_step)
        if not (behind < a_width and abs(rows) < count) and not (behind + b_width > a_step and abs(rows + 1) < count):
            return
    raise ValueError(f"{written_name} must be {read_name} itself or not overlap it")


def _norm_bytes(q: _GroupNorm):
    f, b = C.c_size_t(), C.c_size_t()
    _check(_lib.lp_group_norm_workspace_bytes(C.byref(q), C.byref(f), C.byref(b)))
    return f.value, b.value


def lp_group_norm_workspace_bytes(norm: GroupNorm, x: torch.Tensor, y_dtype=None):
    """(forward bytes, backward bytes) of workspace."""
    return _norm_bytes(norm.c_struct(x, y_dtype))


def lp_group_norm_fwd(norm: GroupNorm, x: torch.Tensor, y: torch.Tensor, stats: Optional[torch.Tensor],
                      workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue the forward: y (shape of x; its type, or a 16-bit one where x is float32) and stats [N][groups][2] (None:
    not wanted) are written."""
    q = norm.c_struct(x, y.dtype, _channel_last(y, "y", x.shape, y.dtype))
    _no_overlap(y, q.y_stride, x, q.x_stride, "y", "x")
    wp, wn = _workspace(workspace)
    _check(_lib.lp_group_norm_fwd(C.byref(q), x.data_ptr(), y.data_ptr(), _dev_f32(stats, "stats", (x.shape[0], norm.groups, 2)),
                                  wp, wn, _stream_ptr(stream)))
    _written(y, stats)


def lp_group_norm_bwd(norm: GroupNorm, x: torch.Tensor, stats: torch.Tensor, d_y: torch.Tensor, d_x: Optional[torch.Tensor],
                      d_gamma: Optional[torch.Tensor], d_beta: Optional[torch.Tensor], workspace: Optional[torch.Tensor],
                      stream=None) -> None:
    """Enqueue the backward: d_x (shape, type and strides of x) is written, d_gamma and d_beta [C] are accumulated into; each
    may be None.  stats as the forward wrote it for the same x."""
    q = norm.c_struct(x, d_y.dtype, _channel_last(d_y, "d_y", x.shape, d_y.dtype))
    if d_x is not None:
        if _channel_last(d_x, "d_x", x.shape, x.dtype) != q.x_stride:
            raise ValueError("d_x must have the strides of x")
        _no_overlap(d_x, q.x_stride, x, q.x_stride, "d_x", "x")
        _no_overlap(d_x, q.x_stride, d_y, q.y_stride, "d_x", "d_y")
    c = (x.shape[-1],)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_group_norm_bwd(C.byref(q), x.data_ptr(), _dev_f32(stats, "stats", (x.shape[0], norm.groups, 2)), d_y.data_ptr(),
                                  None if d_x is None else d_x.data_ptr(), _dev_f32(d_gamma, "d_gamma", c),
                                  _dev_f32(d_beta, "d_beta", c), wp, wn, _stream_ptr(stream)))
    _written(d_x, d_gamma, d_beta)


# (what torch.cuda.current_device() asks for behind its own initialisation, which a tensor on the GPU has been through)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on_current_device(first: torch.Tensor, *others: Optional[torch.Tensor]) -> torch.device:
    """Kernels run on the current device: the tensors of a call (None: not there) lie on it, all of them."""
    device = first.device
    for t in others:
        if t is not None and t.device != device:
            raise ValueError("the tensors of a call must be on one device")
    if device.type == "cuda" and device.index != _current_device():
        raise ValueError("the tensors of a call must be on the current device")
    return device


def _apart(written: torch.Tensor, written_step: int, read: Optional[torch.Tensor], read_step: int, written_name: str, read_name: str) -> None:
    """A tensor that is written shares no value with another one, be it the same."""
    if read is None or written.numel() == 0 or read.numel() == 0:
        return
    if written.data_ptr() == read.data_ptr():
        raise ValueError(f"{written_name} must not overlap {read_name}")
    if written.shape[-1] == read.shape[-1] and written.numel() == read.numel():
        _no_overlap(written, written_step, read, read_step, written_name, read_name)
        return
    ends = []
    for t, step in ((written, written_step), (read, read_step)):
        c = t.shape[-1]
        ends.append((t.data_ptr(), t.data_ptr() + ((t.numel() // c - 1) * step + c) * t.element_size(), step * t.element_size(), c * t.element_size()))
    (a, a_end, a_step, a_width), (b, b_end, b_step, b_width) = ends
    if a_end <= b or b_end <= a:
        return
    if a_step == b_step:   # channels of one wider tensor: the same columns never meet
        behind = (b - a) % a_step
        if behind >= a_width and behind + b_width <= a_step:
            return
    raise ValueError(f"{written_name} must not overlap {read_name}")


@dataclasses.dataclass
class Linear:
    """A product of positions' channels with a weight matrix [N][K] (contiguous, of the type of what it is applied to), a bias
    (float32 [N] or None) and an activation: act(x W^T + b) + residual for x [...][K]."""
    weight: torch.Tensor
    bias: Optional[torch.Tensor] = None
    act: int = LP_ACT_NONE

    def c_struct(self, x: torch.Tensor, y_stride: int = 0, residual: Optional[torch.Tensor] = None) -> _Linear:
        w, dtype = self.weight, x.dtype
        if dtype not in _GRID_DTYPES:
            raise ValueError("x must be float32, bfloat16 or float16")
        if not (w.is_cuda and w.dim() == 2 and w.is_contiguous() and w.dtype is dtype):
            raise ValueError(f"weight must be a contiguous GPU tensor [N][K] of type {dtype}")
        n, k = w.shape
        if x.dim() < 1 or x.shape[-1] != k:
            raise ValueError(f"x must have {k} channels, the weight's columns")
        if (k | n) >> 31:
            raise ValueError("weight's rows and columns do not fit 32 bits")
        bias, r_stride, r_at = self.bias, 0, None
        if residual is not None:
            r_stride, r_at = _channel_last(residual, "residual", x.shape[:-1] + (n,), dtype), residual.data_ptr()
        _on_current_device(x, w, bias, residual)
        return _Linear(x.numel() // k if k else 0, k, n, _int32(self.act, "act"), _GRID_DTYPES[dtype], _position_stride(x, "x"), y_stride,
                       r_stride, w.data_ptr(), None if bias is None else _dev_f32(bias, "bias", (n,)), r_at)


def _linear_bytes(q: _Linear, backward: bool = True):
    f, b = C.c_size_t(), C.c_size_t()
    _check(_lib.lp_linear_workspace_bytes(C.byref(q), C.byref(f), C.byref(b) if backward else None))
    return f.value, b.value


def lp_linear_workspace_bytes(linear: Linear, x: torch.Tensor):
    """(forward bytes, backward bytes) of workspace."""
    return _linear_bytes(linear.c_struct(x))


def _contiguous_like(t: Optional[torch.Tensor], name: str, shape, dtype) -> Optional[int]:
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous() and t.shape == shape and t.dtype is dtype):
        raise ValueError(f"{name} must be a contiguous GPU tensor of shape {tuple(shape)} and type {dtype}")
    return t.data_ptr()


def lp_linear_fwd(linear: Linear, x: torch.Tensor, y: torch.Tensor, pre: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the forward: y [...][N] (the type of x) is written, and pre (contiguous, of y's shape; None: not wanted) for the backward.
    y may be the residual itself."""
    out = x.shape[:-1] + (linear.weight.shape[0],)
    q = linear.c_struct(x, _channel_last(y, "y", out, x.dtype), residual)
    _on_current_device(x, y, pre, workspace)
    w = linear.weight
    _apart(y, q.y_stride, x, q.x_stride, "y", "x")
    _apart(y, q.y_stride, w, w.shape[1], "y", "weight")
    if residual is not None:
        _no_overlap(y, q.y_stride, residual, q.r_stride, "y", "residual")
    pre_at = _contiguous_like(pre, "pre", out, x.dtype)
    if pre is not None:
        for t, step, name in ((x, q.x_stride, "x"), (y, q.y_stride, "y"), (residual, q.r_stride, "residual"), (w, w.shape[1], "weight")):
            _apart(pre, out[-1], t, step, "pre", name)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_linear_fwd(C.byref(q), x.data_ptr(), y.data_ptr(), pre_at, wp, wn, _stream_ptr(stream)))
    _written(y, pre)


def lp_linear_bwd(linear: Linear, x: torch.Tensor, pre: Optional[torch.Tensor], d_y: torch.Tensor, d_x: Optional[torch.Tensor],
                  d_weight: Optional[torch.Tensor], d_bias: Optional[torch.Tensor], workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue the backward: d_x (shape, type and strides of x) is written, d_weight [N][K] and d_bias [N] (float32) are accumulated
    into; each may be None.  pre as the forward wrote it (None without an activation)."""
    n, k = linear.weight.shape
    out = x.shape[:-1] + (n,)
    q = linear.c_struct(x, _channel_last(d_y, "d_y", out, x.dtype))
    _on_current_device(x, pre, d_y, d_x, d_weight, d_bias, workspace)
    pre_at = _contiguous_like(pre, "pre", out, x.dtype)
    if d_x is not None:
        if _channel_last(d_x, "d_x", x.shape, x.dtype) != q.x_stride:
            raise ValueError("d_x must have the strides of x")
        for t, step, name in ((x, q.x_stride, "x"), (d_y, q.y_stride, "d_y"), (pre, n, "pre"), (linear.weight, k, "weight")):
            _apart(d_x, q.x_stride, t, step, "d_x", name)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_linear_bwd(C.byref(q), x.data_ptr(), pre_at, d_y.data_ptr(), None if d_x is None else d_x.data_ptr(),
                              _dev_f32(d_weight, "d_weight", (n, k)), _dev_f32(d_bias, "d_bias", (n,)), wp, wn, _stream_ptr(stream)))
    _written(d_x, d_weight, d_bias)


@dataclasses.dataclass
class ResidualNorm:
    """The norms around a residual block, for tensors [...][C] or, with a gate for each sample, [N][...][C]: with f the block's result
    and h the sum before it, s = alpha h + gate u, u = post_gamma norm(f) (post_norm) or f, and y = gamma norm(s) + beta.
    kind: LP_NORM_RMS or LP_NORM_LAYER, of both norms; gamma, beta, post_gamma: float32 [C] or None; gate: float32 [C], [N][C] or None."""
    kind: int = LP_NORM_RMS
    gamma: Optional[torch.Tensor] = None
    beta: Optional[torch.Tensor] = None
    post_norm: bool = False
    post_gamma: Optional[torch.Tensor] = None
    gate: Optional[torch.Tensor] = None
    alpha: float = 1.0
    eps: float = 1e-5

    def c_struct(self, h: torch.Tensor, f_dtype=None, f_stride: int = 0, y_stride: int = 0) -> _ResidualNorm:
        f_dtype = h.dtype if f_dtype is None else f_dtype
        if h.dtype not in _GRID_DTYPES or f_dtype not in _GRID_DTYPES:
            raise ValueError("h, f and y must be float32, bfloat16 or float16")
        shape = h.shape
        if len(shape) < 1:
            raise ValueError("h must have a last axis of channels")
        c = shape[-1]
        n = shape[0] if len(shape) > 1 else 1
        gamma, beta, post_gamma, gate, per_sample, gate_at = self.gamma, self.beta, self.post_gamma, self.gate, 0, None
        if gate is not None:
            per_sample = int(gate.dim() == 2)
            gate_at = _dev_f32(gate, "gate", (n, c) if per_sample else (c,))
        _on_current_device(h, gamma, beta, post_gamma, gate)
        return _ResidualNorm(n, h.numel() // (n * c) if n and c else 0, _int32(c, "the number of channels"), _int32(self.kind, "kind"),
                             _int32(self.post_norm, "post_norm"), per_sample, self.alpha, self.eps, _GRID_DTYPES[h.dtype],
                             _GRID_DTYPES[f_dtype], _position_stride(h, "h"), f_stride, y_stride,
                             None if post_gamma is None else _dev_f32(post_gamma, "post_gamma", (c,)), gate_at,
                             None if gamma is None else _dev_f32(gamma, "gamma", (c,)), None if beta is None else _dev_f32(beta, "beta", (c,)))


def lp_residual_norm_workspace_bytes(norm: ResidualNorm, h: torch.Tensor) -> int:
    """Bytes of workspace of the backward."""
    n = C.c_size_t()
    _check(_lib.lp_residual_norm_workspace_bytes(C.byref(norm.c_struct(h)), C.byref(n)))
    return n.value


def _same_step(t: Optional[torch.Tensor], name: str, shape, dtype, step: int, of: str) -> Optional[int]:
    if t is None:
        return None
    if _channel_last(t, name, shape, dtype) != step and t.numel():
        raise ValueError(f"{name} must have the strides of {of}")
    return t.data_ptr()


def _f_type(h: torch.Tensor, *tensors: Optional[torch.Tensor]):
    """The type of f and y and their gradients."""
    return next((t.dtype for t in tensors if t is not None), h.dtype)


def lp_residual_norm_fwd(norm: ResidualNorm, h: torch.Tensor, f: Optional[torch.Tensor], s: Optional[torch.Tensor], y: Optional[torch.Tensor],
                         stream=None) -> None:
    """Enqueue the forward: s (shape, type and strides of h) and y (shape of h, type of f) are written; either may be None.  f may be
    None (the first norm of a network).  s may be h itself, y may be f itself."""
    dtype = _f_type(h, f, y)
    steps = [0 if t is None else _channel_last(t, name, h.shape, dtype) for t, name in ((f, "f"), (y, "y"))]
    q = norm.c_struct(h, dtype, *steps)
    _on_current_device(h, f, s, y)
    s_at = _same_step(s, "s", h.shape, h.dtype, q.h_stride, "h")
    if s is not None:
        _no_overlap(s, q.h_stride, h, q.h_stride, "s", "h")
        _apart(s, q.h_stride, f, q.f_stride, "s", "f")
        _apart(s, q.h_stride, y, q.y_stride, "s", "y")
    if y is not None:
        _apart(y, q.y_stride, h, q.h_stride, "y", "h")
        if f is not None:
            _no_overlap(y, q.y_stride, f, q.f_stride, "y", "f")
    _check(_lib.lp_residual_norm_fwd(C.byref(q), h.data_ptr(), None if f is None else f.data_ptr(), s_at, None if y is None else y.data_ptr(),
                                     _stream_ptr(stream)))
    _written(s, y)


def lp_residual_norm_bwd(norm: ResidualNorm, h: torch.Tensor, f: Optional[torch.Tensor], d_s: Optional[torch.Tensor], d_y: Optional[torch.Tensor],
                         d_h: Optional[torch.Tensor], d_f: Optional[torch.Tensor], d_gamma: Optional[torch.Tensor], d_beta: Optional[torch.Tensor],
                         d_post_gamma: Optional[torch.Tensor], d_gate: Optional[torch.Tensor], workspace: torch.Tensor, stream=None) -> None:
    """Enqueue the backward, from the forward's inputs: d_h and d_f are written, d_gamma, d_beta, d_post_gamma and d_gate accumulated
    into; each may be None, and so may d_s and d_y (zero).  d_s and d_h have the strides of h, d_f those of f."""
    dtype = _f_type(h, f, d_y, d_f)
    steps = [0 if t is None else _channel_last(t, name, h.shape, dtype) for t, name in ((f, "f"), (d_y, "d_y"))]
    q = norm.c_struct(h, dtype, *steps)
    _on_current_device(h, f, d_s, d_y, d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate, workspace)
    d_s_at, d_h_at = (_same_step(t, name, h.shape, h.dtype, q.h_stride, "h") for t, name in ((d_s, "d_s"), (d_h, "d_h")))
    d_f_at = _same_step(d_f, "d_f", h.shape, dtype, q.f_stride or h.shape[-1], "f")
    if d_h is not None:
        for t, step, name in ((h, q.h_stride, "h"), (f, q.f_stride, "f"), (d_y, q.y_stride, "d_y"), (d_f, q.f_stride, "d_f")):
            _apart(d_h, q.h_stride, t, step, "d_h", name)
        if d_s is not None:
            _no_overlap(d_h, q.h_stride, d_s, q.h_stride, "d_h", "d_s")
    if d_f is not None:
        for t, step, name in ((h, q.h_stride, "h"), (f, q.f_stride, "f"), (d_s, q.h_stride, "d_s")):
            _apart(d_f, q.f_stride, t, step, "d_f", name)
        if d_y is not None:
            _no_overlap(d_f, q.f_stride, d_y, q.y_stride, "d_f", "d_y")
    c = (h.shape[-1],)
    wp, wn = _workspace(workspace)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    _check(_lib.lp_residual_norm_bwd(C.byref(q), h.data_ptr(), at(f), d_s_at, at(d_y), d_h_at, d_f_at, _dev_f32(d_gamma, "d_gamma", c),
                                     _dev_f32(d_beta, "d_beta", c), _dev_f32(d_post_gamma, "d_post_gamma", c),
                                     _dev_f32(d_gate, "d_gate", c if norm.gate is None else norm.gate.shape), wp, wn, _stream_ptr(stream)))
    _written(d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate)


def _is_dense(t: torch.Tensor) -> bool:
    """Whether a tensor's values lie one behind the other, in any order of its axes."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != step:
            return False
        step *= size
    return True


def _gradients(grads, outs):
    """The call's structs (tensors are also checked to be on the current device)."""
    if len(grads) != len(outs):
        raise ValueError("one output per gradient is needed")
    values, device = [], None
    for k, g in enumerate(grads):
        o, dtype, dense = outs[k], g.dtype, g.is_contiguous()
        if not (g.is_cuda if device is None else g.device == device) or dtype not in _GRID_DTYPES or not (dense or _is_dense(g)):
            raise ValueError(f"grads[{k}] must be a dense float32, bfloat16 or float16 tensor on the GPU, all on one device")
        at = to = g.data_ptr()
        if o is not g:
            if not (o.dtype is dtype and o.shape == g.shape and o.device == g.device and (o.is_contiguous() if dense else o.stride() == g.stride())):
                raise ValueError(f"outs[{k}] must be a tensor of the shape, type and strides of grads[{k}], all on one device")
            to = o.data_ptr()
        if device is None:
            device = _on_current_device(g)
        values += (g.numel(), at, to, _GRID_DTYPES[dtype])
    # (one buffer of structs, laid out as _Gradient is)
    return (_Gradient * max(1, len(grads))).from_buffer(bytearray(struct.pack("qQQi4x" * len(grads), *values) or C.sizeof(_Gradient)))


def _grad_norm_bytes(n: int, arr) -> int:
    size = C.c_size_t(0)
    _check(_lib.lp_grad_norm_workspace_bytes(n, arr, C.byref(size)))
    return size.value


def lp_grad_norm_workspace_bytes(grads: Sequence[torch.Tensor]) -> int:
    return _grad_norm_bytes(len(grads), _gradients(grads, grads))


def lp_grad_norm(grads: Sequence[torch.Tensor], norm: torch.Tensor, workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue the norm of all gradients together: norm (float32, shape ()) is written."""
    arr = _gradients(grads, grads)
    _on_current_device(norm, *grads[:1], workspace)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_grad_norm(len(grads), arr, _dev_f32(norm, "norm", ()), wp, wn, _stream_ptr(stream)))
    _written(norm)


def lp_clip_grad_norm(grads: Sequence[torch.Tensor], outs: Sequence[torch.Tensor], max_norm: float, norm: torch.Tensor,
                      workspace: Optional[torch.Tensor], eps: float = 1e-6, stream=None) -> None:
    """Enqueue the clipping: outs (the gradients themselves, or tensors like them) and norm (float32, shape ()) are written."""
    arr = _gradients(grads, outs)
    _on_current_device(norm, *grads[:1], workspace)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_clip_grad_norm(len(grads), arr, float(max_norm), float(eps), _dev_f32(norm, "norm", ()), wp, wn, _stream_ptr(stream)))
    increment_version([*outs, norm])


def _matrix_shape(t: torch.Tensor, name: str, k: int):
    if not (t.is_cuda and t.is_contiguous() and t.dim() >= 2):
        raise ValueError(f"{name}[{k}] must be a contiguous GPU tensor [...][rows][cols]")
    rows, cols = t.shape[-2], t.shape[-1]
    if (rows | cols) >> 31:
        raise ValueError(f"rows and columns of {name}[{k}] do not fit 32 bits")
    return t.numel() // max(1, rows * cols), rows, cols


def _matrices(mats, outs):
    if len(mats) != len(outs):
        raise ValueError("one output per input is needed")
    arr = (_Matrices * max(1, len(mats)))()
    for k, (g, o) in enumerate(zip(mats, outs)):
        count, rows, cols = _matrix_shape(g, "mats", k)
        if g.dtype not in _GRID_DTYPES:
            raise ValueError("matrices must be float32, bfloat16 or float16")
        if o is not g and not (o.is_cuda and o.is_contiguous() and o.dtype is g.dtype and o.shape == g.shape):
            raise ValueError(f"outs[{k}] must be a contiguous GPU tensor of the shape and type of mats[{k}]")
        arr[k] = _Matrices(count, rows, cols, g.data_ptr(), o.data_ptr(), _GRID_DTYPES[g.dtype])
    return arr


def _orth(steps: int, coeffs, eps: float) -> _Orth:
    """(a struct of `steps` steps; coeffs: one (a, b, c) for all steps, one for each, or None)"""
    steps = _int32(steps, "steps")
    if coeffs is None:
        return _Orth(steps, None, float(eps))
    one = len(coeffs) and isinstance(coeffs[0], (int, float))
    rows = [tuple(float(v) for v in r) for r in ([coeffs] * steps if one else coeffs)]
    if len(rows) != steps or any(len(r) != 3 for r in rows):
        raise ValueError("coeffs must be (a, b, c), or one of these for every step")
    flat = (C.c_float * max(1, 3 * len(rows)))(*[v for r in rows for v in r])
    o = _Orth(steps, flat, float(eps))
    o.keep = flat
    return o


def lp_orthogonalize_workspace_bytes(mats: Sequence[torch.Tensor]) -> int:
    arr, n = _matrices(mats, mats), C.c_size_t(0)
    _check(_lib.lp_orthogonalize_workspace_bytes(len(mats), arr, C.byref(n)))
    return int(n.value)


def lp_orthogonalize(mats: Sequence[torch.Tensor], outs: Sequence[torch.Tensor], workspace: torch.Tensor, steps: int = 5,
                     coeffs=None, eps: float = 1e-7, stream=None) -> None:
    """Enqueue the orthogonalisation of the matrices in `mats` (tensors [...][rows][cols], float32, bfloat16 or float16); outs
    (same shapes and types, or the inputs themselves) are written."""
    arr, o = _matrices(mats, outs), _orth(steps, coeffs, eps)
    wp, wn = _workspace(workspace)
    _check(_lib.lp_orthogonalize(len(mats), arr, C.byref(o), wp, wn, _stream_ptr(stream)))
    increment_version(outs)


def _muon_weights(weights, grads, momenta):
    if not len(weights) == len(grads) == len(momenta):
        raise ValueError("one gradient and one momentum per weight are needed")
    arr = (_MuonWeights * max(1, len(weights)))()
    for k, (w, g, m) in enumerate(zip(weights, grads, momenta)):
        shape = w.shape
        count, rows, cols = _matrix_shape(w, "weights", k)
        arr[k] = _MuonWeights(count, rows, cols, _dev_f32(w, "weights", None, k), _dev_f32(g, "grads", shape, k),
                              _dev_f32(m, "momenta", shape, k))
    return arr


def lp_muon_workspace_bytes(weights: Sequence[torch.Tensor]) -> int:
    arr, n = _muon_weights(weights, weights, weights), C.c_size_t(0)
    _check(_lib.lp_muon_workspace_bytes(len(weights), arr, C.byref(n)))
    return int(n.value)


def lp_muon_step(weights: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], momenta: Sequence[torch.Tensor],
                 workspace: torch.Tensor, lr: float, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 scale: int = LP_MUON_SCALE_ASPECT, steps: int = 5, coeffs=None, eps: float = 1e-7, stream=None) -> None:
    """Enqueue one optimiser step: weights and momenta (float32 tensors [...][rows][cols]) are updated in place."""
    arr = _muon_weights(weights, grads, momenta)
    q = _Muon(float(lr), float(momentum), float(weight_decay), _int32(nesterov, "nesterov"), _int32(scale, "scale"),
              _orth(steps, coeffs, eps))
    wp, wn = _workspace(workspace)
    _check(_lib.lp_muon_step(len(weights), arr, C.byref(q), wp, wn, _stream_ptr(stream)))
    increment_version([*weights, *momenta])


# ---------------------------------------------------------------------------------------
# Conveniences on top of the entry points: move host buffers to the GPU, allocate outputs.

def to_device(inp, device="cuda:0"):
    """Upload host buffers (any object with the fields of `lp_inputs.Inputs`) and return
    (Grid, Mlp, Rays, bg) on `device`."""
    dev = torch.device(device)
    up = lambda a: torch.from_numpy(a).to(dev)
    grid = Grid(kind=int(inp.kind), data=[up(g) for g in inp.grid], res=tuple(inp.res),
                aabb_min=tuple(inp.aabb_min), aabb_max=tuple(inp.aabb_max),
                contract_a=float(getattr(inp, "contract_a", 0.0)), t_range=tuple(getattr(inp, "t_range", (0.0, 1.0))))
    mlp = Mlp(weights=[up(w) for w in inp.weights], biases=[up(b) for b in inp.biases])
    rays = Rays(origins=up(inp.origins), dirs=up(inp.dirs), near=up(inp.near), far=up(inp.far),
                samples=int(inp.samples), scene=None if inp.scene is None else up(inp.scene),
                time=None if getattr(inp, "time", None) is None else up(inp.time))
    return grid, mlp, rays, tuple(float(v) for v in inp.bg)


def decoder_to_device(dec, device="cuda:0") -> Decoder:
    """Upload a host decoder (fields of `lp_inputs.Decoder`)."""
    dev = torch.device(device)
    up = lambda a: torch.from_numpy(a).to(dev)
    return Decoder(opacity=Mlp([up(w) for w in dec.weights_s], [up(b) for b in dec.biases_s]),
                   feature=Mlp([up(w) for w in dec.weights_v], [up(b) for b in dec.biases_v]),
                   n_freq=int(dec.n_freq), n_feat=int(dec.n_feat), feat_act=int(dec.feat_act))


def render_dec_fwd(grid: Grid, dec: Decoder, rays: Rays, bg, math_mode: int = LP_MATH_DEFAULT):
    """Allocate outputs and workspace and run lp_render_dec_fwd.  Returns (out, alpha, depth, ray_cache)."""
    dev = rays.origins.device
    m = rays.n_rays
    out = torch.empty((m, dec.n_feat), dtype=torch.float32, device=dev)
    alpha = torch.empty((m,), dtype=torch.float32, device=dev)
    depth = torch.empty((m,), dtype=torch.float32, device=dev)
    cache = torch.empty((m,), dtype=torch.float32, device=dev)
    ws = torch.empty(lp_dec_workspace_bytes(grid, dec, rays, math_mode)[0], dtype=torch.uint8, device=dev)
    lp_render_dec_fwd(grid, dec, rays, bg, out, alpha, depth, cache, ws, math_mode)
    return out, alpha, depth, cache


def render_dec_bwd(grid: Grid, dec: Decoder, rays: Rays, bg, d_out, ray_cache, d_alpha=None, d_depth=None,
                   math_mode: int = LP_MATH_DEFAULT):
    """Allocate zeroed gradient buffers and a workspace and run lp_render_dec_bwd.
    Returns (d_grid, dW_opacity, db_opacity, dW_feature, db_feature)."""
    dev = rays.origins.device
    d_grid = [torch.zeros_like(t, dtype=torch.float32) for t in grid.data]   # gradients are float32 whatever the storage
    z = lambda lst: [torch.zeros_like(t) for t in lst]
    dWs, dbs, dWv, dbv = z(dec.opacity.weights), z(dec.opacity.biases), z(dec.feature.weights), z(dec.feature.biases)
    ws = torch.empty(lp_dec_workspace_bytes(grid, dec, rays, math_mode)[1], dtype=torch.uint8, device=dev)
    lp_render_dec_bwd(grid, dec, rays, bg, d_out, d_alpha, d_depth, ray_cache, d_grid, dWs, dbs, dWv, dbv, ws,
                      math_mode)
    return d_grid, dWs, dbs, dWv, dbv


def render_fwd(grid: Grid, mlp: Mlp, rays: Rays, bg, math_mode: int = LP_MATH_DEFAULT):
    """Allocate outputs and run lp_render_fwd.  Returns (rgb, alpha, depth, ray_cache)."""
    dev = rays.origins.device
    m = rays.n_rays
    rgb = torch.empty((m, 3), dtype=torch.float32, device=dev)
    alpha = torch.empty((m,), dtype=torch.float32, device=dev)
    depth = torch.empty((m,), dtype=torch.float32, device=dev)
    cache = torch.empty((m,), dtype=torch.float32, device=dev)
    lp_render_fwd(grid, mlp, rays, bg, rgb, alpha, depth, cache, math_mode)
    return rgb, alpha, depth, cache


def render_bwd(grid: Grid, mlp: Mlp, rays: Rays, bg, d_rgb, ray_cache, d_alpha=None, d_depth=None,
               math_mode: int = LP_MATH_DEFAULT, workspace: Optional[torch.Tensor] = None):
    """Allocate zeroed gradient buffers (and a workspace) and run lp_render_bwd.
    Returns (d_grid list, dW list, db list)."""
    dev = rays.origins.device
    d_grid = [torch.zeros_like(t, dtype=torch.float32) for t in grid.data]   # gradients are float32 whatever the storage
    dW = [torch.zeros_like(w) for w in mlp.weights]
    db = [torch.zeros_like(b) for b in mlp.biases]
    if workspace is None:
        workspace = torch.empty(lp_bwd_workspace_bytes(grid, mlp, rays, math_mode), dtype=torch.uint8, device=dev)
    lp_render_bwd(grid, mlp, rays, bg, d_rgb, d_alpha, d_depth, ray_cache, d_grid, dW, db, workspace, math_mode)
    return d_grid, dW, db


def splat_to_device(sp, device="cuda:0"):
    """Upload host buffers with the fields of `lp_inputs.SplatInputs`.  Returns (target, Rays, Splat)."""
    dev = torch.device(device)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    target = target_struct(sp.kind, sp.n_scenes, sp.channels, sp.res, sp.aabb_min, sp.aabb_max, sp.contract_a,
                           getattr(sp, "hash_size", 0))
    rays = Rays(origins=up(sp.origins), dirs=up(sp.dirs), near=up(sp.near), far=up(sp.far),
                samples=int(sp.samples), scene=None if sp.scene is None else up(sp.scene))
    prior = None
    if sp.prior is not None:
        prior = Grid(kind=int(sp.kind), data=[up(g) for g in sp.prior], res=tuple(sp.prior_res),
                     aabb_min=tuple(sp.aabb_min), aabb_max=tuple(sp.aabb_max), contract_a=float(sp.contract_a))
    mlp = None if sp.mlp_dims is None else Mlp([up(w) for w in sp.weights], [up(b) for b in sp.biases])
    return target, rays, Splat(feats=up(sp.feats), prior=prior, mlp=mlp, n_freq=int(sp.n_freq))


def splat_fwd(target: _Grid, rays: Rays, splat: Splat):
    """Allocate outputs and run lp_splat_fwd.  Returns (theta list, theta_w list)."""
    dev = rays.origins.device
    theta = [torch.empty(s, dtype=torch.float32, device=dev) for s in _target_shapes(target, target.C)]
    theta_w = [torch.empty(s, dtype=torch.float32, device=dev) for s in _target_shapes(target, None)]
    lp_splat_fwd(target, rays, splat, theta, theta_w)
    return theta, theta_w


def splat_bwd(target: _Grid, rays: Rays, splat: Splat, theta_w, d_theta):
    """Allocate gradient buffers and workspace and run lp_splat_bwd.
    Returns (d_feats, d_prior list, dW list, db list)."""
    dev = rays.origins.device
    d_feats = torch.empty_like(splat.feats)
    d_prior = [] if splat.prior is None else [torch.zeros_like(t) for t in splat.prior.data]
    dW = [] if splat.mlp is None else [torch.zeros_like(w) for w in splat.mlp.weights]
    db = [] if splat.mlp is None else [torch.zeros_like(b) for b in splat.mlp.biases]
    ws = torch.empty(lp_splat_bwd_workspace_bytes(target, rays, splat), dtype=torch.uint8, device=dev)
    lp_splat_bwd(target, rays, splat, theta_w, d_theta, d_feats, d_prior, dW, db, ws)
    return d_feats, d_prior, dW, db


def group_norm_fwd(norm: GroupNorm, x: torch.Tensor, dtype=None):
    """Allocate outputs and workspace and run lp_group_norm_fwd.  Returns (y, stats); dtype: of y (default: that of x)."""
    q = norm.c_struct(x, dtype)   # (new outputs are dense: what the entry point checks of them holds)
    y = torch.empty(x.shape, dtype=x.dtype if dtype is None else dtype, device=x.device)
    stats = torch.empty((q.N, q.G, 2), device=x.device, dtype=torch.float32)
    n = _norm_bytes(q)[0]
    ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None   # (held until the kernels are enqueued)
    _check(_lib.lp_group_norm_fwd(C.byref(q), x.data_ptr(), y.data_ptr(), stats.data_ptr(), ws.data_ptr() if n else None, n,
                                  _stream_ptr(None)))
    return y, stats


def group_norm_bwd(norm: GroupNorm, x: torch.Tensor, stats: torch.Tensor, d_y: torch.Tensor):
    """Allocate gradients and workspace and run lp_group_norm_bwd.  Returns (d_x, d_gamma, d_beta)."""
    q = norm.c_struct(x, d_y.dtype, _channel_last(d_y, "d_y", x.shape, d_y.dtype))
    d_x = torch.empty_like(x) if x.is_contiguous() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    d_params = torch.zeros((2, q.C), dtype=torch.float32, device=x.device)
    at = d_params.data_ptr()
    n = _norm_bytes(q)[1]
    ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None   # (held until the kernels are enqueued)
    _check(_lib.lp_group_norm_bwd(C.byref(q), x.data_ptr(), _dev_f32(stats, "stats", (q.N, q.G, 2)), d_y.data_ptr(), d_x.data_ptr(),
                                  at, at + 4 * q.C, ws.data_ptr() if n else None, n, _stream_ptr(None)))
    d_gamma, d_beta = d_params.unbind(0)
    return d_x, d_gamma, d_beta


def linear_fwd(linear: Linear, x: torch.Tensor, residual: Optional[torch.Tensor] = None, keep: bool = False):
    """Allocate outputs and workspace and run lp_linear_fwd.  Returns (y, pre); pre (keep; else None) is for linear_bwd, which needs it
    where there is an activation."""
    q = linear.c_struct(x, 0, residual)   # (new outputs are dense: what the entry point checks of them holds)
    shape = x.shape
    y = x.new_empty((shape[0], q.N) if len(shape) == 2 else shape[:-1] + (q.N,))
    pre = torch.empty_like(y) if keep else None
    n = _linear_bytes(q, False)[0]
    ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None   # (held until the kernels are enqueued)
    _check(_lib.lp_linear_fwd(C.byref(q), x.data_ptr(), y.data_ptr(), pre.data_ptr() if keep else None, ws.data_ptr() if n else None, n,
                              _stream_ptr(None)))
    return y, pre


def linear_bwd(linear: Linear, x: torch.Tensor, pre: Optional[torch.Tensor], d_y: torch.Tensor):
    """Allocate gradients and workspace and run lp_linear_bwd.  Returns (d_x, d_weight, d_bias); d_weight and d_bias (None without a
    bias) are float32."""
    out = x.shape[:-1] + (linear.weight.shape[0],)
    q = linear.c_struct(x, _channel_last(d_y, "d_y", out, x.dtype))
    _on_current_device(x, pre, d_y)
    d_x = torch.empty_like(x) if x.is_contiguous() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    d_params = torch.zeros(q.N * q.K + (q.N if linear.bias is not None else 0), dtype=torch.float32, device=x.device)
    at = d_params.data_ptr()
    n = _linear_bytes(q)[1]
    ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None   # (held until the kernels are enqueued)
    _check(_lib.lp_linear_bwd(C.byref(q), x.data_ptr(), _contiguous_like(pre, "pre", out, x.dtype), d_y.data_ptr(), d_x.data_ptr(), at,
                              None if linear.bias is None else at + 4 * q.N * q.K, ws.data_ptr() if n else None, n, _stream_ptr(None)))
    return d_x, d_params[:q.N * q.K].view(q.N, q.K), None if linear.bias is None else d_params[q.N * q.K:]


def residual_norm_fwd(norm: ResidualNorm, h: torch.Tensor, f: Optional[torch.Tensor] = None, dtype=None):
    """Allocate outputs and run lp_residual_norm_fwd.  Returns (s, y); y has the type of f (without f: `dtype`, by default that of h).
    Without f and with alpha 1, s is h itself."""
    if f is not None and dtype is not None and dtype is not f.dtype:
        raise ValueError("y has the type of f")
    y_dtype = f.dtype if f is not None else h.dtype if dtype is None else dtype
    q = norm.c_struct(h, y_dtype, 0 if f is None else _channel_last(f, "f", h.shape, y_dtype))
    if f is not None:
        _on_current_device(h, f)
    same, dense = f is None and norm.alpha == 1.0, h.is_contiguous()
    s = h if same else torch.empty_like(h) if dense else torch.empty_strided(h.shape, h.stride(), dtype=h.dtype, device=h.device)
    y = torch.empty_like(h) if dense and y_dtype is h.dtype else torch.empty(h.shape, dtype=y_dtype, device=h.device)
    _check(_lib.lp_residual_norm_fwd(C.byref(q), h.data_ptr(), None if f is None else f.data_ptr(), None if same else s.data_ptr(),
                                     y.data_ptr(), _stream_ptr(None)))
    return s, y


def residual_norm_bwd(norm: ResidualNorm, h: torch.Tensor, f: Optional[torch.Tensor], d_s: Optional[torch.Tensor], d_y: Optional[torch.Tensor]):
    """Allocate gradients and workspace and run lp_residual_norm_bwd.  Returns (d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate), None
    in the place of the gradient of what the norm does not have."""
    shape, dtype = h.shape, _f_type(h, f, d_y)
    q = norm.c_struct(h, dtype, 0 if f is None else _channel_last(f, "f", shape, dtype), 0 if d_y is None else _channel_last(d_y, "d_y", shape, dtype))
    _on_current_device(h, f, d_s, d_y)
    d_s_at = _same_step(d_s, "d_s", shape, h.dtype, q.h_stride, "h")
    # (new gradients do not overlap anything: what the entry point checks of them holds)
    d_h = torch.empty_like(h) if h.is_contiguous() else torch.empty_strided(shape, h.stride(), dtype=h.dtype, device=h.device)
    d_f = None if f is None else torch.empty_like(f) if f.is_contiguous() else torch.empty_strided(shape, f.stride(), dtype=dtype, device=f.device)
    params = (norm.gamma, norm.beta, None, None) if f is None else (norm.gamma, norm.beta, norm.post_gamma, norm.gate)
    sizes = [0 if p is None else p.numel() for p in params]
    zeros = torch.zeros(sum(sizes), dtype=torch.float32, device=h.device)
    at, parts, ats, first = zeros.data_ptr(), [], [], 0
    for p, size in zip(params, sizes):
        parts.append(None if p is None else zeros[first:first + size].view(p.shape) if p.dim() > 1 else zeros[first:first + size])
        ats.append(None if p is None else at + 4 * first)
        first += size
    n = C.c_size_t()
    _check(_lib.lp_residual_norm_workspace_bytes(C.byref(q), C.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=h.device)   # (held until the kernels are enqueued)
    _check(_lib.lp_residual_norm_bwd(C.byref(q), h.data_ptr(), None if f is None else f.data_ptr(), d_s_at, None if d_y is None else d_y.data_ptr(),
                                     d_h.data_ptr(), None if f is None else d_f.data_ptr(), *ats, ws.data_ptr(), n.value, _stream_ptr(None)))
    return (d_h, d_f, *parts)


def grad_norm(grads: Sequence[torch.Tensor]) -> torch.Tensor:
    """Allocate and run lp_grad_norm.  Returns the norm of all gradients together (float32, shape ())."""
    return _norm_of(grads, None, 0.0, 0.0)


def clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float, eps: float = 1e-6, outs: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
    """Allocate a workspace and run lp_clip_grad_norm on the gradients in place, or into outs.  Returns the norm that they had (float32,
    shape ())."""
    return _norm_of(grads, grads if outs is None else outs, max_norm, eps)


def _norm_of(grads, outs, max_norm, eps) -> torch.Tensor:
    if not len(grads):
        raise ValueError("no gradients: without a tensor there is no device for the norm")
    arr, n = _gradients(grads, grads if outs is None else outs), len(grads)
    first = grads[0]
    norm = first.new_empty(()) if first.dtype is torch.float32 else torch.empty((), dtype=torch.float32, device=first.device)
    size = _grad_norm_bytes(n, arr)
    ws = torch.empty(size, dtype=torch.uint8, device=first.device) if size else None   # (held until the kernels are enqueued)
    at = ws.data_ptr() if size else None
    if outs is None:
        _check(_lib.lp_grad_norm(n, arr, norm.data_ptr(), at, size, _stream_ptr(None)))
    else:
        _check(_lib.lp_clip_grad_norm(n, arr, float(max_norm), float(eps), norm.data_ptr(), at, size, _stream_ptr(None)))
        increment_version(outs)
    return norm


def orthogonalize(mats: Sequence[torch.Tensor], steps: int = 5, coeffs=None, eps: float = 1e-7):
    """Allocate outputs and workspace and run lp_orthogonalize.  Returns the outputs."""
    outs = [torch.empty_like(g) for g in mats]
    if mats:
        ws = torch.empty(lp_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device=mats[0].device)
        lp_orthogonalize(mats, outs, ws, steps, coeffs, eps)
    return outs


def muon_step(weights: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], momenta: Sequence[torch.Tensor], lr: float,
              momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: int = LP_MUON_SCALE_ASPECT,
              steps: int = 5, coeffs=None, eps: float = 1e-7) -> None:
    """Allocate a workspace and run lp_muon_step."""
    if weights:
        ws = torch.empty(lp_muon_workspace_bytes(weights), dtype=torch.uint8, device=weights[0].device)
        lp_muon_step(weights, grads, momenta, ws, lr, momentum, nesterov, weight_decay, scale, steps, coeffs, eps)
