"""ctypes binding over libemc2.so: argument marshalling only, every step runs in the HIP kernels.

Tensors are torch CUDA(=HIP) tensors used purely as device buffers; the current torch stream is
passed as the HIP stream.  There is no CPU fallback: if the library is missing or no GPU is present
the calls raise.
"""
from __future__ import annotations

import ctypes
import operator
import os
from typing import Optional, Sequence, Tuple

import torch

from .configs import VoxelSpec

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libemc2.so")

OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_UNSUPPORTED, ERR_DEVICE, ERR_MAP = 0, 1, 2, 3, 4, 5
F32, F16, BF16, I8 = 0, 1, 2, 3
SUBM, STRIDED = 0, 1
EPI_NONE, EPI_AFFINE, EPI_AFFINE_RELU = 0, 1, 2
W_PLAIN, W_PACKED = 0, 1
POOL_MEAN, POOL_MAX = 0, 1
ACT_SILU, ACT_GELU = 0, 1
MAP_ANY = -1   # emc2_spconv map_hint: SUBM / STRIDED as passed to build_kmap, or unknown

_TORCH_DTYPE = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}

EXPORTS = ["emc2_create", "emc2_destroy", "emc2_status_sync", "emc2_last_error", "emc2_voxelize",
           "emc2_build_kmap", "emc2_spconv", "emc2_project_gather", "emc2_pack_weights", "emc2_spconv_uses_mfma",
           "emc2_spconv_kernel", "emc2_build_inverse_kmap", "emc2_bev_flatten", "emc2_pool_image", "emc2_fuse", "emc2_dispatch", "emc2_spconv_i8_supported",
           "emc2_quantize_i8", "emc2_pack_weights_i8", "emc2_spconv_i8", "emc2_build_kmap_static", "emc2_group_points", "emc2_quantize_e4m3", "emc2_spconv_e4m3",
           "emc2_build_stacks", "emc2_spconv_list", "emc2_group_slots",
           "emc2_frame_offsets", "emc2_layernorm", "emc2_layernorm_work", "emc2_layernorm_backward", "emc2_recurrence", "emc2_recurrence_work",
           "emc2_recurrence_backward", "emc2_recurrence_step", "emc2_ffn_packed_size", "emc2_ffn_pack", "emc2_ffn", "emc2_ffn_work",
           "emc2_ffn_backward", "emc2_causal_conv", "emc2_causal_conv_work", "emc2_causal_conv_backward", "emc2_causal_conv_step",
           "emc2_gated_residual", "emc2_gated_residual_work", "emc2_gated_residual_backward",
           "emc2_selective_scan", "emc2_selective_scan_work", "emc2_selective_scan_backward", "emc2_selective_scan_step"]


class Emc2Error(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"emc2 status {status}: {msg}")
        self.status = status


class _VoxelSpecC(ctypes.Structure):
    _fields_ = [("lo", ctypes.c_float * 3), ("vs", ctypes.c_float * 3), ("grid", ctypes.c_int32 * 3),
                ("n_batch", ctypes.c_int32), ("r2_min", ctypes.c_float), ("r2_max", ctypes.c_float),
                ("stride_f", ctypes.c_int32)]


def voxel_spec_c(spec: VoxelSpec, stride: int) -> _VoxelSpecC:
    return _VoxelSpecC((ctypes.c_float * 3)(*spec.lo), (ctypes.c_float * 3)(*spec.vs), (ctypes.c_int32 * 3)(*spec.grid),
                       spec.n_batch, spec.r2_min, spec.r2_max, stride)


STACK_MAX_LEVELS, MAX_STACKS = 5, 4


class StackLevelC(ctypes.Structure):
    """emc2_stack_level"""
    _fields_ = [("capacity", ctypes.c_int64), ("d_coords", ctypes.c_void_p), ("d_n", ctypes.c_void_p), ("d_subm_nbr", ctypes.c_void_p),
                ("d_down_nbr", ctypes.c_void_p), ("slot", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class StackC(ctypes.Structure):
    """emc2_stack"""
    _fields_ = [("ctx", ctypes.c_void_p), ("spec", _VoxelSpecC), ("expert", ctypes.c_int32), ("n_levels", ctypes.c_int32),
                ("lp_dtype", ctypes.c_int), ("d_batch", ctypes.c_void_p), ("d_route", ctypes.c_void_p), ("d_slot", ctypes.c_void_p),
                ("d_feats", ctypes.c_void_p), ("d_counts", ctypes.c_void_p), ("d_feats_lp", ctypes.c_void_p),
                ("level", StackLevelC * STACK_MAX_LEVELS), ("d_group_batch", ctypes.c_void_p)]


class ConvCallC(ctypes.Structure):
    """emc2_conv_call"""
    _fields_ = [("ctx", ctypes.c_void_p), ("d_in", ctypes.c_void_p), ("d_w", ctypes.c_void_p), ("d_scale", ctypes.c_void_p),
                ("d_shift", ctypes.c_void_p), ("d_nbr", ctypes.c_void_p), ("d_n_out", ctypes.c_void_p), ("d_out", ctypes.c_void_p),
                ("capacity_out", ctypes.c_int64), ("n_in_rows", ctypes.c_int64), ("dtype", ctypes.c_int), ("w_layout", ctypes.c_int),
                ("epilogue", ctypes.c_int), ("map_hint", ctypes.c_int32), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libemc2.so (build it first with ``python -m paper_2507_04123_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is not built; run __graft_entry__.build() or paper_2507_04123_amd/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    lib.emc2_create.restype = ctypes.c_int
    lib.emc2_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, i64, i64, i64, i32]
    lib.emc2_destroy.restype = None
    lib.emc2_destroy.argtypes = [vp]
    lib.emc2_status_sync.restype = ctypes.c_int
    lib.emc2_status_sync.argtypes = [vp, vp]
    lib.emc2_last_error.restype = ctypes.c_char_p
    lib.emc2_last_error.argtypes = [vp]
    lib.emc2_voxelize.restype = ctypes.c_int
    lib.emc2_voxelize.argtypes = [vp, vp, vp, i64, ctypes.POINTER(_VoxelSpecC), i64, vp, vp, vp, vp, ctypes.c_int, vp,
                                  ctypes.POINTER(i32), i32, vp]
    lib.emc2_build_kmap.restype = ctypes.c_int
    lib.emc2_build_kmap.argtypes = [vp, ctypes.c_int, vp, vp, i64, ctypes.POINTER(i32), i32, i32, i32, i64, vp, vp, vp,
                                    ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
    lib.emc2_build_kmap_static.restype = ctypes.c_int
    lib.emc2_build_kmap_static.argtypes = [ctypes.c_int, vp, vp, i64, ctypes.POINTER(i32), i32, i64, vp, vp, vp,
                                           ctypes.POINTER(i32), vp, vp]
    lib.emc2_spconv.restype = ctypes.c_int
    lib.emc2_spconv.argtypes = [vp, ctypes.c_int, vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, vp, i32, vp, i64, i64, i32, i32, vp, vp]
    lib.emc2_pack_weights.restype = ctypes.c_int
    lib.emc2_pack_weights.argtypes = [vp, ctypes.c_int, vp, i32, i32, vp, vp]
    lib.emc2_spconv_kernel.restype = ctypes.c_char_p
    lib.emc2_spconv_kernel.argtypes = [ctypes.c_int, i32, i32, i32]
    lib.emc2_spconv_uses_mfma.restype = i32
    lib.emc2_spconv_uses_mfma.argtypes = [ctypes.c_int, i32, i32]
    lib.emc2_pool_image.restype = ctypes.c_int
    lib.emc2_pool_image.argtypes = [vp, vp, vp, i32, i32, i32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(_VoxelSpecC),
                                    i32, ctypes.c_int, i64, vp, vp, vp, vp, ctypes.POINTER(i32), i32, vp]
    lib.emc2_fuse.restype = ctypes.c_int
    lib.emc2_fuse.argtypes = [vp, ctypes.c_int, vp, vp, vp, i64, i32, vp, vp, vp, i64, i32, ctypes.POINTER(i32), i32, i32,
                              i64, i32, vp, vp, vp, vp, vp, ctypes.POINTER(i32), vp]
    lib.emc2_spconv_i8_supported.restype = i32
    lib.emc2_spconv_i8_supported.argtypes = [i32, i32]
    lib.emc2_quantize_i8.restype = ctypes.c_int
    lib.emc2_quantize_i8.argtypes = [vp, ctypes.c_int, vp, i64, ctypes.c_float, vp, vp]
    lib.emc2_pack_weights_i8.restype = ctypes.c_int
    lib.emc2_pack_weights_i8.argtypes = [vp, vp, i32, i32, vp, vp]
    lib.emc2_spconv_i8.restype = ctypes.c_int
    lib.emc2_spconv_i8.argtypes = [vp, vp, vp, vp, vp, i32, ctypes.c_int, ctypes.c_float, vp, vp, i64, i64, i32, i32, vp, vp]
    lib.emc2_quantize_e4m3.restype = ctypes.c_int
    lib.emc2_quantize_e4m3.argtypes = [vp, ctypes.c_int, vp, i64, ctypes.c_float, vp, vp]
    lib.emc2_spconv_e4m3.restype = ctypes.c_int
    lib.emc2_spconv_e4m3.argtypes = [vp, vp, vp, vp, vp, i32, ctypes.c_int, vp, vp, i64, i64, i32, i32, vp, vp]
    lib.emc2_dispatch.restype = ctypes.c_int
    lib.emc2_dispatch.argtypes = [vp, vp, vp, i64, i32, ctypes.c_float, ctypes.c_float, vp, vp, vp, vp]
    lib.emc2_group_points.restype = ctypes.c_int
    lib.emc2_group_points.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.emc2_project_gather.restype = ctypes.c_int
    lib.emc2_project_gather.argtypes = [vp, vp, i32, i64, ctypes.POINTER(ctypes.c_float), vp, i32, i32, i32, vp, vp, vp, vp]
    lib.emc2_build_stacks.restype = ctypes.c_int
    lib.emc2_build_stacks.argtypes = [ctypes.POINTER(StackC), i32, vp, i64, vp]
    lib.emc2_spconv_list.restype = ctypes.c_int
    lib.emc2_spconv_list.argtypes = [ctypes.POINTER(ConvCallC), i32, vp]
    lib.emc2_group_slots.restype = ctypes.c_int
    lib.emc2_group_slots.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.emc2_build_inverse_kmap.restype = ctypes.c_int
    lib.emc2_build_inverse_kmap.argtypes = [vp, vp, vp, i64, ctypes.POINTER(i32), i32, i32, vp, vp, vp]
    lib.emc2_bev_flatten.restype = ctypes.c_int
    lib.emc2_bev_flatten.argtypes = [vp, ctypes.c_int, vp, vp, vp, i64, ctypes.POINTER(i32), i32, i32, vp, vp]
    f32 = ctypes.c_float
    lib.emc2_frame_offsets.restype = ctypes.c_int
    lib.emc2_frame_offsets.argtypes = [vp, vp, vp, i64, i32, vp, vp]
    lib.emc2_layernorm.restype = ctypes.c_int
    lib.emc2_layernorm.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, vp, f32, vp, i64, i32, vp, i64, vp, i64, vp]
    lib.emc2_layernorm_work.restype = i64
    lib.emc2_layernorm_work.argtypes = [ctypes.c_int, i64, i32]
    lib.emc2_layernorm_backward.restype = ctypes.c_int
    lib.emc2_layernorm_backward.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i64, vp, f32, vp, i64, i32, vp, i64, vp, vp, vp, i64, vp]
    lib.emc2_recurrence.restype = ctypes.c_int
    lib.emc2_recurrence.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i32, i64, i32, i32, vp, vp, i64, vp, vp, i64, vp]
    lib.emc2_recurrence_work.restype = i64
    lib.emc2_recurrence_work.argtypes = [ctypes.c_int, i64, i32]
    lib.emc2_recurrence_backward.restype = ctypes.c_int
    lib.emc2_recurrence_backward.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i32, i64, i32, i32, vp, vp, i64, vp, vp, i64, vp, i64, vp,
                                             vp, i64, vp]
    lib.emc2_recurrence_step.restype = ctypes.c_int
    lib.emc2_recurrence_step.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i64, i32, vp, vp, i64, vp]
    lib.emc2_ffn_packed_size.restype = i64
    lib.emc2_ffn_packed_size.argtypes = [ctypes.c_int, i32, i32]
    lib.emc2_ffn_pack.restype = ctypes.c_int
    lib.emc2_ffn_pack.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i32, vp, vp]
    lib.emc2_ffn.restype = ctypes.c_int
    lib.emc2_ffn.argtypes = [vp, ctypes.c_int, i32, vp, i64, vp, vp, i64, vp, i64, i32, i32, vp, i64, vp]
    lib.emc2_ffn_work.restype = i64
    lib.emc2_ffn_work.argtypes = [ctypes.c_int, i64, i32, i32]
    lib.emc2_ffn_backward.restype = ctypes.c_int
    lib.emc2_ffn_backward.argtypes = [vp, ctypes.c_int, i32, vp, i64, vp, vp, i64, vp, i64, i32, i32, vp, i64, vp, vp, vp, vp, i64, vp]
    lib.emc2_causal_conv.restype = ctypes.c_int
    lib.emc2_causal_conv.argtypes = [vp, ctypes.c_int, vp, i64, vp, vp, i32, vp, i32, i64, i32, i32, i32, vp, vp, i64, vp, vp]
    lib.emc2_causal_conv_work.restype = i64
    lib.emc2_causal_conv_work.argtypes = [ctypes.c_int, i64, i32, i32]
    lib.emc2_causal_conv_backward.restype = ctypes.c_int
    lib.emc2_causal_conv_backward.argtypes = [vp, ctypes.c_int, vp, i64, vp, vp, i32, vp, i32, i64, i32, i32, i32, vp, vp, i64, vp, vp, i64, vp, vp,
                                              vp, vp, i64, vp]
    lib.emc2_causal_conv_step.restype = ctypes.c_int
    lib.emc2_causal_conv_step.argtypes = [vp, ctypes.c_int, vp, i64, vp, vp, i32, vp, i64, i32, i32, vp, vp, i64, vp]
    lib.emc2_gated_residual.restype = ctypes.c_int
    lib.emc2_gated_residual.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i64, vp, vp, vp, f32, vp, i64, i32, vp, i64, vp, i64, vp]
    lib.emc2_gated_residual_work.restype = i64
    lib.emc2_gated_residual_work.argtypes = [ctypes.c_int, i64, i32]
    lib.emc2_gated_residual_backward.restype = ctypes.c_int
    lib.emc2_gated_residual_backward.argtypes = [vp, ctypes.c_int, vp, i64, vp, i64, vp, i64, vp, vp, vp, f32, vp, i64, vp, i64, vp, i64, i32, vp,
                                                 i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp]
    scan = [vp, ctypes.c_int, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp]
    lib.emc2_selective_scan.restype = ctypes.c_int
    lib.emc2_selective_scan.argtypes = scan + [vp, i32, i64, i32, i32, i32, vp, vp, i64, vp, vp, i64, vp]
    lib.emc2_selective_scan_work.restype = i64
    lib.emc2_selective_scan_work.argtypes = [ctypes.c_int, i64, i32, i32]
    lib.emc2_selective_scan_backward.restype = ctypes.c_int
    lib.emc2_selective_scan_backward.argtypes = scan + [vp, i32, i64, i32, i32, i32, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp,
                                                        vp, i64, vp]
    lib.emc2_selective_scan_step.restype = ctypes.c_int
    lib.emc2_selective_scan_step.argtypes = scan + [vp, i64, i32, i32, vp, vp, i64, vp]
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev_check(t: torch.Tensor, dtype: torch.dtype, name: str) -> None:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous {dtype} device tensor, got {t.dtype} on {t.device}")


_PLACE_TYPE_SHAPE = operator.attrgetter("is_cuda", "dtype", "shape")


def _rows_of(x: torch.Tensor, dtype: int, name: str = "x") -> Tuple[tuple, int, int]:
    """What the rows of a sequence operator must look like (those of its first operand): (place, type, shape), rows, channels."""
    like = _PLACE_TYPE_SHAPE(x)
    if like[:2] != (True, _TORCH_DTYPE[dtype]) or len(like[2]) != 2:
        raise ValueError(f"{name}: need {_TORCH_DTYPE[dtype]} rows [n][channels] on the device, got {x.dtype} {tuple(x.shape)} on {x.device}")
    return like, like[2][0], like[2][1]


def _pitch(t: Optional[torch.Tensor], like: tuple, name: str) -> int:
    """Distance of the rows of `t`: as many as `like` says, any distance apart, channels neighbours."""
    if t is None:
        return 0
    if _PLACE_TYPE_SHAPE(t) != like:
        raise ValueError(f"{name}: need {like[1]} rows {tuple(like[2])} on the device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    ld, step = t.stride()
    n, c = like[2]
    if (step != 1 and c > 1 and n > 0) or (ld < c and n > 1):
        raise ValueError(f"{name}: channels of a row must be neighbours and rows must not overlap, got strides {t.stride()}")
    return ld if ld > c else c


def _params_check(t: Optional[torch.Tensor], dtype: torch.dtype, shape: Tuple[int, ...], name: str) -> None:
    if t is not None and (_PLACE_TYPE_SHAPE(t) != (True, dtype, shape) or not t.is_contiguous()):
        raise ValueError(f"{name}: need a contiguous {dtype} device tensor {tuple(shape)}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _at(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _raw_stream() -> int:
    """torch's current stream, without the object around it."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream_of(dev: int) -> int:
    """The stream of torch that is current on device `dev`."""
    return torch._C._cuda_getCurrentRawStream(dev)


def _shape_of(x: torch.Tensor) -> torch.Size:
    """Shape of the first operand of a call, whose rows the others' are like."""
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"x: need rows [n][channels], got {tuple(shape)}")
    return shape


def _rows_at(dev: int, td: torch.dtype, shape: torch.Size, names: Tuple[str, ...], *rows: Optional[torch.Tensor]) -> list:
    """Pointer and pitch of each operand, one after the other (None and 0: there is none): rows of the one shape and type on device `dev`, any distance apart,
    channels neighbours.  One pass over all of a call's rows: with checks and pointers one by one, issuing a call of a few rows took up to 0.5 us longer."""
    out = []
    for name, t in zip(names, rows):
        if t is None:
            out += (None, 0)
            continue
        if t.shape != shape or t.dtype is not td or t.get_device() != dev:
            raise ValueError(f"{name}: need {td} rows {tuple(shape)} on device {dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        ld, step = t.stride()
        out += (t.data_ptr(), ld if step == 1 and ld >= shape[1] else _pitch(t, (True, td, shape), name))
    return out


def _floats_at(dev: int, *operands: Tuple[Optional[torch.Tensor], Tuple[int, ...], str]) -> list:
    """Pointers of contiguous fp32 operands (tensor, shape, name) on device `dev`."""
    out = []
    for t, shape, name in operands:
        if t is None:
            out.append(None)
            continue
        if t.shape != shape or t.dtype is not torch.float32 or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"{name}: need a contiguous {torch.float32} tensor {tuple(shape)} on device {dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        out.append(t.data_ptr())
    return out


def _ints_at(dev: int, t: Optional[torch.Tensor], name: str) -> Optional[int]:
    """Pointer of a contiguous int32 operand on device `dev` with one value at least."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous() or t.numel() < 1:
        raise ValueError(f"{name}: need a contiguous {torch.int32} tensor on device {dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _count_check(n: Optional[torch.Tensor]) -> None:
    if n is not None:
        _dev_check(n, torch.int32, "n")
        if n.numel() < 1:
            raise ValueError("n: need one count")


def _work_at(dev: int, work: torch.Tensor, need: int) -> Tuple[int, int]:
    """Pointer and bytes of a work buffer on device `dev`."""
    size = _work_check(work, need)
    if work.get_device() != dev:
        raise ValueError(f"work: need a tensor on device {dev}, got {work.device}")
    return work.data_ptr(), size


def _work_check(work: torch.Tensor, need: int) -> int:
    """Bytes of a work buffer; `need`: what the library's query says."""
    if not work.is_cuda or not work.is_contiguous():
        raise ValueError(f"work: need a contiguous device tensor, got {work.device}")
    size = work.numel() * work.element_size()
    if size < need:
        raise ValueError(f"work: {size} bytes, {need} are needed")
    return size


_SHAPE_TYPE_PLACE = operator.attrgetter("shape", "dtype", "is_cuda")


def tensor_keys(tensors: Sequence[Optional[torch.Tensor]]) -> list:
    """What calls are told of tensors, and what the checks here look at: arguments filled from them hold for others with the
    same keys, and for no others.  Attribute by attribute, so that the loops run in C: a pass does this before it launches
    anything."""
    held = [t for t in tensors if t is not None]
    return [[t is None for t in tensors], list(map(torch.Tensor.data_ptr, held)), list(map(_SHAPE_TYPE_PLACE, held)),
            list(map(torch.Tensor.is_contiguous, held))]


STATIC_KMAP_MAX_CELLS = 1 << 24


def build_kmap_static(kind: int, in_coords: torch.Tensor, n_in: torch.Tensor, capacity_in: int, grid_in: Sequence[int],
                      n_batch: int, capacity_out: int, nbr: torch.Tensor, n_out: torch.Tensor,
                      out_coords: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> Tuple[int, int, int]:
    """emc2_build_kmap_static: the kernel map without a context (static device scratch, nothing allocated), on the
    current device and torch's current stream.  Returns the output grid."""
    if not torch.cuda.is_available():
        raise RuntimeError("emc2 needs a GPU: there is no CPU path")
    lib = load_library()
    check_kmap(in_coords, n_in, capacity_in, nbr, n_out, capacity_out, out_coords)
    if status is not None:
        _dev_check(status, torch.int32, "status")
    g_in = (ctypes.c_int32 * 3)(*grid_in)
    g_out = (ctypes.c_int32 * 3)()
    st = lib.emc2_build_kmap_static(kind, _ptr(in_coords), _ptr(n_in), capacity_in, g_in, n_batch, capacity_out,
                                    _ptr(out_coords), _ptr(n_out), _ptr(nbr), g_out, _ptr(status), _stream())
    if st != OK:
        raise Emc2Error(st, lib.emc2_last_error(None).decode())
    return g_out[0], g_out[1], g_out[2]


def check_points(points: torch.Tensor, batch: Optional[torch.Tensor]) -> Tuple[int, int]:
    """(number of points, floats per point) of what is voxelized."""
    _dev_check(points, torch.float32, "points")
    n, stride = (points.shape[0], points.shape[1]) if points.dim() == 2 else (0, 4)
    if batch is not None:
        _dev_check(batch, torch.int32, "batch")
        if batch.numel() != n:
            raise ValueError("batch length != number of points")
    return n, stride


def check_voxels(capacity: int, coords: torch.Tensor, feats: torch.Tensor, counts: torch.Tensor, n_voxels: torch.Tensor,
                 feats_lp: Optional[torch.Tensor]) -> int:
    """What the library cannot see of a voxelization's outputs (devices, types, sizes); returns the type of the copy."""
    _dev_check(coords, torch.int32, "coords")
    _dev_check(feats, torch.float32, "feats")
    _dev_check(counts, torch.int32, "counts")
    _dev_check(n_voxels, torch.int32, "n_voxels")
    if coords.numel() < 4 * capacity or feats.numel() < 4 * capacity or counts.numel() < capacity:
        raise ValueError("output buffers smaller than capacity")
    if feats_lp is None:
        return F16
    lp_dtype = {torch.float16: F16, torch.bfloat16: BF16}[feats_lp.dtype]
    if feats_lp.numel() < 4 * capacity or not feats_lp.is_cuda:
        raise ValueError("feats_lp smaller than capacity")
    return lp_dtype


def check_group_batch(group_batch: torch.Tensor, n_points: int) -> None:
    _dev_check(group_batch, torch.int32, "group_batch")
    if group_batch.numel() != n_points:
        raise ValueError("group_batch length != number of points")


def check_kmap(in_coords: torch.Tensor, n_in: torch.Tensor, capacity_in: int, nbr: torch.Tensor, n_out: torch.Tensor,
               capacity_out: int, out_coords: Optional[torch.Tensor]) -> None:
    """What the library cannot see of a kernel map's arguments."""
    _dev_check(in_coords, torch.int32, "in_coords")
    _dev_check(n_in, torch.int32, "n_in")
    _dev_check(nbr, torch.int32, "nbr")
    _dev_check(n_out, torch.int32, "n_out")
    if in_coords.numel() < 4 * capacity_in or nbr.numel() < 27 * capacity_out:
        raise ValueError("buffers smaller than capacity")
    if out_coords is not None:
        _dev_check(out_coords, torch.int32, "out_coords")
        if out_coords.numel() < 4 * capacity_out:
            raise ValueError("out_coords smaller than capacity_out")


def check_conv(dtype: int, x: torch.Tensor, w: torch.Tensor, scale: Optional[torch.Tensor], shift: Optional[torch.Tensor],
               nbr: torch.Tensor, n_out: torch.Tensor, capacity_out: int, out: torch.Tensor) -> Tuple[int, int]:
    """What emc2_spconv cannot see of its arguments (devices, types, sizes); returns (Cin, Cout)."""
    td = _TORCH_DTYPE[dtype]
    _dev_check(x, td, "x")
    _dev_check(w, td, "w")
    _dev_check(out, td, "out")
    _dev_check(nbr, torch.int32, "nbr")
    _dev_check(n_out, torch.int32, "n_out")
    if w.dim() != 3 or w.shape[0] != 27 or x.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("w must be [27][Cin][Cout] and x [n][Cin]")
    cin, cout = int(w.shape[1]), int(w.shape[2])
    if out.numel() < capacity_out * cout or nbr.numel() < 27 * capacity_out:
        raise ValueError("out / nbr smaller than capacity_out")
    if scale is not None:
        _dev_check(scale, torch.float32, "scale")
        _dev_check(shift, torch.float32, "shift")
        if scale.numel() != cout or shift.numel() != cout:
            raise ValueError("scale/shift must have Cout entries")
    return cin, cout


def _why(lib: ctypes.CDLL, ctx: Optional[int]) -> str:
    """What a call that takes several contexts says went wrong: kept with the first of them."""
    return lib.emc2_last_error(ctx).decode() if ctx else "the context is closed"


def build_stacks(stacks, n_stacks: int, points: torch.Tensor) -> None:
    """emc2_build_stacks over a ctypes array of StackC whose buffers and frame ids the caller has checked and keeps alive."""
    n, stride = check_points(points, None)
    for i in range(n_stacks):
        stacks[i].spec.stride_f = stride
    lib = load_library()
    st = lib.emc2_build_stacks(stacks, n_stacks, points.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    if st != OK:
        raise Emc2Error(st, _why(lib, stacks[0].ctx))


def spconv_list(calls, n: int) -> None:
    """emc2_spconv_list over a ctypes array of ConvCallC whose buffers the caller keeps alive."""
    lib = load_library()
    st = lib.emc2_spconv_list(calls, n, torch.cuda.current_stream().cuda_stream)
    if st != OK:
        raise Emc2Error(st, _why(lib, calls[0].ctx))


class Context:
    """Owns the library's scratch on one GPU (see emc2_create)."""

    def __init__(self, max_points: int, max_voxels: int, max_cells: int, n_slots: int = 4, device: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("emc2 needs a GPU: there is no CPU path")
        self.lib = load_library()
        self.device = device
        h = ctypes.c_void_p()
        st = self.lib.emc2_create(ctypes.byref(h), device, max_points, max_voxels, max_cells, n_slots)
        if st != OK:
            raise Emc2Error(st, "emc2_create failed")
        self.h = h
        self.max_voxels = max_voxels

    def close(self) -> None:
        if getattr(self, "h", None):
            self.lib.emc2_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, st: int) -> None:
        if st != OK:
            raise Emc2Error(st, self.lib.emc2_last_error(self.h).decode())

    def status_sync(self) -> None:
        self._chk(self.lib.emc2_status_sync(self.h, _stream()))

    # ------------------------------------------------------------------------------------------
    def voxelize(self, points: torch.Tensor, batch: Optional[torch.Tensor], spec: VoxelSpec, capacity: int,
                 coords: torch.Tensor, feats: torch.Tensor, counts: torch.Tensor, n_voxels: torch.Tensor,
                 feats_lp: Optional[torch.Tensor] = None, index_slot: int = 0, sync_count: bool = False) -> Optional[int]:
        n, stride = check_points(points, batch)
        lp_dtype = check_voxels(capacity, coords, feats, counts, n_voxels, feats_lp)
        cs = voxel_spec_c(spec, stride)
        h_n = ctypes.c_int32(0)
        self._chk(self.lib.emc2_voxelize(self.h, _ptr(points), _ptr(batch), n, ctypes.byref(cs), capacity, _ptr(coords),
                                         _ptr(feats), _ptr(counts), _ptr(feats_lp), lp_dtype, _ptr(n_voxels),
                                         ctypes.byref(h_n) if sync_count else None, index_slot, _stream()))
        return int(h_n.value) if sync_count else None

    def build_kmap(self, kind: int, in_coords: torch.Tensor, n_in: torch.Tensor, capacity_in: int, grid_in: Sequence[int],
                   n_batch: int, capacity_out: int, nbr: torch.Tensor, n_out: torch.Tensor,
                   out_coords: Optional[torch.Tensor] = None, in_slot: int = -1, out_slot: int = -1,
                   sync_count: bool = False) -> Tuple[Tuple[int, int, int], Optional[int]]:
        check_kmap(in_coords, n_in, capacity_in, nbr, n_out, capacity_out, out_coords)
        g_in = (ctypes.c_int32 * 3)(*grid_in)
        g_out = (ctypes.c_int32 * 3)()
        h_n = ctypes.c_int32(0)
        self._chk(self.lib.emc2_build_kmap(self.h, kind, _ptr(in_coords), _ptr(n_in), capacity_in, g_in, n_batch, in_slot,
                                           out_slot, capacity_out, _ptr(out_coords), _ptr(n_out), _ptr(nbr), g_out,
                                           ctypes.byref(h_n) if sync_count else None, _stream()))
        return (g_out[0], g_out[1], g_out[2]), (int(h_n.value) if sync_count else None)

    def build_inverse_kmap(self, fine_coords: torch.Tensor, n_fine: torch.Tensor, capacity_fine: int,
                           grid_coarse: Sequence[int], n_batch: int, coarse_slot: int, n_coarse: torch.Tensor,
                           nbr: torch.Tensor) -> None:
        """Gather table of the transposed stride-2 conv: nbr[27][capacity_fine] over the fine sites."""
        _dev_check(fine_coords, torch.int32, "fine_coords")
        _dev_check(n_fine, torch.int32, "n_fine")
        _dev_check(n_coarse, torch.int32, "n_coarse")
        _dev_check(nbr, torch.int32, "nbr")
        if fine_coords.numel() < 4 * capacity_fine or nbr.numel() < 27 * capacity_fine:
            raise ValueError("buffers smaller than capacity_fine")
        g = (ctypes.c_int32 * 3)(*grid_coarse)
        self._chk(self.lib.emc2_build_inverse_kmap(self.h, _ptr(fine_coords), _ptr(n_fine), capacity_fine, g, n_batch,
                                                   coarse_slot, _ptr(n_coarse), _ptr(nbr), _stream()))

    def bev_flatten(self, dtype: int, coords: torch.Tensor, feats: torch.Tensor, n: torch.Tensor, capacity: int,
                    grid: Sequence[int], n_batch: int, out: torch.Tensor) -> None:
        """out[B][Gy][Gx][Gz*C] <- feats[v][C] at (b, z, y, x) = coords[v], zero elsewhere."""
        td = _TORCH_DTYPE[dtype]
        _dev_check(coords, torch.int32, "coords")
        _dev_check(feats, td, "feats")
        _dev_check(out, td, "out")
        _dev_check(n, torch.int32, "n")
        c = int(feats.shape[1])
        if coords.numel() < 4 * capacity or feats.numel() < capacity * c:
            raise ValueError("coords / feats smaller than capacity")
        if out.numel() != n_batch * grid[0] * grid[1] * grid[2] * c:
            raise ValueError("out must be [n_batch][Gy][Gx][Gz*C]")
        g = (ctypes.c_int32 * 3)(*grid)
        self._chk(self.lib.emc2_bev_flatten(self.h, dtype, _ptr(coords), _ptr(feats), _ptr(n), capacity, g, n_batch, c,
                                            _ptr(out), _stream()))

    def pool_image(self, img: torch.Tensor, depth: torch.Tensor, qmat: Sequence[float], spec: VoxelSpec, mode: int,
                   capacity: int, coords: torch.Tensor, feats: torch.Tensor, counts: torch.Tensor, n_cells: torch.Tensor,
                   batch_index: int = 0, index_slot: int = 0, sync_count: bool = False) -> Optional[int]:
        """img[H][W][C] f16 + depth[H][W] f32 -> pooled cells (coords, feats[cap][C] f16, counts) on spec's grid."""
        _dev_check(img, torch.float16, "img")
        _dev_check(depth, torch.float32, "depth")
        _dev_check(coords, torch.int32, "coords")
        _dev_check(feats, torch.float16, "feats")
        _dev_check(counts, torch.int32, "counts")
        _dev_check(n_cells, torch.int32, "n_cells")
        if img.dim() != 3 or tuple(depth.shape) != tuple(img.shape[:2]):
            raise ValueError("img must be [H][W][C] and depth [H][W]")
        h, w, c = (int(v) for v in img.shape)
        if coords.numel() < 4 * capacity or feats.numel() < capacity * c or counts.numel() < capacity:
            raise ValueError("output buffers smaller than capacity")
        q = (ctypes.c_float * 12)(*[float(v) for v in qmat])
        cs = _VoxelSpecC((ctypes.c_float * 3)(*spec.lo), (ctypes.c_float * 3)(*spec.vs), (ctypes.c_int32 * 3)(*spec.grid),
                         spec.n_batch, 0.0, float("inf"), 4)
        h_n = ctypes.c_int32(0)
        self._chk(self.lib.emc2_pool_image(self.h, _ptr(img), _ptr(depth), h, w, c, q, ctypes.byref(cs), batch_index, mode,
                                           capacity, _ptr(coords), _ptr(feats), _ptr(counts), _ptr(n_cells),
                                           ctypes.byref(h_n) if sync_count else None, index_slot, _stream()))
        return int(h_n.value) if sync_count else None

    def fuse(self, dtype: int, coords_l: torch.Tensor, feats_l: torch.Tensor, n_l: torch.Tensor, capacity_l: int,
             coords_i: torch.Tensor, feats_i: torch.Tensor, n_i: torch.Tensor, capacity_i: int, grid: Sequence[int],
             n_batch: int, capacity_out: int, coords_out: torch.Tensor, feats_out: torch.Tensor, n_out: torch.Tensor,
             src_l: Optional[torch.Tensor] = None, src_i: Optional[torch.Tensor] = None, out_slot: int = 0,
             sync_count: bool = False) -> Optional[int]:
        """Union of the LiDAR voxels and the image cells, rows [LiDAR | image | zero padding up to feats_out's width]."""
        td = _TORCH_DTYPE[dtype]
        for t, nm in ((coords_l, "coords_l"), (coords_i, "coords_i"), (coords_out, "coords_out"), (n_l, "n_l"), (n_i, "n_i"),
                      (n_out, "n_out")):
            _dev_check(t, torch.int32, nm)
        for t, nm in ((feats_l, "feats_l"), (feats_i, "feats_i"), (feats_out, "feats_out")):
            _dev_check(t, td, nm)
        c_l, c_i, c_out = int(feats_l.shape[1]), int(feats_i.shape[1]), int(feats_out.shape[1])
        if coords_l.numel() < 4 * capacity_l or feats_l.numel() < capacity_l * c_l:
            raise ValueError("LiDAR buffers smaller than capacity_l")
        if coords_i.numel() < 4 * capacity_i or feats_i.numel() < capacity_i * c_i:
            raise ValueError("image buffers smaller than capacity_i")
        if coords_out.numel() < 4 * capacity_out or feats_out.numel() < capacity_out * c_out:
            raise ValueError("output buffers smaller than capacity_out")
        for t, nm in ((src_l, "src_l"), (src_i, "src_i")):
            if t is not None:
                _dev_check(t, torch.int32, nm)
                if t.numel() < capacity_out:
                    raise ValueError(f"{nm} smaller than capacity_out")
        g = (ctypes.c_int32 * 3)(*grid)
        h_n = ctypes.c_int32(0)
        self._chk(self.lib.emc2_fuse(self.h, dtype, _ptr(coords_l), _ptr(feats_l), _ptr(n_l), capacity_l, c_l, _ptr(coords_i),
                                     _ptr(feats_i), _ptr(n_i), capacity_i, c_i, g, n_batch, out_slot, capacity_out, c_out,
                                     _ptr(coords_out), _ptr(feats_out), _ptr(src_l), _ptr(src_i), _ptr(n_out),
                                     ctypes.byref(h_n) if sync_count else None, _stream()))
        return int(h_n.value) if sync_count else None

    def dispatch(self, props: torch.Tensor, scene: Optional[torch.Tensor], n_scenes: int, dist: float, conf: float,
                 expert: torch.Tensor, counts: torch.Tensor, order: torch.Tensor) -> None:
        """props[N][4] f32 (x, y, z, confidence), scene[N] i32 -> expert[S], counts[3], order[S] (scenes grouped by expert)."""
        _dev_check(props, torch.float32, "props")
        for t, nm in ((expert, "expert"), (counts, "counts"), (order, "order")):
            _dev_check(t, torch.int32, nm)
        n = int(props.shape[0]) if props.dim() == 2 else 0
        if props.dim() != 2 or props.shape[1] != 4:
            raise ValueError("props must be [N][4]")
        if scene is not None:
            _dev_check(scene, torch.int32, "scene")
            if scene.numel() != n:
                raise ValueError("scene length != number of proposals")
        if expert.numel() < n_scenes or order.numel() < n_scenes or counts.numel() < 3:
            raise ValueError("output buffers too small")
        self._chk(self.lib.emc2_dispatch(self.h, _ptr(props), _ptr(scene), n, n_scenes, dist, conf, _ptr(expert),
                                         _ptr(counts), _ptr(order), _stream()))

    def spconv_i8_supported(self, cin: int, cout: int) -> bool:
        return bool(self.lib.emc2_spconv_i8_supported(cin, cout))

    def quantize_i8(self, x: torch.Tensor, inv_scale: float, q: torch.Tensor) -> None:
        """q = clamp(rint(x * inv_scale), -127, 127) for an F32 or F16 tensor x."""
        dt = {torch.float32: F32, torch.float16: F16}[x.dtype]
        _dev_check(x, x.dtype, "x")
        _dev_check(q, torch.int8, "q")
        if q.numel() < x.numel():
            raise ValueError("q smaller than x")
        self._chk(self.lib.emc2_quantize_i8(self.h, dt, _ptr(x), x.numel(), inv_scale, _ptr(q), _stream()))

    def pack_weights_i8(self, w: torch.Tensor, packed: torch.Tensor) -> None:
        """w [27][Cin][Cout] int8 -> packed (same size) in the int8 matrix-core fragment order."""
        _dev_check(w, torch.int8, "w")
        _dev_check(packed, torch.int8, "packed")
        if w.dim() != 3 or w.shape[0] != 27 or packed.numel() != w.numel():
            raise ValueError("w must be [27][Cin][Cout] and packed the same size")
        self._chk(self.lib.emc2_pack_weights_i8(self.h, _ptr(w), int(w.shape[1]), int(w.shape[2]), _ptr(packed), _stream()))

    def spconv_i8(self, x: torch.Tensor, w_packed: torch.Tensor, cin: int, cout: int, mul: torch.Tensor, add: torch.Tensor,
                  relu: bool, nbr: torch.Tensor, n_out: torch.Tensor, capacity_out: int, out: torch.Tensor,
                  inv_out_scale: float = 0.0, n_in_rows: Optional[int] = None) -> None:
        """Quantised conv: x [n][Cin] int8, packed int8 weights, out [cap][Cout] int8 (re-quantised) or float16.
        n_in_rows: rows of x a map entry may name (default: all rows of the tensor)."""
        _dev_check(x, torch.int8, "x")
        _dev_check(w_packed, torch.int8, "w_packed")
        _dev_check(mul, torch.float32, "mul")
        _dev_check(add, torch.float32, "add")
        _dev_check(nbr, torch.int32, "nbr")
        _dev_check(n_out, torch.int32, "n_out")
        if out.dtype not in (torch.int8, torch.float16) or not out.is_cuda or not out.is_contiguous():
            raise ValueError("out must be a contiguous int8 or float16 device tensor")
        if x.dim() != 2 or x.shape[1] != cin or w_packed.numel() != 27 * cin * cout or mul.numel() != cout or add.numel() != cout:
            raise ValueError("shape mismatch")
        if out.numel() < capacity_out * cout or nbr.numel() < 27 * capacity_out:
            raise ValueError("out / nbr smaller than capacity_out")
        self._chk(self.lib.emc2_spconv_i8(self.h, _ptr(x), _ptr(w_packed), _ptr(mul), _ptr(add), int(bool(relu)),
                                          I8 if out.dtype == torch.int8 else F16, inv_out_scale, _ptr(nbr), _ptr(n_out),
                                          capacity_out, int(x.shape[0]) if n_in_rows is None else n_in_rows, cin, cout,
                                          _ptr(out), _stream()))

    def quantize_e4m3(self, x: torch.Tensor, inv_scale: float, q: torch.Tensor) -> None:
        """q[i] = E4M3 code (uint8) nearest to x[i] * inv_scale; x float32 or float16."""
        if x.dtype not in (torch.float32, torch.float16) or not x.is_cuda or not x.is_contiguous():
            raise ValueError("x must be a contiguous float32 or float16 device tensor")
        _dev_check(q, torch.uint8, "q")
        if q.numel() != x.numel():
            raise ValueError("q and x differ in size")
        self._chk(self.lib.emc2_quantize_e4m3(self.h, F32 if x.dtype == torch.float32 else F16, _ptr(x), x.numel(),
                                              inv_scale, _ptr(q), _stream()))

    def spconv_e4m3(self, x: torch.Tensor, w_packed: torch.Tensor, cin: int, cout: int, mul: torch.Tensor, add: torch.Tensor,
                    relu: bool, nbr: torch.Tensor, n_out: torch.Tensor, capacity_out: int, out: torch.Tensor,
                    n_in_rows: Optional[int] = None) -> None:
        """E4M3 conv: x [n][Cin] uint8 codes, weights packed by pack_weights_i8 (as bytes), out float32 or float16."""
        _dev_check(x, torch.uint8, "x")
        _dev_check(mul, torch.float32, "mul")
        _dev_check(add, torch.float32, "add")
        _dev_check(nbr, torch.int32, "nbr")
        _dev_check(n_out, torch.int32, "n_out")
        if w_packed.dtype not in (torch.uint8, torch.int8) or not w_packed.is_cuda or not w_packed.is_contiguous():
            raise ValueError("w_packed must be a contiguous 8-bit device tensor")
        if out.dtype not in (torch.float32, torch.float16) or not out.is_cuda or not out.is_contiguous():
            raise ValueError("out must be a contiguous float32 or float16 device tensor")
        if x.dim() != 2 or x.shape[1] != cin or w_packed.numel() != 27 * cin * cout or mul.numel() != cout or add.numel() != cout:
            raise ValueError("shape mismatch")
        if out.numel() < capacity_out * cout or nbr.numel() < 27 * capacity_out:
            raise ValueError("out / nbr smaller than capacity_out")
        self._chk(self.lib.emc2_spconv_e4m3(self.h, _ptr(x), _ptr(w_packed), _ptr(mul), _ptr(add), int(bool(relu)),
                                            F32 if out.dtype == torch.float32 else F16, _ptr(nbr), _ptr(n_out), capacity_out,
                                            int(x.shape[0]) if n_in_rows is None else n_in_rows, cin, cout, _ptr(out), _stream()))

    def uses_mfma(self, dtype: int, cin: int, cout: int) -> bool:
        return bool(self.lib.emc2_spconv_uses_mfma(dtype, cin, cout))

    def pack_weights(self, dtype: int, w: torch.Tensor, packed: torch.Tensor) -> None:
        """w [27][Cin][Cout] -> packed (same shape/dtype buffer) in MFMA fragment order."""
        td = _TORCH_DTYPE[dtype]
        _dev_check(w, td, "w")
        _dev_check(packed, td, "packed")
        if w.dim() != 3 or w.shape[0] != 27 or packed.numel() != w.numel():
            raise ValueError("w must be [27][Cin][Cout] and packed the same size")
        self._chk(self.lib.emc2_pack_weights(self.h, dtype, _ptr(w), int(w.shape[1]), int(w.shape[2]), _ptr(packed),
                                             _stream()))

    def spconv_kernel(self, dtype: int, cin: int, cout: int, map_hint: int = MAP_ANY) -> str:
        """Name of the device kernel `spconv` launches for these arguments (for matching profiles to layers)."""
        return self.lib.emc2_spconv_kernel(dtype, cin, cout, map_hint).decode()

    def spconv(self, dtype: int, x: torch.Tensor, w: torch.Tensor, scale: Optional[torch.Tensor],
               shift: Optional[torch.Tensor], epilogue: int, nbr: torch.Tensor, n_out: torch.Tensor, capacity_out: int,
               out: torch.Tensor, w_layout: int = W_PLAIN, map_hint: int = MAP_ANY, n_in_rows: Optional[int] = None) -> None:
        """n_in_rows: rows of x a map entry may name (default: all rows of the tensor)."""
        cin, cout = check_conv(dtype, x, w, scale, shift, nbr, n_out, capacity_out, out)
        self._chk(self.lib.emc2_spconv(self.h, dtype, _ptr(x), _ptr(w), w_layout, _ptr(scale), _ptr(shift), epilogue, _ptr(nbr),
                                       map_hint, _ptr(n_out), capacity_out,
                                       int(x.shape[0]) if n_in_rows is None else n_in_rows, cin, cout, _ptr(out), _stream()))

    def group_points(self, scene: Optional[torch.Tensor], n_points: int, expert: torch.Tensor, order: torch.Tensor,
                     counts: torch.Tensor, n_scenes: int, e: int, slot: torch.Tensor, group_batch: torch.Tensor) -> None:
        """Dispatcher outputs -> slot[n_scenes] and, for expert e, group_batch[n_points] (-1 for other experts' points)."""
        for t, nm in ((expert, "expert"), (order, "order"), (counts, "counts"), (slot, "slot"), (group_batch, "group_batch")):
            _dev_check(t, torch.int32, nm)
        if scene is not None:
            _dev_check(scene, torch.int32, "scene")
            if scene.numel() != n_points:
                raise ValueError("scene length != n_points")
        if expert.numel() < n_scenes or order.numel() < n_scenes or counts.numel() < 3 or slot.numel() < n_scenes or \
                group_batch.numel() < n_points:
            raise ValueError("buffers smaller than n_scenes / n_points")
        self._chk(self.lib.emc2_group_points(self.h, _ptr(scene), n_points, _ptr(expert), _ptr(order), _ptr(counts), n_scenes,
                                             e, _ptr(slot), _ptr(group_batch), _stream()))

    def group_slots(self, expert: torch.Tensor, order: torch.Tensor, counts: torch.Tensor, n_scenes: int, slot: torch.Tensor) -> None:
        """Dispatcher outputs -> slot[n_scenes]: each scene's position in its expert's group (group_points without batch ids)."""
        for t, nm in ((expert, "expert"), (order, "order"), (counts, "counts"), (slot, "slot")):
            _dev_check(t, torch.int32, nm)
        if expert.numel() < n_scenes or order.numel() < n_scenes or counts.numel() < 3 or slot.numel() < n_scenes:
            raise ValueError("buffers smaller than n_scenes")
        self._chk(self.lib.emc2_group_slots(self.h, _ptr(expert), _ptr(order), _ptr(counts), n_scenes, _ptr(slot), _stream()))

    def project_gather(self, points: torch.Tensor, pmat: Sequence[float], img: torch.Tensor, out: torch.Tensor,
                       valid: torch.Tensor, uv: Optional[torch.Tensor] = None) -> None:
        _dev_check(points, torch.float32, "points")
        _dev_check(img, torch.float16, "img")
        _dev_check(out, torch.float16, "out")
        _dev_check(valid, torch.uint8, "valid")
        n, stride = points.shape
        h, w, c = img.shape
        if out.numel() < n * c or valid.numel() < n:
            raise ValueError("out / valid too small")
        if uv is not None:
            _dev_check(uv, torch.float32, "uv")
            if uv.numel() < 2 * n:
                raise ValueError("uv too small")
        pm = (ctypes.c_float * 12)(*[float(v) for v in pmat])
        self._chk(self.lib.emc2_project_gather(self.h, _ptr(points), stride, n, pm, _ptr(img), h, w, c, _ptr(out),
                                               _ptr(valid), _ptr(uv), _stream()))

    # ------------------------------------------------------------------------------------------
    # sequence operators: rows [n][channels], any distance apart, of packed frames
    def frame_offsets(self, coords: torch.Tensor, n: Optional[torch.Tensor], capacity: int, n_batch: int, offsets: torch.Tensor) -> None:
        """offsets[n_batch + 1] = first row of every frame of a voxel list, and the number of rows."""
        _dev_check(coords, torch.int32, "coords")
        _dev_check(offsets, torch.int32, "offsets")
        _count_check(n)
        if coords.numel() < 4 * capacity or offsets.numel() < n_batch + 1:
            raise ValueError("coords smaller than capacity or offsets smaller than n_batch + 1")
        self._chk(self.lib.emc2_frame_offsets(self.h, _ptr(coords), _ptr(n), capacity, n_batch, _ptr(offsets), _stream()))

    def layernorm(self, dtype: int, x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float, y: torch.Tensor,
                  residual: Optional[torch.Tensor] = None, total: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None) -> None:
        """y = layer norm of x (+ residual, the sum going to `total` if it is given); n: device count of the rows present."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(residual, like, "residual"), _pitch(total, like, "total"), _pitch(y, like, "y")
        _params_check(gamma, torch.float32, (c,), "gamma")
        _params_check(beta, torch.float32, (c,), "beta")
        _count_check(n)
        self._chk(self.lib.emc2_layernorm(self.h, dtype, _at(x), ld[0], _at(residual), ld[1], _at(gamma), _at(beta), eps, _at(n), rows, c,
                                          _at(total), ld[2], _at(y), ld[3], _raw_stream()))

    def layernorm_work(self, dtype: int, capacity: int, channels: int) -> int:
        return self.lib.emc2_layernorm_work(dtype, capacity, channels)

    def layernorm_backward(self, dtype: int, x: torch.Tensor, gamma: torch.Tensor, eps: float, dy: torch.Tensor, dx: torch.Tensor,
                           dgamma: torch.Tensor, dbeta: torch.Tensor, work: torch.Tensor, add: Optional[torch.Tensor] = None,
                           n: Optional[torch.Tensor] = None) -> None:
        """dx (+ add), dgamma, dbeta of a layer norm of x for dy."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(dy, like, "dy"), _pitch(add, like, "add"), _pitch(dx, like, "dx")
        for t, nm in ((gamma, "gamma"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            _params_check(t, torch.float32, (c,), nm)
        _count_check(n)
        size = _work_check(work, self.lib.emc2_layernorm_work(dtype, rows, c))
        self._chk(self.lib.emc2_layernorm_backward(self.h, dtype, _at(x), ld[0], _at(dy), ld[1], _at(add), ld[2], _at(gamma), eps, _at(n),
                                                   rows, c, _at(dx), ld[3], _at(dgamma), _at(dbeta), _at(work), size, _raw_stream()))

    def recurrence_work(self, dtype: int, capacity: int, channels: int) -> int:
        return self.lib.emc2_recurrence_work(dtype, capacity, channels)

    def recurrence(self, dtype: int, x: torch.Tensor, gate: torch.Tensor, offsets: torch.Tensor, y: torch.Tensor, work: torch.Tensor,
                   backwards: bool = False, h0: Optional[torch.Tensor] = None, last: Optional[torch.Tensor] = None) -> None:
        """y_t = h_t = a_t h_{t-1} + (1 - a_t) x_t along every sequence, a = sigmoid(gate); offsets [sequences + 1] device int32.
        `last` must not overlap h0."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(gate, like, "gate"), _pitch(y, like, "y")
        _dev_check(offsets, torch.int32, "offsets")
        n_seq = offsets.numel() - 1
        _params_check(h0, torch.float32, (n_seq, c), "h0")
        _params_check(last, torch.float32, (n_seq, c), "last")
        size = _work_check(work, self.lib.emc2_recurrence_work(dtype, rows, c))
        self._chk(self.lib.emc2_recurrence(self.h, dtype, _at(x), ld[0], _at(gate), ld[1], _at(offsets), n_seq, rows, c,
                                           int(bool(backwards)), _at(h0), _at(y), ld[2], _at(last), _at(work), size, _raw_stream()))

    def recurrence_backward(self, dtype: int, x: torch.Tensor, gate: torch.Tensor, offsets: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor,
                            dgate: torch.Tensor, work: torch.Tensor, backwards: bool = False, h0: Optional[torch.Tensor] = None,
                            dlast: Optional[torch.Tensor] = None, dh0: Optional[torch.Tensor] = None) -> None:
        """dx, dgate and dh0 of a recurrence over x and gate, for dy and the gradient of the last states; dh0 must not overlap dlast."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(gate, like, "gate"), _pitch(dy, like, "dy"), _pitch(dx, like, "dx"), _pitch(dgate, like, "dgate")
        _dev_check(offsets, torch.int32, "offsets")
        n_seq = offsets.numel() - 1
        for t, nm in ((h0, "h0"), (dlast, "dlast"), (dh0, "dh0")):
            _params_check(t, torch.float32, (n_seq, c), nm)
        size = _work_check(work, self.lib.emc2_recurrence_work(dtype, rows, c))
        self._chk(self.lib.emc2_recurrence_backward(self.h, dtype, _at(x), ld[0], _at(gate), ld[1], _at(offsets), n_seq, rows, c,
                                                    int(bool(backwards)), _at(h0), _at(dy), ld[2], _at(dlast), _at(dx), ld[3], _at(dgate),
                                                    ld[4], _at(dh0), _at(work), size, _raw_stream()))

    def recurrence_step(self, dtype: int, x: torch.Tensor, gate: torch.Tensor, h: torch.Tensor, h_out: torch.Tensor, y: torch.Tensor) -> None:
        """One row per sequence: h_out = a h + (1 - a) x (h_out may be h), y the same rounded."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(gate, like, "gate"), _pitch(y, like, "y")
        _params_check(h, torch.float32, (rows, c), "h")
        _params_check(h_out, torch.float32, (rows, c), "h_out")
        self._chk(self.lib.emc2_recurrence_step(self.h, dtype, _at(x), ld[0], _at(gate), ld[1], _at(h), rows, c, _at(h_out), _at(y),
                                                ld[2], _raw_stream()))

    def ffn_packed_size(self, dtype: int, channels: int, hidden: int) -> int:
        """Values of the packed weights of a gated feed-forward network."""
        return self.lib.emc2_ffn_packed_size(dtype, channels, hidden)

    def ffn_pack(self, dtype: int, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor, packed: torch.Tensor) -> None:
        """wg, wu [channels][hidden], wd [hidden][channels] -> packed, in matrix-core fragment order."""
        td, (c, f) = _TORCH_DTYPE[dtype], tuple(wg.shape)
        for t, shape, nm in ((wg, (c, f), "wg"), (wu, (c, f), "wu"), (wd, (f, c), "wd")):
            _params_check(t, td, shape, nm)
        self._packed_check(packed, dtype, c, f)
        self._chk(self.lib.emc2_ffn_pack(self.h, dtype, _at(wg), _at(wu), _at(wd), c, f, _at(packed), _raw_stream()))

    def _packed_check(self, packed: torch.Tensor, dtype: int, c: int, f: int) -> None:
        _dev_check(packed, _TORCH_DTYPE[dtype], "packed")
        if packed.numel() < self.lib.emc2_ffn_packed_size(dtype, c, f):
            raise ValueError("packed: smaller than ffn_packed_size")

    def ffn(self, dtype: int, activation: int, x: torch.Tensor, packed: torch.Tensor, hidden: int, y: torch.Tensor,
            residual: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None) -> None:
        """y = (act(x wg) * (x wu)) wd (+ residual); packed: ffn_pack's; n: device count of the rows present."""
        like, rows, c = _rows_of(x, dtype)
        ld = _pitch(x, like, "x"), _pitch(residual, like, "residual"), _pitch(y, like, "y")
        _count_check(n)
        self._packed_check(packed, dtype, c, hidden)
        self._chk(self.lib.emc2_ffn(self.h, dtype, activation, _at(x), ld[0], _at(packed), _at(residual), ld[1], _at(n), rows, c,
                                    hidden, _at(y), ld[2], _raw_stream()))

    def ffn_work(self, dtype: int, capacity: int, channels: int, hidden: int) -> int:
        return self.lib.emc2_ffn_work(dtype, capacity, channels, hidden)

    def ffn_backward(self, dtype: int, activation: int, x: torch.Tensor, packed: torch.Tensor, hidden: int, dy: torch.Tensor, dx: torch.Tensor,
                     dwg: torch.Tensor, dwu: torch.Tensor, dwd: torch.Tensor, work: torch.Tensor, n: Optional[torch.Tensor] = None) -> None:
        """dx and the weights' gradients of ffn for dy."""
        like, rows, c = _rows_of(x, dtype)
        td = like[1]
        ld = _pitch(x, like, "x"), _pitch(dy, like, "dy"), _pitch(dx, like, "dx")
        for t, shape, nm in ((dwg, (c, hidden), "dwg"), (dwu, (c, hidden), "dwu"), (dwd, (hidden, c), "dwd")):
            _params_check(t, td, shape, nm)
        _count_check(n)
        self._packed_check(packed, dtype, c, hidden)
        size = _work_check(work, self.lib.emc2_ffn_work(dtype, rows, c, hidden))
        self._chk(self.lib.emc2_ffn_backward(self.h, dtype, activation, _at(x), ld[0], _at(packed), _at(dy), ld[1], _at(n), rows, c, hidden,
                                             _at(dx), ld[2], _at(dwg), _at(dwu), _at(dwd), _at(work), size, _raw_stream()))

    def causal_conv(self, dtype: int, x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, y: torch.Tensor, bias: Optional[torch.Tensor] = None,
                    silu: bool = True, backwards: bool = False, before: Optional[torch.Tensor] = None, last: Optional[torch.Tensor] = None) -> None:
        """y_t = silu(bias + sum of w[k] x_{t-k}) along every sequence; w [taps][channels]; before and last [sequences][taps - 1][channels]: the rows
        before each sequence's first and the last ones behind it, oldest first.  y must not overlap x, nor last before."""
        dev, shape = self._current(), _shape_of(x)
        rows, c = shape
        xp, ld_x, yp, ld_y = _rows_at(dev, _TORCH_DTYPE[dtype], shape, ("x", "y"), x, y)
        at, taps, n_seq = _ints_at(dev, offsets, "offsets"), w.shape[0] if w.dim() == 2 else 0, offsets.numel() - 1
        kept = (n_seq, taps - 1, c)
        wp, bp, fp, lp = _floats_at(dev, (w, (taps, c), "w"), (bias, (c,), "bias"), (before, kept, "before"), (last, kept, "last"))
        self._chk(self.lib.emc2_causal_conv(self.h, dtype, xp, ld_x, wp, bp, bool(silu), at, n_seq, rows, c, taps, bool(backwards), fp, yp, ld_y, lp,
                                            _stream_of(dev)))

    def _current(self) -> int:
        """The current device, which has to be the context's."""
        dev = torch._C._cuda_getDevice()
        if dev != self.device:
            raise ValueError(f"the context's device is {self.device}, the current one {dev}")
        return dev

    def causal_conv_work(self, dtype: int, capacity: int, channels: int, taps: int) -> int:
        return self.lib.emc2_causal_conv_work(dtype, capacity, channels, taps)

    def causal_conv_backward(self, dtype: int, x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor,
                             dw: torch.Tensor, work: torch.Tensor, bias: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             silu: bool = True, backwards: bool = False, before: Optional[torch.Tensor] = None,
                             dlast: Optional[torch.Tensor] = None, dbefore: Optional[torch.Tensor] = None) -> None:
        """dx, dw, dbias and dbefore of a causal_conv of x for dy and the gradient of the rows kept; dx must not overlap x or dy."""
        dev, shape = self._current(), _shape_of(x)
        rows, c = shape
        xp, ld_x, dyp, ld_dy, dxp, ld_dx = _rows_at(dev, _TORCH_DTYPE[dtype], shape, ("x", "dy", "dx"), x, dy, dx)
        at, taps, n_seq = _ints_at(dev, offsets, "offsets"), w.shape[0] if w.dim() == 2 else 0, offsets.numel() - 1
        kept = (n_seq, taps - 1, c)
        wp, bp, fp, dlp, dwp, dbp, dfp = _floats_at(dev, (w, (taps, c), "w"), (bias, (c,), "bias"), (before, kept, "before"), (dlast, kept, "dlast"),
                                                    (dw, (taps, c), "dw"), (dbias, (c,), "dbias"), (dbefore, kept, "dbefore"))
        wk, size = _work_at(dev, work, self.lib.emc2_causal_conv_work(dtype, rows, c, taps))
        self._chk(self.lib.emc2_causal_conv_backward(self.h, dtype, xp, ld_x, wp, bp, bool(silu), at, n_seq, rows, c, taps, bool(backwards), fp, dyp, ld_dy,
                                                     dlp, dxp, ld_dx, dwp, dbp, dfp, wk, size, _stream_of(dev)))

    def causal_conv_step(self, dtype: int, x: torch.Tensor, w: torch.Tensor, state: torch.Tensor, state_out: torch.Tensor, y: torch.Tensor,
                         bias: Optional[torch.Tensor] = None, silu: bool = True) -> None:
        """One row per sequence; state [rows][taps - 1][channels]: the rows before, oldest first; state_out (may be state): moved on by the row."""
        dev, shape = self._current(), _shape_of(x)
        rows, c = shape
        xp, ld_x, yp, ld_y = _rows_at(dev, _TORCH_DTYPE[dtype], shape, ("x", "y"), x, y)
        taps = w.shape[0] if w.dim() == 2 else 0
        kept = (rows, taps - 1, c)
        wp, bp, sp, op = _floats_at(dev, (w, (taps, c), "w"), (bias, (c,), "bias"), (state, kept, "state"), (state_out, kept, "state_out"))
        self._chk(self.lib.emc2_causal_conv_step(self.h, dtype, xp, ld_x, wp, bp, bool(silu), sp, rows, c, taps, op, yp, ld_y, _stream_of(dev)))

    def gated_residual(self, dtype: int, x: torch.Tensor, branch: torch.Tensor, post: torch.Tensor, scale: torch.Tensor, total: torch.Tensor,
                       eps: float, gate: Optional[torch.Tensor] = None, next_gain: Optional[torch.Tensor] = None,
                       y: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None) -> None:
        """total = x + scale silu(gate) rms(branch) post and, if y is given, y = rms(total) next_gain; scale: one value; n: device count of the rows present."""
        dev, shape = self._current(), _shape_of(x)
        rows, c = shape
        xp, ld_x, bp, ld_b, gp, ld_g, tp, ld_t, yp, ld_y = _rows_at(dev, _TORCH_DTYPE[dtype], shape, ("x", "branch", "gate", "total", "y"),
                                                                    x, branch, gate, total, y)
        pp, sp, np = _floats_at(dev, (post, (c,), "post"), (scale, (1,), "scale"), (next_gain, (c,), "next_gain"))
        self._chk(self.lib.emc2_gated_residual(self.h, dtype, xp, ld_x, bp, ld_b, gp, ld_g, pp, sp, np, eps, _ints_at(dev, n, "n"), rows, c, tp, ld_t, yp,
                                               ld_y, _stream_of(dev)))

    def gated_residual_work(self, dtype: int, capacity: int, channels: int) -> int:
        return self.lib.emc2_gated_residual_work(dtype, capacity, channels)

    def gated_residual_backward(self, dtype: int, x: torch.Tensor, branch: torch.Tensor, post: torch.Tensor, scale: torch.Tensor, eps: float,
                                dtotal: Optional[torch.Tensor], dx: torch.Tensor, dbranch: torch.Tensor, dpost: torch.Tensor,
                                dscale: torch.Tensor, work: torch.Tensor, gate: Optional[torch.Tensor] = None,
                                dgate: Optional[torch.Tensor] = None, next_gain: Optional[torch.Tensor] = None,
                                dy: Optional[torch.Tensor] = None, dnext: Optional[torch.Tensor] = None,
                                n: Optional[torch.Tensor] = None) -> None:
        """dx, dbranch, dgate, dpost, dscale and dnext of a gated_residual for dtotal and dy (either may be None)."""
        dev, shape = self._current(), _shape_of(x)
        rows, c = shape
        xp, ld_x, bp, ld_b, gp, ld_g, dtp, ld_dt, dyp, ld_dy, dxp, ld_dx, dbp, ld_db, dgp, ld_dg = _rows_at(
            dev, _TORCH_DTYPE[dtype], shape, ("x", "branch", "gate", "dtotal", "dy", "dx", "dbranch", "dgate"), x, branch, gate, dtotal, dy, dx, dbranch, dgate)
        pp, sp, np, dpp, dsp, dnp = _floats_at(dev, (post, (c,), "post"), (scale, (1,), "scale"), (next_gain, (c,), "next_gain"), (dpost, (c,), "dpost"),
                                               (dscale, (1,), "dscale"), (dnext, (c,), "dnext"))
        wk, size = _work_at(dev, work, self.lib.emc2_gated_residual_work(dtype, rows, c))
        self._chk(self.lib.emc2_gated_residual_backward(self.h, dtype, xp, ld_x, bp, ld_b, gp, ld_g, pp, sp, np, eps, dtp, ld_dt, dyp, ld_dy,
                                                        _ints_at(dev, n, "n"), rows, c, dxp, ld_dx, dbp, ld_db, dgp, ld_dg, dpp, dsp, dnp, wk, size,
                                                        _stream_of(dev)))

    def selective_scan_work(self, dtype: int, capacity: int, channels: int, states: int) -> int:
        return self.lib.emc2_selective_scan_work(dtype, capacity, channels, states)

    def selective_scan(self, dtype: int, x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor, offsets: torch.Tensor,
                       y: torch.Tensor, work: torch.Tensor, skip: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None,
                       backwards: bool = False, h0: Optional[torch.Tensor] = None, last: Optional[torch.Tensor] = None) -> None:
        """h_t = exp(D_t a) h_{t-1} + D_t x_t b_t and y_t = c_t . h_t + skip x_t along every sequence, D = softplus(dt + dt_bias); x, dt, y rows of channels,
        b, c rows of states, a [channels][states], h0 and last [sequences][channels][states].  `last` must not overlap h0."""
        dev, shape = self._current(), _shape_of(x)
        td, (rows, ch), m = _TORCH_DTYPE[dtype], shape, a.shape[1] if a.dim() == 2 else 0
        xp, ld_x, dtp, ld_dt, yp, ld_y = _rows_at(dev, td, shape, ("x", "dt", "y"), x, dt, y)
        bp, ld_b, cp, ld_c = _rows_at(dev, td, torch.Size((rows, m)), ("b", "c"), b, c)
        at, n_seq = _ints_at(dev, offsets, "offsets"), offsets.numel() - 1
        ap, sp, op, hp, lp = _floats_at(dev, (a, (ch, m), "a"), (skip, (ch,), "skip"), (dt_bias, (ch,), "dt_bias"), (h0, (n_seq, ch, m), "h0"),
                                        (last, (n_seq, ch, m), "last"))
        wk, size = _work_at(dev, work, self.lib.emc2_selective_scan_work(dtype, rows, ch, m))
        self._chk(self.lib.emc2_selective_scan(self.h, dtype, xp, ld_x, dtp, ld_dt, ap, bp, ld_b, cp, ld_c, sp, op, at, n_seq, rows, ch, m, bool(backwards),
                                               hp, yp, ld_y, lp, wk, size, _stream_of(dev)))

    def selective_scan_backward(self, dtype: int, x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor,
                                offsets: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor, ddt: torch.Tensor, da: torch.Tensor, db: torch.Tensor,
                                dc: torch.Tensor, work: torch.Tensor, skip: Optional[torch.Tensor] = None, dskip: Optional[torch.Tensor] = None,
                                dt_bias: Optional[torch.Tensor] = None, ddt_bias: Optional[torch.Tensor] = None, backwards: bool = False,
                                h0: Optional[torch.Tensor] = None, dlast: Optional[torch.Tensor] = None,
                                dh0: Optional[torch.Tensor] = None) -> None:
        """The gradients of a selective_scan for dy and the gradient of the last states; dh0 must not overlap dlast or h0."""
        dev, shape = self._current(), _shape_of(x)
        td, (rows, ch), m = _TORCH_DTYPE[dtype], shape, a.shape[1] if a.dim() == 2 else 0
        xp, ld_x, dtp, ld_dt, dyp, ld_dy, dxp, ld_dx, ddtp, ld_ddt = _rows_at(dev, td, shape, ("x", "dt", "dy", "dx", "ddt"), x, dt, dy, dx, ddt)
        bp, ld_b, cp, ld_c, dbp, ld_db, dcp, ld_dc = _rows_at(dev, td, torch.Size((rows, m)), ("b", "c", "db", "dc"), b, c, db, dc)
        at, n_seq = _ints_at(dev, offsets, "offsets"), offsets.numel() - 1
        kept = (n_seq, ch, m)
        ap, sp, op, hp, dlp, dap, dsp, dop, dhp = _floats_at(dev, (a, (ch, m), "a"), (skip, (ch,), "skip"), (dt_bias, (ch,), "dt_bias"), (h0, kept, "h0"),
                                                             (dlast, kept, "dlast"), (da, (ch, m), "da"), (dskip, (ch,), "dskip"),
                                                             (ddt_bias, (ch,), "ddt_bias"), (dh0, kept, "dh0"))
        wk, size = _work_at(dev, work, self.lib.emc2_selective_scan_work(dtype, rows, ch, m))
        self._chk(self.lib.emc2_selective_scan_backward(self.h, dtype, xp, ld_x, dtp, ld_dt, ap, bp, ld_b, cp, ld_c, sp, op, at, n_seq, rows, ch, m,
                                                        bool(backwards), hp, dyp, ld_dy, dlp, dxp, ld_dx, ddtp, ld_ddt, dap, dbp, ld_db, dcp, ld_dc, dsp, dop,
                                                        dhp, wk, size, _stream_of(dev)))

    def selective_scan_step(self, dtype: int, x: torch.Tensor, dt: torch.Tensor, a: torch.Tensor, b: torch.Tensor, c: torch.Tensor, h: torch.Tensor,
                            h_out: torch.Tensor, y: torch.Tensor, skip: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None) -> None:
        """One row per sequence: the states h [rows][channels][states] moved on by the row, to h_out (may be h), and y."""
        dev, shape = self._current(), _shape_of(x)
        td, (rows, ch), m = _TORCH_DTYPE[dtype], shape, a.shape[1] if a.dim() == 2 else 0
        xp, ld_x, dtp, ld_dt, yp, ld_y = _rows_at(dev, td, shape, ("x", "dt", "y"), x, dt, y)
        bp, ld_b, cp, ld_c = _rows_at(dev, td, torch.Size((rows, m)), ("b", "c"), b, c)
        kept = (rows, ch, m)
        ap, sp, op, hp, to = _floats_at(dev, (a, (ch, m), "a"), (skip, (ch,), "skip"), (dt_bias, (ch,), "dt_bias"), (h, kept, "h"), (h_out, kept, "h_out"))
        self._chk(self.lib.emc2_selective_scan_step(self.h, dtype, xp, ld_x, dtp, ld_dt, ap, bp, ld_b, cp, ld_c, sp, op, hp, rows, ch, m, to, yp, ld_y,
                                                    _stream_of(dev)))
