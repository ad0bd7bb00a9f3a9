"""ctypes binding of libvp.so.  Function names and argument order follow include/vp.h.

Tensors are torch tensors on the GPU; bf16 data may be passed as torch.bfloat16 or as
int16/uint16 bit patterns.  Nothing here computes: the functions check dtype / device /
contiguity, take raw pointers and the current HIP stream, and call the library.  The checks run in
native code (_vphost.so); what does not pass there is checked again here, where the message is made
(everything is, where that module is missing or belongs to another PyTorch: small passes then take
twice as long).  The library has no fallback: if it is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings
from typing import Optional

import torch

VP_F32 = 0
VP_BF16 = 1
VP_SAVE_LOGITS = 1
VP_SKIP_DH = 2
VP_DH_OVERWRITE = 4
VP_NORM_POST = 8
VP_NORM_CENTER = 16

VP_CALL_OUTPUT_FWD = 0
VP_CALL_COMBINE_STATS = 1
VP_CALL_OUTPUT_BWD = 2
VP_CALL_EMBED_FWD = 3
VP_CALL_EMBED_BWD = 4
VP_CALL_OUTPUT_FWD_ALG2 = 5
VP_CALL_OUTPUT_DX_ALG2 = 6

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None
_HOST = None      # _vphost.so, loaded with the library, or None
_ADDRESS = {}     # of the library's functions that _vphost.so calls itself


class VPError(RuntimeError):
    pass


def lib_path() -> str:
    return os.path.join(_HERE, "libvp.so")


def host_path() -> str:
    return os.path.join(_HERE, "_vphost.so")


def _load_host(path: str):
    """The native checks, or None where there are none that fit this PyTorch, whose objects they read."""
    if not os.path.exists(path):
        return None
    try:
        spec = importlib.util.spec_from_file_location("_vphost", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError as e:
        warnings.warn("%s cannot be loaded (%s): tensors are checked in Python" % (path, e))
        return None
    if module.torch_version != torch.__version__.split("+")[0]:
        warnings.warn("%s was built for PyTorch %s: tensors are checked in Python" % (path, module.torch_version))
        return None
    return module


def load_library() -> ctypes.CDLL:
    """Loads libvp.so (built by ``python -m paper_2411_05288_amd.build``)."""
    global _LIB, _HOST
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise VPError("libvp.so not found at %s: build it with `python -m paper_2411_05288_amd.build`" % path)
    host = _load_host(host_path()) if _HOST is None else _HOST
    lib = ctypes.CDLL(path)
    c = ctypes
    vp, i64, i32, u32, sz, fl = c.c_void_p, c.c_int64, c.c_int32, c.c_uint32, c.c_size_t, c.c_float
    lib.vp_version.restype = c.c_int
    lib.vp_version.argtypes = []
    lib.vp_status_string.restype = c.c_char_p
    lib.vp_status_string.argtypes = [c.c_int]
    lib.vp_workspace_bytes.restype = sz
    lib.vp_workspace_bytes.argtypes = [c.c_int, i64, i64, i64, c.c_int, u32]
    lib.vp_dlogits_row_stride.restype = i64
    lib.vp_dlogits_row_stride.argtypes = [i64, c.c_int]
    lib.vp_output_fwd.restype = c.c_int
    lib.vp_output_fwd.argtypes = [vp, vp, vp, i64, i64, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_output_fwd_noalloc.restype = c.c_int
    lib.vp_output_fwd_noalloc.argtypes = [vp, vp, vp, i64, i64, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp]
    lib.vp_output_fwd_noalloc_max_scratch.restype = sz
    lib.vp_output_fwd_noalloc_max_scratch.argtypes = []
    lib.vp_combine_stats.restype = c.c_int
    lib.vp_combine_stats.argtypes = [vp, vp, vp, i32, i64, vp, vp, vp, vp, vp]
    lib.vp_output_bwd.restype = c.c_int
    lib.vp_output_bwd.argtypes = [vp, vp, vp, i64, i64, i64, i64, c.c_int, u32, vp, vp, vp, fl, vp, vp, vp, sz, vp]
    lib.vp_output_group_workspace_bytes.restype = sz
    lib.vp_output_group_workspace_bytes.argtypes = [c.c_int, i32, i64, i64, vp, c.c_int, u32]
    lib.vp_output_fwd_group.restype = c.c_int
    lib.vp_output_fwd_group.argtypes = [vp, vp, vp, vp, i32, vp, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_output_bwd_group.restype = c.c_int
    lib.vp_output_bwd_group.argtypes = [vp, vp, vp, vp, i32, vp, i64, i64, c.c_int, u32, vp, vp, vp, fl, vp, vp, vp, sz, vp]
    lib.vp_output_fwd_alg2.restype = c.c_int
    lib.vp_output_fwd_alg2.argtypes = [vp, vp, vp, i64, i64, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_output_dx_alg2.restype = c.c_int
    lib.vp_output_dx_alg2.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, c.c_int, u32, fl, vp, vp]
    lib.vp_output_fwd_alg2_group.restype = c.c_int
    lib.vp_output_fwd_alg2_group.argtypes = [vp, vp, vp, vp, i32, vp, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_output_dx_alg2_gather.restype = c.c_int
    lib.vp_output_dx_alg2_gather.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, i64, i64, c.c_int, u32, fl, vp, vp]
    lib.vp_output_dx_alg2_group.restype = c.c_int
    lib.vp_output_dx_alg2_group.argtypes = [vp, vp, i32, vp, vp, vp, vp, i64, i64, c.c_int, u32, fl, vp, vp]
    lib.vp_embed_fwd.restype = c.c_int
    lib.vp_embed_fwd.argtypes = [vp, vp, i64, i64, i64, i64, c.c_int, vp, vp]
    lib.vp_embed_bwd.restype = c.c_int
    lib.vp_embed_bwd.argtypes = [vp, vp, i64, i64, i64, i64, c.c_int, vp, vp, sz, vp]
    lib.vp_embed_fwd_group.restype = c.c_int
    lib.vp_embed_fwd_group.argtypes = [vp, vp, i32, i64, i64, i64, i64, c.c_int, vp, vp]
    lib.vp_embed_bwd_group.restype = c.c_int
    lib.vp_embed_bwd_group.argtypes = [vp, vp, i32, i64, i64, i64, i64, c.c_int, vp, vp, sz, vp]
    lib.vp_block_norm_fwd.restype = c.c_int
    lib.vp_block_norm_fwd.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i64, i64, c.c_int, u32, fl, fl, vp, vp, vp, vp]
    lib.vp_block_norm_bwd_workspace_bytes.restype = sz
    lib.vp_block_norm_bwd_workspace_bytes.argtypes = [i64, i64, i64, u32]
    lib.vp_block_norm_bwd.restype = c.c_int
    lib.vp_block_norm_bwd.argtypes = [vp, c.c_int, vp, vp, vp, vp, i64, vp, vp, vp, vp, i64, i64, c.c_int, u32, fl, c.c_int,
                                      vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_grad_workspace_bytes.restype = sz
    lib.vp_grad_workspace_bytes.argtypes = [i32]
    lib.vp_grad_norm.restype = c.c_int
    lib.vp_grad_norm.argtypes = [vp, vp, vp, i32, vp, vp, sz, vp]
    lib.vp_grad_clip.restype = c.c_int
    lib.vp_grad_clip.argtypes = [vp, vp, vp, i32, vp, fl, vp, vp, sz, vp]
    lib.vp_grad_scale.restype = c.c_int
    lib.vp_grad_scale.argtypes = [vp, vp, vp, i32, vp, fl, vp, vp, sz, vp]
    lib.vp_i8_row_stride.restype = i64
    lib.vp_i8_row_stride.argtypes = [i64]
    lib.vp_quantize_rows.restype = c.c_int
    lib.vp_quantize_rows.argtypes = [vp, i64, i64, c.c_int, vp, vp, vp]
    lib.vp_output_i8_workspace_bytes.restype = sz
    lib.vp_output_i8_workspace_bytes.argtypes = [i32, i64, vp]
    lib.vp_output_fwd_i8.restype = c.c_int
    lib.vp_output_fwd_i8.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_output_fwd_i8_group.restype = c.c_int
    lib.vp_output_fwd_i8_group.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, i64, i64, c.c_int, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.vp_logits_stats_workspace_bytes.restype = sz
    lib.vp_logits_stats_workspace_bytes.argtypes = [i32, i64, vp]
    lib.vp_logits_stats.restype = c.c_int
    lib.vp_logits_stats.argtypes = [vp, vp, i32, c.c_int, i64, vp, vp, vp, sz, vp]
    lib.vp_verify_workspace_bytes.restype = sz
    lib.vp_verify_workspace_bytes.argtypes = [i32, i64]
    lib.vp_verify_drafts.restype = c.c_int
    lib.vp_verify_drafts.argtypes = [vp, vp, vp, i32, c.c_int, vp, vp, vp, vp, vp, vp, vp, vp, i64, i32, vp, vp, vp, sz, vp]
    lib.vp_profile_mfma_loop.restype = c.c_int
    lib.vp_profile_mfma_loop.argtypes = [vp, vp, i32, i32, vp]
    lib.vp_profile_mfma_variant.restype = c.c_int
    lib.vp_profile_mfma_variant.argtypes = [vp, vp, i32, i32, i32, vp]
    lib.vp_profile_mfma_variant_count.restype = c.c_int
    lib.vp_profile_mfma_variant_count.argtypes = []
    lib.vp_profile_mfma_variant_flops.restype = c.c_double
    lib.vp_profile_mfma_variant_flops.argtypes = [i32]
    lib.vp_profile_force_generic_gemm.restype = c.c_int
    lib.vp_profile_force_generic_gemm.argtypes = [c.c_int]
    lib.vp_profile_f32_scratch_written.restype = sz
    lib.vp_profile_f32_scratch_written.argtypes = [c.c_int, i64, i64, i64]
    lib.vp_profile_gemm_trace.restype = c.c_int
    lib.vp_profile_gemm_trace.argtypes = [vp, sz, c.c_int]
    lib.vp_profile_kernel_count.restype = c.c_int
    lib.vp_profile_kernel_count.argtypes = []
    lib.vp_profile_kernel_name.restype = c.c_char_p
    lib.vp_profile_kernel_name.argtypes = [c.c_int]
    lib.vp_profile_enable.restype = c.c_int
    lib.vp_profile_enable.argtypes = [c.c_int]
    lib.vp_profile_read.restype = c.c_int
    lib.vp_profile_read.argtypes = [c.POINTER(c.c_double), c.POINTER(c.c_int64), c.c_int]
    for name in ("vp_block_norm_fwd", "vp_block_norm_bwd", "vp_quantize_rows", "vp_output_fwd_i8_group", "vp_logits_stats",
                 "vp_verify_drafts"):
        _ADDRESS[name] = c.cast(getattr(lib, name), vp).value
    _LIB, _HOST = lib, host      # (only now: the native checks call the library's functions)
    return lib


def _check(status: int, what: str) -> None:
    if status != 0:
        name = load_library().vp_status_string(status).decode()
        raise VPError("%s failed: %s" % (what, name))


_BF16_LIKE = (torch.bfloat16, torch.int16, torch.uint16)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return VP_F32
    if t.dtype in _BF16_LIKE:
        return VP_BF16
    raise VPError("unsupported tensor dtype %s" % t.dtype)


def _ptr(t: Optional[torch.Tensor], name: str, dtypes=None, shape=None) -> Optional[int]:
    if t is None:
        return None
    if _HOST is not None:
        p = _HOST.ptr(t, dtypes, shape)
        if p is not None:
            return p
    if not t.is_cuda:
        raise VPError("%s must be a GPU tensor" % name)
    if not t.is_contiguous():
        raise VPError("%s must be contiguous" % name)
    if dtypes is not None and t.dtype not in dtypes:
        raise VPError("%s has dtype %s, expected one of %s" % (name, t.dtype, dtypes))
    if shape is not None and t.shape != shape:
        raise VPError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


def _ptrs(ts, name: str, dtypes, shape):
    """Array of the device pointers of one tensor per shard."""
    if _HOST is not None:
        a = _HOST.ptrs(ts, dtypes, shape)
        if a is not None:
            return a
    return (ctypes.c_void_p * len(ts))(*[_ptr(t, name, dtypes, shape) for t in ts])


def same_shapes(ts) -> bool:
    """Whether all tensors of the list have one shape."""
    same = _HOST.same_shapes(ts) if _HOST is not None else None
    return all(t.shape == ts[0].shape for t in ts) if same is None else same


def _stream(stream) -> int:
    if stream is None:
        s = _HOST.stream() if _HOST is not None else None
        if s is not None:
            return s
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def vp_version() -> int:
    return load_library().vp_version()


def vp_workspace_bytes(which: int, N: int, h: int, Vs: int, dt: int, flags: int = 0) -> int:
    n = load_library().vp_workspace_bytes(which, N, h, Vs, dt, flags)
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_workspace_bytes: invalid arguments")
    return n


def vp_dlogits_row_stride(Vs: int, dt: int) -> int:
    n = load_library().vp_dlogits_row_stride(Vs, dt)
    if n < 0:
        raise VPError("vp_dlogits_row_stride: invalid arguments")
    return n


def _ws(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    return _ptr(workspace, "workspace"), workspace.numel() * workspace.element_size()


def vp_output_fwd(H, W_shard, labels, shard_offset: int, local_max, local_sumexp, local_target,
                  logits_out=None, workspace=None, stream=None) -> None:
    """Pass S for one shard; writes local_max / local_sumexp / local_target ([N] fp32 each)."""
    N, h = H.shape
    Vs = W_shard.shape[0]
    dt = _dtype_code(H)
    if _dtype_code(W_shard) != dt or W_shard.shape[1] != h:
        raise VPError("W_shard must be [Vs, h] with the dtype of H")
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd(
        _ptr(H, "H"), _ptr(W_shard, "W_shard"), _ptr(labels, "labels", (torch.int64,), (N,)),
        N, h, Vs, shard_offset, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", (torch.float32,), (N,)),
        _ptr(local_sumexp, "local_sumexp", (torch.float32,), (N,)),
        _ptr(local_target, "local_target", (torch.float32,), (N,)),
        _ptr(logits_out, "logits_out", same, (N, Vs)), wp, wb, _stream(stream))
    _check(st, "vp_output_fwd")


def vp_output_fwd_noalloc(H, W_shard, labels, shard_offset: int, local_max, local_sumexp, local_target,
                          logits_out=None, stream=None) -> None:
    """vp_output_fwd with the scratch in a static device array of the library: no workspace argument,
    nothing allocated.  Sizes whose scratch exceeds vp_output_fwd_noalloc_max_scratch() are refused."""
    N, h = H.shape
    Vs = W_shard.shape[0]
    dt = _dtype_code(H)
    if _dtype_code(W_shard) != dt or W_shard.shape[1] != h:
        raise VPError("W_shard must be [Vs, h] with the dtype of H")
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    st = load_library().vp_output_fwd_noalloc(
        _ptr(H, "H"), _ptr(W_shard, "W_shard"), _ptr(labels, "labels", (torch.int64,), (N,)),
        N, h, Vs, shard_offset, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", (torch.float32,), (N,)),
        _ptr(local_sumexp, "local_sumexp", (torch.float32,), (N,)),
        _ptr(local_target, "local_target", (torch.float32,), (N,)),
        _ptr(logits_out, "logits_out", same, (N, Vs)), _stream(stream))
    _check(st, "vp_output_fwd_noalloc")


def vp_output_fwd_noalloc_max_scratch() -> int:
    return load_library().vp_output_fwd_noalloc_max_scratch()


def vp_combine_stats(local_max, local_sumexp, local_target, global_max, global_sumexp, loss_per_row,
                     loss_mean, stream=None) -> None:
    """Barrier C1 over the p rows of the [p, N] statistics."""
    p, N = local_max.shape
    f = (torch.float32,)
    st = load_library().vp_combine_stats(
        _ptr(local_max, "local_max", f, (p, N)), _ptr(local_sumexp, "local_sumexp", f, (p, N)),
        _ptr(local_target, "local_target", f, (p, N)), p, N,
        _ptr(global_max, "global_max", f, (N,)), _ptr(global_sumexp, "global_sumexp", f, (N,)),
        _ptr(loss_per_row, "loss_per_row", f, (N,)), _ptr(loss_mean, "loss_mean", f, (1,)), _stream(stream))
    _check(st, "vp_combine_stats")


def vp_output_bwd(H, W_shard, labels, shard_offset: int, global_max, global_sumexp, logits_saved,
                  grad_scale: float, dH_accum, dW_shard, workspace, stream=None, dh_overwrite: bool = False) -> None:
    """Pass T for one shard: dH_accum += D W_shard, dW_shard = D^T H.  dH_accum=None selects pass T of
    Algorithm 2 (flag VP_SKIP_DH): only dW_shard is formed.  dh_overwrite=True (flag VP_DH_OVERWRITE)
    writes dH_accum = D W_shard: the first term of the reduce, no zero-fill needed."""
    N, h = H.shape
    Vs = W_shard.shape[0]
    dt = _dtype_code(H)
    if _dtype_code(W_shard) != dt or W_shard.shape[1] != h:
        raise VPError("W_shard must be [Vs, h] with the dtype of H")
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    f = (torch.float32,)
    wp, wb = _ws(workspace)
    st = load_library().vp_output_bwd(
        _ptr(H, "H"), _ptr(W_shard, "W_shard"), _ptr(labels, "labels", (torch.int64,), (N,)),
        N, h, Vs, shard_offset, dt,
        (VP_SAVE_LOGITS if logits_saved is not None else 0) | (VP_SKIP_DH if dH_accum is None else 0)
        | (VP_DH_OVERWRITE if (dh_overwrite and dH_accum is not None) else 0),
        _ptr(global_max, "global_max", f, (N,)), _ptr(global_sumexp, "global_sumexp", f, (N,)),
        _ptr(logits_saved, "logits_saved", same, (N, Vs)), float(grad_scale),
        _ptr(dH_accum, "dH_accum", f, (N, h)), _ptr(dW_shard, "dW_shard", f, (Vs, h)),
        wp, wb, _stream(stream))
    _check(st, "vp_output_bwd")


def _i64s(xs):
    return (ctypes.c_int64 * len(xs))(*xs)


def vp_output_group_workspace_bytes(which: int, N: int, h: int, rows, dt: int, flags: int = 0) -> int:
    n = load_library().vp_output_group_workspace_bytes(which, len(rows), N, h, _i64s(rows), dt, flags)
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_output_group_workspace_bytes: invalid arguments")
    return n


def _shards(H, W_shards, offsets):
    """dtype code and row counts of the shards of a group call."""
    dt = _dtype_code(H)
    if len(offsets) != len(W_shards):
        raise VPError("one offset per shard")
    for w in W_shards:
        if _dtype_code(w) != dt or w.shape[1] != H.shape[1]:
            raise VPError("W_shards must be [rows, h] with the dtype of H")
    return dt, [int(w.shape[0]) for w in W_shards]


def _each(ts, name, dtypes, shapes):
    if ts is None:
        return None
    if len(ts) != len(shapes):
        raise VPError("%s: one tensor per shard" % name)
    if _HOST is not None:
        a = _HOST.ptrs(ts, dtypes, shapes)
        if a is not None:
            return a
    return (ctypes.c_void_p * len(ts))(*[_ptr(t, name, dtypes, s) for t, s in zip(ts, shapes)])


def vp_output_fwd_group(H, W_shards, labels, shard_offsets, local_max, local_sumexp, local_target, logits_out=None,
                        workspace=None, stream=None) -> None:
    """vp_output_fwd for several shards on this device in one call; the statistics are [p, N]."""
    N, h = H.shape
    dt, rows = _shards(H, W_shards, shard_offsets)
    p = len(rows)
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    f = (torch.float32,)
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd_group(
        _ptr(H, "H"), _each(W_shards, "W_shards", None, [(n, h) for n in rows]), _i64s(rows), _i64s(shard_offsets), p,
        _ptr(labels, "labels", (torch.int64,), (N,)), N, h, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", f, (p, N)), _ptr(local_sumexp, "local_sumexp", f, (p, N)),
        _ptr(local_target, "local_target", f, (p, N)), _each(logits_out, "logits_out", same, [(N, n) for n in rows]),
        wp, wb, _stream(stream))
    _check(st, "vp_output_fwd_group")


def vp_output_bwd_group(H, W_shards, labels, shard_offsets, global_max, global_sumexp, logits_saved, grad_scale: float,
                        dH_accum, dW_shards, workspace, stream=None, dh_overwrite: bool = False) -> None:
    """vp_output_bwd for several shards on this device in one call (arguments as there, one entry per shard)."""
    N, h = H.shape
    dt, rows = _shards(H, W_shards, shard_offsets)
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    f = (torch.float32,)
    wp, wb = _ws(workspace)
    st = load_library().vp_output_bwd_group(
        _ptr(H, "H"), _each(W_shards, "W_shards", None, [(n, h) for n in rows]), _i64s(rows), _i64s(shard_offsets),
        len(rows), _ptr(labels, "labels", (torch.int64,), (N,)), N, h, dt,
        (VP_SAVE_LOGITS if logits_saved is not None else 0) | (VP_SKIP_DH if dH_accum is None else 0)
        | (VP_DH_OVERWRITE if (dh_overwrite and dH_accum is not None) else 0),
        _ptr(global_max, "global_max", f, (N,)), _ptr(global_sumexp, "global_sumexp", f, (N,)),
        _each(logits_saved, "logits_saved", same, [(N, n) for n in rows]), float(grad_scale),
        _ptr(dH_accum, "dH_accum", f, (N, h)), _each(dW_shards, "dW_shards", f, [(n, h) for n in rows]),
        wp, wb, _stream(stream))
    _check(st, "vp_output_bwd_group")


def vp_output_fwd_alg2(H, W_shard, labels, shard_offset: int, local_max, local_sumexp, local_target,
                       A_out, B_out, logits_out=None, workspace=None, stream=None) -> None:
    """Pass S of Algorithm 2 for one shard: the outputs of vp_output_fwd plus A = softmax' W_shard
    ([N, h] fp32) and B = G W_shard ([N, h], dtype of W)."""
    N, h = H.shape
    Vs = W_shard.shape[0]
    dt = _dtype_code(H)
    if _dtype_code(W_shard) != dt or W_shard.shape[1] != h:
        raise VPError("W_shard must be [Vs, h] with the dtype of H")
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    f = (torch.float32,)
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd_alg2(
        _ptr(H, "H"), _ptr(W_shard, "W_shard"), _ptr(labels, "labels", (torch.int64,), (N,)),
        N, h, Vs, shard_offset, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", f, (N,)), _ptr(local_sumexp, "local_sumexp", f, (N,)),
        _ptr(local_target, "local_target", f, (N,)), _ptr(logits_out, "logits_out", same, (N, Vs)),
        _ptr(A_out, "A_out", f, (N, h)), _ptr(B_out, "B_out", same, (N, h)), wp, wb, _stream(stream))
    _check(st, "vp_output_fwd_alg2")


def vp_output_dx_alg2(A, B, local_max, local_sumexp, global_max, global_sumexp, grad_scale: float, dH_accum,
                      stream=None, dh_overwrite: bool = False) -> None:
    """dH_accum += (A * sum' e^{m'-m} / sum - B) * grad_scale: this shard's term of Algorithm 2's input gradient
    (dh_overwrite=True, flag VP_DH_OVERWRITE: = instead of +=, the first term of the reduce)."""
    N, h = A.shape
    f = (torch.float32,)
    dt = _dtype_code(B)
    st = load_library().vp_output_dx_alg2(
        _ptr(A, "A", f, (N, h)), _ptr(B, "B", None, (N, h)), _ptr(local_max, "local_max", f, (N,)),
        _ptr(local_sumexp, "local_sumexp", f, (N,)), _ptr(global_max, "global_max", f, (N,)),
        _ptr(global_sumexp, "global_sumexp", f, (N,)), N, h, dt, VP_DH_OVERWRITE if dh_overwrite else 0,
        float(grad_scale), _ptr(dH_accum, "dH_accum", f, (N, h)), _stream(stream))
    _check(st, "vp_output_dx_alg2")


def vp_output_fwd_alg2_group(H, W_shards, labels, shard_offsets, local_max, local_sumexp, local_target, A_out, B_out,
                             logits_out=None, workspace=None, stream=None) -> None:
    """vp_output_fwd_alg2 for several shards on this device in one call: the statistics are [p, N], A_out is [p, N, h]."""
    N, h = H.shape
    dt, rows = _shards(H, W_shards, shard_offsets)
    p = len(rows)
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    f = (torch.float32,)
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd_alg2_group(
        _ptr(H, "H"), _each(W_shards, "W_shards", None, [(n, h) for n in rows]), _i64s(rows), _i64s(shard_offsets), p,
        _ptr(labels, "labels", (torch.int64,), (N,)), N, h, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", f, (p, N)), _ptr(local_sumexp, "local_sumexp", f, (p, N)),
        _ptr(local_target, "local_target", f, (p, N)), _each(logits_out, "logits_out", same, [(N, n) for n in rows]),
        _ptr(A_out, "A_out", f, (p, N, h)), _each(B_out, "B_out", same, [(N, h)] * p), wp, wb, _stream(stream))
    _check(st, "vp_output_fwd_alg2_group")


def vp_output_dx_alg2_gather(A, W_shards, labels, shard_offsets, local_max, local_sumexp, global_max, global_sumexp,
                             grad_scale: float, dH_accum, stream=None, dh_overwrite: bool = False) -> None:
    """vp_output_dx_alg2_group with A [p, N, h] and the rows of B taken from the shards."""
    p, N, h = A.shape
    f = (torch.float32,)
    rows = [int(w.shape[0]) for w in W_shards]
    if len(shard_offsets) != p or len(rows) != p:
        raise VPError("one offset and one matrix per shard")
    st = load_library().vp_output_dx_alg2_gather(
        _ptr(A, "A", f, (p, N, h)), _each(W_shards, "W_shards", (W_shards[0].dtype,), [(n, h) for n in rows]), _i64s(rows),
        _i64s(shard_offsets), p, _ptr(labels, "labels", (torch.int64,), (N,)), _ptr(local_max, "local_max", f, (p, N)),
        _ptr(local_sumexp, "local_sumexp", f, (p, N)), _ptr(global_max, "global_max", f, (N,)),
        _ptr(global_sumexp, "global_sumexp", f, (N,)), N, h, _dtype_code(W_shards[0]), VP_DH_OVERWRITE if dh_overwrite else 0,
        float(grad_scale), _ptr(dH_accum, "dH_accum", f, (N, h)), _stream(stream))
    _check(st, "vp_output_dx_alg2_gather")


def vp_output_dx_alg2_group(A, B, local_max, local_sumexp, global_max, global_sumexp, grad_scale: float, dH_accum,
                            stream=None, dh_overwrite: bool = False) -> None:
    """vp_output_dx_alg2 for several shards in one call, in order; local_max and local_sumexp are [p, N]."""
    N, h = A[0].shape
    p = len(A)
    f = (torch.float32,)
    st = load_library().vp_output_dx_alg2_group(
        _ptrs(A, "A", f, (N, h)), _each(B, "B", (B[0].dtype,), [(N, h)] * p), p, _ptr(local_max, "local_max", f, (p, N)),
        _ptr(local_sumexp, "local_sumexp", f, (p, N)), _ptr(global_max, "global_max", f, (N,)),
        _ptr(global_sumexp, "global_sumexp", f, (N,)), N, h, _dtype_code(B[0]), VP_DH_OVERWRITE if dh_overwrite else 0,
        float(grad_scale), _ptr(dH_accum, "dH_accum", f, (N, h)), _stream(stream))
    _check(st, "vp_output_dx_alg2_group")


def vp_embed_fwd(table_shard, ids, shard_offset: int, out, stream=None) -> None:
    Vs, h = table_shard.shape
    N = ids.shape[0]
    dt = _dtype_code(table_shard)
    st = load_library().vp_embed_fwd(
        _ptr(table_shard, "table_shard"), _ptr(ids, "ids", (torch.int64,), (N,)), N, h, Vs, shard_offset, dt,
        _ptr(out, "out", (table_shard.dtype,), (N, h)), _stream(stream))
    _check(st, "vp_embed_fwd")


def vp_embed_bwd(grad_out, ids, shard_offset: int, dtable_shard, workspace, stream=None) -> None:
    N, h = grad_out.shape
    Vs = dtable_shard.shape[0]
    dt = _dtype_code(grad_out)
    wp, wb = _ws(workspace)
    st = load_library().vp_embed_bwd(
        _ptr(grad_out, "grad_out"), _ptr(ids, "ids", (torch.int64,), (N,)), N, h, Vs, shard_offset, dt,
        _ptr(dtable_shard, "dtable_shard", (torch.float32,), (Vs, h)), wp, wb, _stream(stream))
    _check(st, "vp_embed_bwd")


def vp_embed_fwd_group(table_shards, ids, shard_offset: int, outs, stream=None) -> None:
    """vp_embed_fwd for consecutive shards of equal size in one call; shard_offset is that of the first."""
    Vs, h = table_shards[0].shape
    N, p = ids.shape[0], len(table_shards)
    if len(outs) != p:
        raise VPError("one output per shard")
    dtype = table_shards[0].dtype
    st = load_library().vp_embed_fwd_group(
        _ptrs(table_shards, "table_shards", (dtype,), (Vs, h)), _ptr(ids, "ids", (torch.int64,), (N,)), p, N, h, Vs,
        shard_offset, _dtype_code(table_shards[0]), _ptrs(outs, "outs", (dtype,), (N, h)), _stream(stream))
    _check(st, "vp_embed_fwd_group")


def vp_embed_bwd_group(grad_out, ids, shard_offset: int, dtable_shards, workspace, stream=None) -> None:
    """vp_embed_bwd for consecutive shards of equal size in one call; shard_offset is that of the first."""
    N, h = grad_out.shape
    Vs = dtable_shards[0].shape[0]
    wp, wb = _ws(workspace)
    st = load_library().vp_embed_bwd_group(
        _ptr(grad_out, "grad_out"), _ptr(ids, "ids", (torch.int64,), (N,)), len(dtable_shards), N, h, Vs, shard_offset,
        _dtype_code(grad_out), _ptrs(dtable_shards, "dtable_shards", (torch.float32,), (Vs, h)), wp, wb, _stream(stream))
    _check(st, "vp_embed_bwd_group")


def _on_current_device(ts) -> None:
    """Refuses tensors of another device than the current one, whose stream the call would go to."""
    if _HOST is not None and _HOST.on_current_device(ts):
        return
    here = torch.cuda.current_device()
    for t in ts:
        if t is not None and t.is_cuda and t.get_device() != here:
            raise VPError("tensor on %s, but the current device is cuda:%d" % (t.device, here))


def _norm_flags(post: bool, center: bool) -> int:
    return (VP_NORM_POST if post else 0) | (VP_NORM_CENTER if center else 0)


def _gate_rows(gate) -> int:
    if gate is None:
        return 0
    if gate.dim() != 2 or gate.shape[0] == 0:
        raise VPError("gate must be [rows, h], with a row at least")
    return gate.shape[0]


def vp_block_norm_fwd(x, y, H, *, r=None, stats=None, gate=None, w=None, b=None, w_post=None, b_post=None, scale: float = 1.0,
                      eps: float = 1e-5, post: bool = False, center: bool = False, stream=None) -> None:
    """The norms around a block: u = norm(y) (post) or y, r = x + scale * gate * u, H = norm(r); RMS norms, or layer norms with
    center=True.  y=None: H = norm(x) alone.  r, stats ([4, N], for the backward call) and every vector may be None."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.block_norm_fwd(_ADDRESS["vp_block_norm_fwd"], x, y, H, r, stats, gate, w, b, w_post, b_post, scale, eps,
                                  _norm_flags(post, center), stream)
        if st is not None:      # the call was made: whatever it returned, not once more
            _check(st, "vp_block_norm_fwd")
            return
    if x.dim() != 2:
        raise VPError("x must be [N, h]")
    N, h = x.shape
    dt = _dtype_code(x)
    same = (torch.float32,) if dt == VP_F32 else _BF16_LIKE
    rows = _gate_rows(gate)
    _on_current_device((x, y, H, r, stats, gate, w, b, w_post, b_post))
    st = load_library().vp_block_norm_fwd(
        _ptr(x, "x"), _ptr(y, "y", same, (N, h)), _ptr(gate, "gate", same, (rows, h)), rows,
        _ptr(w_post, "w_post", same, (h,)), _ptr(b_post, "b_post", same, (h,)), _ptr(w, "w", same, (h,)),
        _ptr(b, "b", same, (h,)), N, h, dt, _norm_flags(post, center), scale, eps, _ptr(r, "r", same, (N, h)),
        _ptr(H, "H", same, (N, h)), _ptr(stats, "stats", (torch.float32,), (4, N)), _stream(stream))
    _check(st, "vp_block_norm_fwd")


def vp_block_norm_bwd_workspace_bytes(N: int, h: int, gate_rows: int = 0, post: bool = False) -> int:
    n = load_library().vp_block_norm_bwd_workspace_bytes(N, h, gate_rows, _norm_flags(post, False))
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_block_norm_bwd_workspace_bytes: invalid arguments")
    return n


def vp_block_norm_bwd(dH, r, y, stats, *, dx, dy=None, dr=None, gate=None, w=None, w_post=None, b_post=None, scale: float = 1.0,
                      post: bool = False, center: bool = False, dgate=None, dw=None, db=None, dw_post=None, db_post=None,
                      workspace=None, stream=None) -> None:
    """The gradients of vp_block_norm_fwd, from its r (x where y was None) and stats.  dH is fp32 or of the type of r; dr, dx
    and dy are of one type, fp32 or that of r; the parameters' gradients are fp32, and None where they are not wanted."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.block_norm_bwd(_ADDRESS["vp_block_norm_bwd"], dH, r, y, stats, dx, dy, dr, gate, w, w_post, b_post, scale,
                                  _norm_flags(post, center), dgate, dw, db, dw_post, db_post, workspace, stream)
        if st is not None:      # the call was made: whatever it returned, not once more
            _check(st, "vp_block_norm_bwd")
            return
    if r.dim() != 2:
        raise VPError("r must be [N, h]")
    N, h = r.shape
    dt, dH_dt, grad_dt = _dtype_code(r), _dtype_code(dH), _dtype_code(dx)
    f = (torch.float32,)
    same = f if dt == VP_F32 else _BF16_LIKE
    grad = f if grad_dt == VP_F32 else _BF16_LIKE
    rows = _gate_rows(gate)
    _on_current_device((dH, r, y, stats, dx, dy, dr, gate, w, w_post, b_post, dgate, dw, db, dw_post, db_post, workspace))
    wp, wb = _ws(workspace)
    st = load_library().vp_block_norm_bwd(
        _ptr(dH, "dH", None, (N, h)), dH_dt, _ptr(dr, "dr", grad, (N, h)), _ptr(r, "r"), _ptr(y, "y", same, (N, h)),
        _ptr(gate, "gate", same, (rows, h)), rows, _ptr(w_post, "w_post", same, (h,)), _ptr(b_post, "b_post", same, (h,)),
        _ptr(w, "w", same, (h,)), _ptr(stats, "stats", f, (4, N)), N, h, dt, _norm_flags(post, center), scale, grad_dt,
        _ptr(dx, "dx", grad, (N, h)), _ptr(dy, "dy", grad, (N, h)), _ptr(dgate, "dgate", f, (rows, h)),
        _ptr(dw_post, "dw_post", f, (h,)), _ptr(db_post, "db_post", f, (h,)), _ptr(dw, "dw", f, (h,)), _ptr(db, "db", f, (h,)),
        wp, wb, _stream(stream))
    _check(st, "vp_block_norm_bwd")


class GradientArguments:
    """The host arrays that the calls over many gradients take: addresses and sizes of the tensors, which it keeps alive.  A
    tensor that moved or changed its size or type since is refused by every call with these arguments (a captured call has the
    addresses for good).  outs: where the clipped gradients go, None = in place."""

    def __init__(self, grads, outs=None):
        self.grads, self.outs = list(grads), None if outs is None else list(outs)
        n = self.n = len(self.grads)
        if outs is not None and len(self.outs) != n:
            raise VPError("outs: one tensor per gradient")
        ptrs = [_ptr(g, "grads") for g in self.grads]
        counts = [g.numel() for g in self.grads]
        dts = [_dtype_code(g) for g in self.grads]
        out_ptrs = None if outs is None else [_ptr(o, "outs", (g.dtype,), g.shape) for g, o in zip(self.grads, self.outs)]
        if len({t.get_device() for t in self.grads + (self.outs or [])}) > 1:
            raise VPError("gradients of one call are on one device")
        self.first = self.grads[0] if n else None
        self.ptrs, self.counts, self.dts = (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*dts)
        self.out_ptrs = None if outs is None else (ctypes.c_void_p * n)(*out_ptrs)
        # What is written is written in no order: outputs are apart from one another and from all gradients but their own.
        sizes = [c * (2 if d == VP_BF16 else 4) for c, d in zip(counts, dts)]
        spans = [(p, z, True) for p, z in zip(ptrs if outs is None else out_ptrs, sizes) if z]
        if outs is not None:
            spans += [(p, z, False) for p, z, o in zip(ptrs, sizes, out_ptrs) if z and p != o]
        read = written = 0      # ends of the spans before
        self.overlap = False
        for start, size, is_written in sorted(spans):
            self.overlap |= start < written or (is_written and start < read)
            if is_written:
                written = max(written, start + size)
            else:
                read = max(read, start + size)

    def unchanged(self, outs: bool = True) -> bool:
        """Whether the tensors (with their outputs) are where and what they were when this was made."""
        return _unchanged(self.grads, self.ptrs, self.counts, self.dts) and (
            not outs or self.outs is None or _unchanged(self.outs, self.out_ptrs, self.counts, self.dts))


def _unchanged(ts, ptrs, counts, dts) -> bool:
    if _HOST is not None and _HOST.unchanged(ts, ptrs, counts, dts):
        return True
    kinds = {VP_F32: (torch.float32,), VP_BF16: _BF16_LIKE}
    return len(ts) == len(ptrs) and all(
        t.numel() == n and t.dtype in kinds[d] and t.is_contiguous() and (n == 0 or t.data_ptr() == p)
        for t, p, n, d in zip(ts, ptrs, counts, dts))


def _grad_call(name: str, a, norm, workspace, stream, max_norm=None):
    if not a.unchanged(outs=max_norm is not None):
        raise VPError("%s: a tensor has moved or changed its size or type since the arguments were made" % name)
    if max_norm is not None and a.overlap:
        raise VPError("%s: an output shares memory with another one or with another gradient" % name)
    lib = load_library()
    _on_current_device((a.first, norm, workspace))
    wp, wb = _ws(workspace)
    np, s = _ptr(norm, "norm", (torch.float32,), (1,)), _stream(stream)
    if max_norm is None:
        st = lib.vp_grad_norm(a.ptrs, a.counts, a.dts, a.n, np, wp, wb, s)
    else:
        st = getattr(lib, name)(a.ptrs, a.counts, a.dts, a.n, a.out_ptrs, max_norm, np, wp, wb, s)
    _check(st, name)


def _gradients(grads, outs=None) -> GradientArguments:
    if not isinstance(grads, GradientArguments):
        return GradientArguments(grads, outs)
    if outs is not None:
        raise VPError("outs belong to the GradientArguments")
    return grads


def vp_grad_workspace_bytes(n: int) -> int:
    b = load_library().vp_grad_workspace_bytes(n)
    if b == ctypes.c_size_t(-1).value:
        raise VPError("vp_grad_workspace_bytes: invalid arguments")
    return b


def vp_grad_norm(grads, norm, workspace, stream=None) -> None:
    """norm[0] = the 2-norm of all gradients together.  grads: tensors of fp32 or bf16, or GradientArguments made of them once."""
    _grad_call("vp_grad_norm", _gradients(grads), norm, workspace, stream)


def vp_grad_clip(grads, max_norm: float, norm, workspace, outs=None, stream=None) -> None:
    """vp_grad_norm, and every gradient times max_norm / norm where the norm exceeds max_norm: in place, or into outs.  A norm
    that is not finite leaves the gradients as they are."""
    _grad_call("vp_grad_clip", _gradients(grads, outs), norm, workspace, stream, float(max_norm))


def vp_grad_scale(grads, max_norm: float, norm, workspace, outs=None, stream=None) -> None:
    """vp_grad_clip with a norm that is known already."""
    _grad_call("vp_grad_scale", _gradients(grads, outs), norm, workspace, stream, float(max_norm))


def vp_i8_row_stride(h: int) -> int:
    """Bytes of a row of h elements in 8-bit integers."""
    n = load_library().vp_i8_row_stride(h)
    if n < 0:
        raise VPError("vp_i8_row_stride: invalid arguments")
    return n


def vp_quantize_rows(x, q, scales, stream=None) -> None:
    """Rows of x [N, h] in 8-bit integers: scales [N] = max |x| / 127, q [N, vp_i8_row_stride(h)] = 127 x / max |x| to the
    nearest integer, zero behind column h."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.quantize_rows(_ADDRESS["vp_quantize_rows"], x, q, scales, stream)
        if st is not None:      # the call was made
            _check(st, "vp_quantize_rows")
            return
    if x.dim() != 2:
        raise VPError("x must be [N, h]")
    N, h = x.shape
    _on_current_device((x, q, scales))
    st = load_library().vp_quantize_rows(
        _ptr(x, "x"), N, h, _dtype_code(x), _ptr(q, "q", (torch.int8,), (N, vp_i8_row_stride(h))),
        _ptr(scales, "scales", (torch.float32,), (N,)), _stream(stream))
    _check(st, "vp_quantize_rows")


def vp_output_i8_workspace_bytes(N: int, rows) -> int:
    n = load_library().vp_output_i8_workspace_bytes(len(rows), N, _i64s(rows))
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_output_i8_workspace_bytes: invalid arguments")
    return n


def _logits_code(logits_out) -> int:
    if logits_out is None:
        return VP_BF16
    if not logits_out or any(t.dtype != logits_out[0].dtype for t in logits_out):
        raise VPError("logits_out: a tensor for each shard, of one type")
    return _dtype_code(logits_out[0])


def vp_output_fwd_i8(H, H_scales, W_shard, W_scales, labels, shard_offset: int, local_max, local_sumexp, local_target,
                     logits_out=None, workspace=None, stream=None) -> None:
    """vp_output_fwd from 8-bit integers H [N, k] and W_shard [Vs, k] and their scales (vp_quantize_rows); the logits are bf16 or
    fp32, by the type of logits_out."""
    if H.dim() != 2 or W_shard.dim() != 2:
        raise VPError("H must be [N, k] and W_shard [Vs, k]")
    N, k = H.shape
    Vs = W_shard.shape[0]
    i8, f = (torch.int8,), (torch.float32,)
    logits = None if logits_out is None else [logits_out]
    dt = _logits_code(logits)
    _on_current_device((H, H_scales, W_shard, W_scales, labels, local_max, local_sumexp, local_target, logits_out, workspace))
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd_i8(
        _ptr(H, "H", i8), _ptr(H_scales, "H_scales", f, (N,)), _ptr(W_shard, "W_shard", i8, (Vs, k)),
        _ptr(W_scales, "W_scales", f, (Vs,)), _ptr(labels, "labels", (torch.int64,), (N,)), N, k, Vs, shard_offset, dt,
        VP_SAVE_LOGITS if logits_out is not None else 0, _ptr(local_max, "local_max", f, (N,)),
        _ptr(local_sumexp, "local_sumexp", f, (N,)), _ptr(local_target, "local_target", f, (N,)),
        _ptr(logits_out, "logits_out", None, (N, Vs)), wp, wb, _stream(stream))
    _check(st, "vp_output_fwd_i8")


def vp_output_fwd_i8_group(H, H_scales, W_shards, W_scales, labels, shard_offsets, local_max, local_sumexp, local_target,
                           logits_out=None, workspace=None, stream=None) -> None:
    """vp_output_fwd_i8 for several shards on this device in one call; the statistics are [p, N]."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.output_fwd_i8_group(_ADDRESS["vp_output_fwd_i8_group"], H, H_scales, W_shards, W_scales, labels, shard_offsets,
                                       local_max, local_sumexp, local_target, logits_out, workspace, stream)
        if st is not None:      # the call was made
            _check(st, "vp_output_fwd_i8_group")
            return
    if H.dim() != 2 or any(w.dim() != 2 for w in W_shards):
        raise VPError("H must be [N, k] and W_shards [rows, k]")
    N, k = H.shape
    p = len(W_shards)
    if len(shard_offsets) != p:
        raise VPError("one offset per shard")
    rows = [int(w.shape[0]) for w in W_shards]
    i8, f = (torch.int8,), (torch.float32,)
    dt = _logits_code(logits_out)
    _on_current_device((H, H_scales, *W_shards, *W_scales, labels, local_max, local_sumexp, local_target, *(logits_out or ()),
                        workspace))
    wp, wb = _ws(workspace)
    st = load_library().vp_output_fwd_i8_group(
        _ptr(H, "H", i8), _ptr(H_scales, "H_scales", f, (N,)), _each(W_shards, "W_shards", i8, [(n, k) for n in rows]),
        _each(W_scales, "W_scales", f, [(n,) for n in rows]), _i64s(rows), _i64s(shard_offsets), p,
        _ptr(labels, "labels", (torch.int64,), (N,)), N, k, dt, VP_SAVE_LOGITS if logits_out is not None else 0,
        _ptr(local_max, "local_max", f, (p, N)), _ptr(local_sumexp, "local_sumexp", f, (p, N)),
        _ptr(local_target, "local_target", f, (p, N)), _each(logits_out, "logits_out", None, [(N, n) for n in rows]),
        wp, wb, _stream(stream))
    _check(st, "vp_output_fwd_i8_group")


def vp_logits_stats_workspace_bytes(N: int, rows) -> int:
    n = load_library().vp_logits_stats_workspace_bytes(len(rows), N, _i64s(rows))
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_logits_stats_workspace_bytes: invalid arguments")
    return n


def vp_logits_stats(logits, global_max, global_sumexp, workspace, stream=None) -> None:
    """Row maxima and row sums of exponentials [N] of the shards' logits ([N, rows] each) as they are stored: what
    vp_verify_drafts takes."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.logits_stats(_ADDRESS["vp_logits_stats"], logits, global_max, global_sumexp, workspace, stream)
        if st is not None:      # the call was made
            _check(st, "vp_logits_stats")
            return
    if not logits or any(t.dim() != 2 for t in logits):
        raise VPError("logits must be [N, rows], a shard at least")
    N, rows = logits[0].shape[0], [int(t.shape[1]) for t in logits]
    f = (torch.float32,)
    _on_current_device((*logits, global_max, global_sumexp, workspace))
    wp, wb = _ws(workspace)
    st = load_library().vp_logits_stats(
        _each(logits, "logits", (logits[0].dtype,), [(N, n) for n in rows]), _i64s(rows), len(rows), _dtype_code(logits[0]), N,
        _ptr(global_max, "global_max", f, (N,)), _ptr(global_sumexp, "global_sumexp", f, (N,)), wp, wb, _stream(stream))
    _check(st, "vp_logits_stats")


def vp_verify_workspace_bytes(sequences: int, V: int) -> int:
    n = load_library().vp_verify_workspace_bytes(sequences, V)
    if n == ctypes.c_size_t(-1).value:
        raise VPError("vp_verify_workspace_bytes: invalid arguments")
    return n


def vp_verify_drafts(logits, shard_offsets, global_max, global_sumexp, drafts, starts, uniforms, accepted, tokens, workspace, *,
                     draft_logits=None, draft_max=None, draft_sumexp=None, stream=None) -> None:
    """Verification of drafted tokens over the shards' logits ([N, rows] each) and the draw of the token behind them.  The
    statistics are those of exactly these logits (vp_logits_stats).  Sequence b has the rows starts[b] .. starts[b + 1] - 1, one for each draft and a last one; draft_*: the draft model's, row by row, or
    None (drafts that no model drew).  accepted [sequences] int32, tokens [N]: accepted drafts, the next token, -1 behind it."""
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if _HOST is not None:
        st = _HOST.verify_drafts(_ADDRESS["vp_verify_drafts"], logits, shard_offsets, global_max, global_sumexp, drafts, starts,
                                 uniforms, accepted, tokens, workspace, draft_logits, draft_max, draft_sumexp, stream)
        if st is not None:      # the call was made
            _check(st, "vp_verify_drafts")
            return
    if not logits or any(t.dim() != 2 for t in logits):
        raise VPError("logits must be [N, rows], a shard at least")
    N, p = logits[0].shape[0], len(logits)
    if len(shard_offsets) != p:
        raise VPError("one offset per shard")
    rows = [int(t.shape[1]) for t in logits]
    shapes, dtype = [(N, n) for n in rows], (logits[0].dtype,)
    if starts.dim() != 1 or starts.shape[0] < 2:
        raise VPError("starts must be [sequences + 1], a sequence at least")
    S = starts.shape[0] - 1
    f, ids = (torch.float32,), (torch.int64,)
    _on_current_device((*logits, global_max, global_sumexp, drafts, starts, uniforms, accepted, tokens, workspace,
                        *(draft_logits or ()), draft_max, draft_sumexp))
    wp, wb = _ws(workspace)
    st = load_library().vp_verify_drafts(
        _each(logits, "logits", dtype, shapes), _i64s(rows), _i64s(shard_offsets), p, _dtype_code(logits[0]),
        _ptr(global_max, "global_max", f, (N,)), _ptr(global_sumexp, "global_sumexp", f, (N,)),
        _each(draft_logits, "draft_logits", dtype, shapes), _ptr(draft_max, "draft_max", f, (N,)),
        _ptr(draft_sumexp, "draft_sumexp", f, (N,)), _ptr(drafts, "drafts", ids, (N,)), _ptr(starts, "starts", ids),
        _ptr(uniforms, "uniforms", f, (N,)), N, S, _ptr(accepted, "accepted", (torch.int32,), (S,)),
        _ptr(tokens, "tokens", ids, (N,)), wp, wb, _stream(stream))
    _check(st, "vp_verify_drafts")


def vp_profile_mfma_loop(operands, out, iters: int, blocks: int, stream=None) -> None:
    """Measurement aid: back-to-back MFMAs on register operands (see include/vp.h)."""
    if operands.numel() * operands.element_size() < 8 * 256 * 16 or out.numel() < blocks * 256:
        raise VPError("vp_profile_mfma_loop: buffers too small")
    st = load_library().vp_profile_mfma_loop(_ptr(operands, "operands", _BF16_LIKE), _ptr(out, "out", (torch.float32,)),
                                             iters, blocks, _stream(stream))
    _check(st, "vp_profile_mfma_loop")


def vp_profile_mfma_variant(operands, out, iters: int, blocks: int, variant: int, stream=None) -> float:
    """Measurement aid: the MFMA loop in another instruction shape / issue order (see include/vp.h).
    Returns the flop count of the launch."""
    lib = load_library()
    if operands.numel() * operands.element_size() < 32 * 256 * 16 or out.numel() < blocks * 256:
        raise VPError("vp_profile_mfma_variant: buffers too small")
    st = lib.vp_profile_mfma_variant(_ptr(operands, "operands", _BF16_LIKE), _ptr(out, "out", (torch.float32,)),
                                     iters, blocks, variant, _stream(stream))
    _check(st, "vp_profile_mfma_variant")
    return lib.vp_profile_mfma_variant_flops(variant) * blocks * 4 * iters


def vp_profile_mfma_variant_count() -> int:
    return load_library().vp_profile_mfma_variant_count()


def vp_profile_force_generic_gemm(on: bool) -> None:
    """Test switch: route every bf16 product through the generic GEMM kernel."""
    _check(load_library().vp_profile_force_generic_gemm(1 if on else 0), "vp_profile_force_generic_gemm")


def vp_profile_gemm_trace(buffer, kernel: Optional[str] = None) -> None:
    """Measurement aid: phase stamps of the fast GEMM kernel into `buffer` (a GPU tensor of int64; None = off),
    optionally only for launches timed under the kernel name `kernel` (see vp_profile_read)."""
    lib = load_library()
    if buffer is None:
        _check(lib.vp_profile_gemm_trace(None, 0, -1), "vp_profile_gemm_trace")
        return
    kid = -1
    if kernel is not None:
        names = [lib.vp_profile_kernel_name(i).decode() for i in range(lib.vp_profile_kernel_count())]
        if kernel not in names:
            raise VPError("unknown kernel name %r" % kernel)
        kid = names.index(kernel)
    _check(lib.vp_profile_gemm_trace(_ptr(buffer, "buffer", (torch.int64,)), buffer.numel() * 8, kid),
           "vp_profile_gemm_trace")


def vp_profile_enable(on: bool) -> None:
    _check(load_library().vp_profile_enable(1 if on else 0), "vp_profile_enable")


def vp_profile_read() -> dict:
    """{kernel name: (total milliseconds, launches)} since the last read; clears the records."""
    lib = load_library()
    n = lib.vp_profile_kernel_count()
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(lib.vp_profile_read(ms, cnt, n), "vp_profile_read")
    return {lib.vp_profile_kernel_name(i).decode(): (ms[i], cnt[i]) for i in range(n) if cnt[i] > 0}
