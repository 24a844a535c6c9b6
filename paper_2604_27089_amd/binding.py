"""ctypes binding of libsp_hotpath.so: argument marshalling only.

Function names and argument order mirror include/sp_hotpath.h.  Tensors are
torch CUDA(HIP) tensors used purely as device memory; the stream is torch's
current stream unless one is given.  There is no fallback: a missing library
raises ImportError at first use, and a non-zero status raises SpError.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# SP_HOTPATH_LIB points at another build of the same library (e.g. an experimental variant).
LIB_PATH = os.environ.get("SP_HOTPATH_LIB") or os.path.join(_HERE, "libsp_hotpath.so")

SP_OK, SP_ERR_NULL, SP_ERR_SHAPE, SP_ERR_UNSUPPORTED, SP_ERR_WORKSPACE, SP_ERR_ALIGN, SP_ERR_LAUNCH = range(7)

EXPORTS = (
    "sp_status_str", "sp_abi_version", "sp_pack_seq_to_head", "sp_unpack_head_to_seq", "sp_attn_fwd",
    "sp_attn_bwd_workspace_bytes", "sp_attn_varlen_fwd_workspace_bytes", "sp_attn_bwd", "sp_attn_bwd_stages",
    "sp_attn_varlen_fwd", "sp_attn_varlen_bwd", "sp_attn_varlen_fwd_static", "sp_varlen_check_cu_seqlens", "sp_attn_fwd_seqlayout", "sp_attn_bwd_seqlayout",
    "sp_attn_block_fwd", "sp_attn_merge", "sp_attn_block_bwd_workspace_bytes", "sp_attn_block_bwd",
    "sp_rmsnorm_bwd_workspace_bytes", "sp_rmsnorm_fwd", "sp_rmsnorm_bwd", "sp_rope", "sp_swiglu_fwd", "sp_swiglu_bwd",
    "sp_rmsnorm_fp8_fwd", "sp_rmsnorm_res_bwd", "sp_fp8_quant", "sp_fp8_matmul",
    "sp_fp8_matmul_workspace_bytes", "sp_fp8_matmul_split",
)


class SpError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_str(code)}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load the HIP library (once).  Fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    _lib = open_library(LIB_PATH)
    return _lib


def open_library(path: str) -> ctypes.CDLL:
    """Load a build of the library and declare its entry points (tests compare two builds through this)."""
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2604_27089_amd.build` "
                          "(there is no CPU or PyTorch fallback)")
    L = ctypes.CDLL(path)
    c = ctypes
    vp, i64, i32, f32, sz = c.c_void_p, c.c_int64, c.c_int32, c.c_float, c.c_size_t
    L.sp_status_str.restype = c.c_char_p; L.sp_status_str.argtypes = [c.c_int]
    L.sp_abi_version.restype = i32; L.sp_abi_version.argtypes = []
    for name in ("sp_pack_seq_to_head", "sp_unpack_head_to_seq"):
        f = getattr(L, name); f.restype = c.c_int
        f.argtypes = [vp, vp, i64, i64, i64, i64, i32, i32, vp]
    L.sp_attn_fwd.restype = c.c_int
    L.sp_attn_fwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, i32, i32, f32, vp]
    L.sp_attn_bwd_workspace_bytes.restype = sz
    L.sp_attn_bwd_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i32]
    L.sp_attn_varlen_fwd_workspace_bytes.restype = sz
    L.sp_attn_varlen_fwd_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    L.sp_attn_bwd.restype = c.c_int
    L.sp_attn_bwd.argtypes = [vp] * 10 + [sz, i64, i64, i32, i32, i32, f32, vp]
    L.sp_attn_bwd_stages.restype = c.c_int
    L.sp_attn_bwd_stages.argtypes = [vp] * 10 + [sz, i64, i64, i32, i32, i32, f32, i32, vp]
    L.sp_attn_fwd_seqlayout.restype = c.c_int
    L.sp_attn_fwd_seqlayout.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, f32, vp]
    L.sp_attn_bwd_seqlayout.restype = c.c_int
    L.sp_attn_bwd_seqlayout.argtypes = [vp] * 10 + [sz, i64, i64, i32, i32, i32, i32, f32, vp]
    L.sp_attn_block_fwd.restype = c.c_int
    L.sp_attn_block_fwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, i32, i64, f32, vp]
    L.sp_attn_merge.restype = c.c_int
    L.sp_attn_merge.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, i32, vp]
    L.sp_attn_block_bwd_workspace_bytes.restype = sz
    L.sp_attn_block_bwd_workspace_bytes.argtypes = [i64, i64, i64, i32, i32, i32]
    L.sp_attn_block_bwd.restype = c.c_int
    L.sp_attn_block_bwd.argtypes = [vp] * 10 + [sz, i64, i64, i64, i32, i32, i32, i64, f32, i32, vp]
    L.sp_attn_varlen_fwd.restype = c.c_int
    L.sp_attn_varlen_fwd.argtypes = [vp] * 6 + [i32, i32, i64, i32, i32, i32, f32, vp, sz, vp]
    L.sp_attn_varlen_fwd_static.restype = c.c_int
    L.sp_attn_varlen_fwd_static.argtypes = [vp] * 6 + [i32, i32, i64, i32, i32, i32, f32, vp]
    L.sp_varlen_check_cu_seqlens.restype = c.c_int
    L.sp_varlen_check_cu_seqlens.argtypes = [vp, i32, i64, vp, vp]
    L.sp_attn_varlen_bwd.restype = c.c_int
    L.sp_attn_varlen_bwd.argtypes = [vp] * 10 + [i32, i32, i64, i32, i32, i32, f32, vp, sz, vp]
    L.sp_rmsnorm_bwd_workspace_bytes.restype = sz
    L.sp_rmsnorm_bwd_workspace_bytes.argtypes = [i64, i32]
    L.sp_rmsnorm_fwd.restype = c.c_int
    L.sp_rmsnorm_fwd.argtypes = [vp, vp, vp, vp, i64, i32, f32, vp]
    L.sp_rmsnorm_bwd.restype = c.c_int
    L.sp_rmsnorm_bwd.argtypes = [vp] * 7 + [sz, i64, i32, vp]
    L.sp_rope.restype = c.c_int
    L.sp_rope.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, vp]
    L.sp_swiglu_fwd.restype = c.c_int
    L.sp_swiglu_fwd.argtypes = [vp, vp, vp, i64, vp]
    L.sp_swiglu_bwd.restype = c.c_int
    L.sp_swiglu_bwd.argtypes = [vp] * 5 + [i64, vp]
    L.sp_rmsnorm_fp8_fwd.restype = c.c_int
    L.sp_rmsnorm_fp8_fwd.argtypes = [vp] * 7 + [i64, i32, f32, vp]
    L.sp_rmsnorm_res_bwd.restype = c.c_int
    L.sp_rmsnorm_res_bwd.argtypes = [vp] * 8 + [sz, i64, i32, vp]
    L.sp_fp8_quant.restype = c.c_int
    L.sp_fp8_quant.argtypes = [vp] * 7 + [i64, i32, i32, vp]
    L.sp_fp8_matmul.restype = c.c_int
    L.sp_fp8_matmul.argtypes = [vp] * 5 + [i64, i64, i64, i32, i32, i32, vp]
    L.sp_fp8_matmul_workspace_bytes.restype = sz
    L.sp_fp8_matmul_workspace_bytes.argtypes = [i64, i64, i64]
    L.sp_fp8_matmul_split.restype = c.c_int
    L.sp_fp8_matmul_split.argtypes = [vp] * 6 + [sz, i64, i64, i64, i32, vp]
    return L


def status_str(code: int) -> str:
    return lib().sp_status_str(int(code)).decode()


def _check(code: int, where: str):
    if code != SP_OK:
        raise SpError(code, where)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous"
    return t.data_ptr()  # the declared argument types make a pointer of it


# The raw handle of the current stream, without the Stream object that torch.cuda.current_stream() builds around it; through
# that object where torch does not have the lookup (a build without a GPU backend, which can still import this module).
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)
if _current_raw_stream is None or _current_device is None:
    _current_device, _current_raw_stream = (lambda: None), (lambda device: torch.cuda.current_stream().cuda_stream)


def _stream(stream) -> int:
    return _current_raw_stream(_current_device()) if stream is None else stream.cuda_stream


def _expect(t: torch.Tensor, shape, dtype, name: str):
    """The C ABI sees pointers only: extents and element types are checked here, before any launch."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _new(stream, shape, dtype, device) -> torch.Tensor:
    """A tensor allocated by a wrapper.  torch's allocator ties a block to the stream that is current when it is allocated, and may
    hand out one that work queued there still uses.  When the kernels go to another stream the block comes from that one, and
    is marked as in use on the caller's, whose work may still read it when the caller lets go of it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    caller = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(caller)
    return t


def _attn_shapes(q, k, v, lse_shape, kv_like_q_dims: int, o=None, lse=None, do=None, dq=None, dk=None, dv=None):
    """bf16 everywhere, k/v agree, the leading `kv_like_q_dims` extents of k equal q's, the head dim agrees."""
    bf = torch.bfloat16
    _expect(q, q.shape, bf, "q")
    kshape = tuple(q.shape[:kv_like_q_dims]) + tuple(k.shape[kv_like_q_dims:-1]) + (q.shape[-1],)
    _expect(k, kshape, bf, "k")
    _expect(v, k.shape, bf, "v")
    for t, like, name in ((o, q, "o"), (do, q, "dO"), (dq, q, "dq"), (dk, k, "dk"), (dv, k, "dv")):
        if t is not None:
            _expect(t, like.shape, bf, name)
    if lse is not None:
        _expect(lse, lse_shape, torch.float32, "lse")


# --------------------------------------------------------------------------- re-layout
def sp_pack_seq_to_head(x: torch.Tensor, P: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x [B, S_l, H, D] -> out [B, P*S_l, H/P, D]."""
    B, S_l, H, D = x.shape
    shape = (B, P * S_l, H // P if P > 0 else H, D)
    if out is None:
        out = _new(stream, shape, x.dtype, x.device)
    elif P > 0 and H % P == 0:
        _expect(out, shape, x.dtype, "out")
    _check(lib().sp_pack_seq_to_head(_ptr(x), _ptr(out), B, S_l, H, D, P, x.element_size(), _stream(stream)),
           "sp_pack_seq_to_head")
    return out


def sp_unpack_head_to_seq(y: torch.Tensor, P: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """y [B, P*S_l, h, D] -> out [B, S_l, P*h, D]."""
    B, PS, h, D = y.shape
    if P <= 0 or PS % P != 0:
        raise ValueError(f"y has {PS} rows, not a multiple of P = {P}")
    S_l, H = PS // P, h * P
    if out is None:
        out = _new(stream, (B, S_l, H, D), y.dtype, y.device)
    else:
        _expect(out, (B, S_l, H, D), y.dtype, "out")
    _check(lib().sp_unpack_head_to_seq(_ptr(y), _ptr(out), B, S_l, H, D, P, y.element_size(), _stream(stream)),
           "sp_unpack_head_to_seq")
    return out


# --------------------------------------------------------------------------- attention
def sp_attn_fwd(q, k, v, softmax_scale: float = 0.0, o=None, lse=None, stream=None):
    """q [B,S,Hq,D], k,v [B,S,Hkv,D] bf16 -> (o [B,S,Hq,D] bf16, lse [B,Hq,S] fp32)."""
    B, S, Hq, D = q.shape
    Hkv = k.shape[2]
    _attn_shapes(q, k, v, (B, Hq, S), 2, o=o, lse=lse)
    o = _new(stream, q.shape, q.dtype, q.device) if o is None else o
    lse = _new(stream, (B, Hq, S), torch.float32, q.device) if lse is None else lse
    _check(lib().sp_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, S, Hq, Hkv, D,
                             float(softmax_scale), _stream(stream)), "sp_attn_fwd")
    return o, lse


def sp_attn_bwd_workspace_bytes(B, S_or_T, Hq, Hkv, D, n_docs=0) -> int:
    return int(lib().sp_attn_bwd_workspace_bytes(B, S_or_T, Hq, Hkv, D, n_docs))


def sp_attn_varlen_fwd_workspace_bytes(T, Hq, Hkv, D, n_docs) -> int:
    return int(lib().sp_attn_varlen_fwd_workspace_bytes(T, Hq, Hkv, D, n_docs))


def _workspace(nbytes: int, device, stream=None) -> torch.Tensor:
    return _new(stream, (max(int(nbytes), 256),), torch.uint8, device)


def _grads(stream, q, k, v, dq, dk, dv):
    return (_new(stream, q.shape, q.dtype, q.device) if dq is None else dq,
            _new(stream, k.shape, k.dtype, k.device) if dk is None else dk,
            _new(stream, v.shape, v.dtype, v.device) if dv is None else dv)


def sp_attn_bwd(q, k, v, o, lse, do, softmax_scale: float = 0.0, dq=None, dk=None, dv=None,
                workspace=None, stream=None):
    """Returns (dq, dk, dv), bf16, shaped like q, k, v."""
    B, S, Hq, D = q.shape
    Hkv = k.shape[2]
    _attn_shapes(q, k, v, (B, Hq, S), 2, o=o, lse=lse, do=do, dq=dq, dk=dk, dv=dv)
    dq, dk, dv = _grads(stream, q, k, v, dq, dk, dv)
    if workspace is None:
        workspace = _workspace(sp_attn_bwd_workspace_bytes(B, S, Hq, Hkv, D, 0), q.device, stream)
    _check(lib().sp_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do), _ptr(dq), _ptr(dk),
                             _ptr(dv), _ptr(workspace), workspace.numel() * workspace.element_size(), B, S, Hq,
                             Hkv, D, float(softmax_scale), _stream(stream)), "sp_attn_bwd")
    return dq, dk, dv


SP_BWD_STAGE_DELTA, SP_BWD_STAGE_DKDV, SP_BWD_STAGE_DQ, SP_BWD_STAGE_ALL = 1, 2, 4, 7


def sp_attn_bwd_stages(q, k, v, o, lse, do, dq, dk, dv, workspace, stages: int, softmax_scale: float = 0.0,
                       stream=None):
    """One or more stages of the backward (bit mask of SP_BWD_STAGE_*); buffers are the caller's."""
    B, S, Hq, D = q.shape
    Hkv = k.shape[2]
    _attn_shapes(q, k, v, (B, Hq, S), 2, o=o, lse=lse, do=do, dq=dq, dk=dk, dv=dv)
    _check(lib().sp_attn_bwd_stages(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do), _ptr(dq),
                                    _ptr(dk), _ptr(dv), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), B, S, Hq, Hkv, D,
                                    float(softmax_scale), int(stages), _stream(stream)), "sp_attn_bwd_stages")
    return dq, dk, dv


def _seq_heads(q, k, P: int):
    if P <= 0 or q.shape[2] % P != 0 or k.shape[2] % P != 0:
        raise ValueError(f"head counts {q.shape[2]} / {k.shape[2]} are not multiples of P = {P}")
    return q.shape[2] // P, k.shape[2] // P


def sp_attn_fwd_seqlayout(q, k, v, P: int, softmax_scale: float = 0.0, o=None, lse=None, stream=None):
    """Sequence-side tensors q [B,S_l,P*Hq,D], k,v [B,S_l,P*Hkv,D] -> (o [B,S_l,P*Hq,D], lse [B,Hq,P*S_l])."""
    B, S_l, _, D = q.shape
    Hq, Hkv = _seq_heads(q, k, P)
    _attn_shapes(q, k, v, (B, Hq, P * S_l), 2, o=o, lse=lse)
    o = _new(stream, q.shape, q.dtype, q.device) if o is None else o
    lse = _new(stream, (B, Hq, P * S_l), torch.float32, q.device) if lse is None else lse
    _check(lib().sp_attn_fwd_seqlayout(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, S_l, Hq, Hkv, D, P,
                                       float(softmax_scale), _stream(stream)), "sp_attn_fwd_seqlayout")
    return o, lse


def sp_attn_bwd_seqlayout(q, k, v, o, lse, do, P: int, softmax_scale: float = 0.0, dq=None, dk=None, dv=None,
                          workspace=None, stream=None):
    """Backward on sequence-side tensors; returns (dq, dk, dv) shaped like q, k, v."""
    B, S_l, _, D = q.shape
    Hq, Hkv = _seq_heads(q, k, P)
    _attn_shapes(q, k, v, (B, Hq, P * S_l), 2, o=o, lse=lse, do=do, dq=dq, dk=dk, dv=dv)
    dq, dk, dv = _grads(stream, q, k, v, dq, dk, dv)
    if workspace is None:
        workspace = _workspace(sp_attn_bwd_workspace_bytes(B, P * S_l, Hq, Hkv, D, 0), q.device, stream)
    _check(lib().sp_attn_bwd_seqlayout(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do), _ptr(dq),
                                       _ptr(dk), _ptr(dv), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), B, S_l, Hq, Hkv,
                                       D, P, float(softmax_scale), _stream(stream)), "sp_attn_bwd_seqlayout")
    return dq, dk, dv


def sp_attn_block_fwd(q, k, v, causal_offset: int, softmax_scale: float = 0.0, o=None, lse=None, stream=None):
    """q [B,Sq,Hq,D], k,v [B,Skv,Hkv,D]; row i sees keys j <= i + causal_offset -> (o, lse [B,Hq,Sq])."""
    B, Sq, Hq, D = q.shape
    Skv, Hkv = k.shape[1], k.shape[2]
    _attn_shapes(q, k, v, (B, Hq, Sq), 1, o=o, lse=lse)
    o = _new(stream, q.shape, q.dtype, q.device) if o is None else o
    lse = _new(stream, (B, Hq, Sq), torch.float32, q.device) if lse is None else lse
    _check(lib().sp_attn_block_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, Sq, Skv, Hq, Hkv, D,
                                   int(causal_offset), float(softmax_scale), _stream(stream)), "sp_attn_block_fwd")
    return o, lse


def sp_attn_merge(o_acc, lse_acc, o_blk, lse_blk, o_out=None, stream=None):
    """Folds (o_blk bf16, lse_blk) into the running (o_acc fp32 [B,S,Hq,D], lse_acc fp32 [B,Hq,S]) in place;
    also writes the merged O as bf16 into o_out if given."""
    B, S, Hq, D = o_acc.shape
    _expect(o_acc, (B, S, Hq, D), torch.float32, "o_acc")
    _expect(lse_acc, (B, Hq, S), torch.float32, "lse_acc")
    _expect(o_blk, (B, S, Hq, D), torch.bfloat16, "o_blk")
    _expect(lse_blk, (B, Hq, S), torch.float32, "lse_blk")
    if o_out is not None:
        _expect(o_out, (B, S, Hq, D), torch.bfloat16, "o_out")
    _check(lib().sp_attn_merge(_ptr(o_acc), _ptr(lse_acc), _ptr(o_blk), _ptr(lse_blk), _ptr(o_out), B, S, Hq, D,
                               _stream(stream)), "sp_attn_merge")
    return o_acc, lse_acc


def sp_attn_block_bwd_workspace_bytes(B, Sq, Skv, Hq, Hkv, D) -> int:
    return int(lib().sp_attn_block_bwd_workspace_bytes(B, Sq, Skv, Hq, Hkv, D))


def sp_attn_block_bwd(q, k, v, o, lse, do, causal_offset: int, softmax_scale: float = 0.0, dq=None, dk=None,
                      dv=None, workspace=None, stages: int = SP_BWD_STAGE_ALL, stream=None):
    """This block pair's shares (dq, dk, dv), from the final o, lse of the query rows."""
    B, Sq, Hq, D = q.shape
    Skv, Hkv = k.shape[1], k.shape[2]
    _attn_shapes(q, k, v, (B, Hq, Sq), 1, o=o, lse=lse, do=do, dq=dq, dk=dk, dv=dv)
    dq, dk, dv = _grads(stream, q, k, v, dq, dk, dv)
    if workspace is None:
        workspace = _workspace(sp_attn_block_bwd_workspace_bytes(B, Sq, Skv, Hq, Hkv, D), q.device, stream)
    _check(lib().sp_attn_block_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do), _ptr(dq), _ptr(dk),
                                   _ptr(dv), _ptr(workspace), workspace.numel() * workspace.element_size(), B, Sq,
                                   Skv, Hq, Hkv, D, int(causal_offset), float(softmax_scale), int(stages),
                                   _stream(stream)),
           "sp_attn_block_bwd")
    return dq, dk, dv


def _docs(cu_seqlens) -> int:
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise ValueError(f"cu_seqlens: expected a device int32 vector of n_docs + 1 entries, got "
                         f"{cu_seqlens.dtype} {tuple(cu_seqlens.shape)}")
    return cu_seqlens.numel() - 1


def sp_attn_varlen_fwd(q, k, v, cu_seqlens, max_seqlen: int = 0, softmax_scale: float = 0.0, o=None,
                       lse=None, workspace=None, stream=None):
    """q [T,Hq,D], k,v [T,Hkv,D]; cu_seqlens device int32 [n_docs+1] -> (o, lse [Hq,T])."""
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    n_docs = _docs(cu_seqlens)
    _attn_shapes(q, k, v, (Hq, T), 1, o=o, lse=lse)
    o = _new(stream, q.shape, q.dtype, q.device) if o is None else o
    lse = _new(stream, (Hq, T), torch.float32, q.device) if lse is None else lse
    if workspace is None:
        workspace = _workspace(sp_attn_varlen_fwd_workspace_bytes(T, Hq, Hkv, D, n_docs), q.device, stream)
    _check(lib().sp_attn_varlen_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens), n_docs,
                                    int(max_seqlen), T, Hq, Hkv, D, float(softmax_scale), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream)),
           "sp_attn_varlen_fwd")
    return o, lse


def sp_attn_varlen_fwd_static(q, k, v, cu_seqlens, o, lse, max_seqlen: int = 0, softmax_scale: float = 0.0, stream=None):
    """sp_attn_varlen_fwd on the library's own static scratch: allocates nothing, so o and lse are the caller's."""
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    n_docs = _docs(cu_seqlens)
    _attn_shapes(q, k, v, (Hq, T), 1, o=o, lse=lse)
    _check(lib().sp_attn_varlen_fwd_static(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(cu_seqlens), n_docs,
                                           int(max_seqlen), T, Hq, Hkv, D, float(softmax_scale), _stream(stream)),
           "sp_attn_varlen_fwd_static")
    return o, lse


def sp_varlen_check_cu_seqlens(cu_seqlens, T: int, flag=None, stream=None):
    """Debug aid: returns a device int32 tensor holding 0 if cu_seqlens is well formed for T rows, else a bit
    mask (1: cu[0] != 0, 2: decreasing somewhere, 4: cu[-1] != T).  Does not synchronise."""
    n_docs = _docs(cu_seqlens)
    flag = _new(stream, (1,), torch.int32, cu_seqlens.device) if flag is None else flag
    _expect(flag, (1,), torch.int32, "flag")
    _check(lib().sp_varlen_check_cu_seqlens(_ptr(cu_seqlens), n_docs, int(T), _ptr(flag), _stream(stream)),
           "sp_varlen_check_cu_seqlens")
    return flag


def sp_attn_varlen_bwd(q, k, v, o, lse, do, cu_seqlens, max_seqlen: int = 0, softmax_scale: float = 0.0,
                       dq=None, dk=None, dv=None, workspace=None, stream=None):
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    n_docs = _docs(cu_seqlens)
    _attn_shapes(q, k, v, (Hq, T), 1, o=o, lse=lse, do=do, dq=dq, dk=dk, dv=dv)
    dq, dk, dv = _grads(stream, q, k, v, dq, dk, dv)
    if workspace is None:
        workspace = _workspace(sp_attn_bwd_workspace_bytes(1, T, Hq, Hkv, D, n_docs), q.device, stream)
    _check(lib().sp_attn_varlen_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do), _ptr(dq),
                                    _ptr(dk), _ptr(dv), _ptr(cu_seqlens), n_docs, int(max_seqlen), T, Hq,
                                    Hkv, D, float(softmax_scale), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream)),
           "sp_attn_varlen_bwd")
    return dq, dk, dv


# --------------------------------------------------------------------------- pointwise operators
def sp_rmsnorm_fwd(x, w, eps: float, y=None, rstd=None, stream=None):
    """x [T, C] bf16, w [C] bf16 -> (y [T, C] bf16, rstd [T] fp32)."""
    T, C = x.shape
    _expect(x, (T, C), torch.bfloat16, "x"); _expect(w, (C,), torch.bfloat16, "w")
    y = _new(stream, x.shape, x.dtype, x.device) if y is None else y
    rstd = _new(stream, (T,), torch.float32, x.device) if rstd is None else rstd
    _check(lib().sp_rmsnorm_fwd(_ptr(x), _ptr(w), _ptr(y), _ptr(rstd), T, C, float(eps), _stream(stream)), "sp_rmsnorm_fwd")
    return y, rstd


def sp_rmsnorm_bwd_workspace_bytes(T, C) -> int:
    return int(lib().sp_rmsnorm_bwd_workspace_bytes(T, C))


def sp_rmsnorm_bwd(x, w, rstd, dy, dx=None, dw=None, workspace=None, stream=None):
    """Returns (dx [T, C], dw [C]) bf16."""
    T, C = x.shape
    _expect(x, (T, C), torch.bfloat16, "x"); _expect(w, (C,), torch.bfloat16, "w")
    _expect(dy, (T, C), torch.bfloat16, "dy"); _expect(rstd, (T,), torch.float32, "rstd")
    dx = _new(stream, x.shape, x.dtype, x.device) if dx is None else dx
    dw = _new(stream, w.shape, w.dtype, w.device) if dw is None else dw
    if workspace is None:
        workspace = _workspace(sp_rmsnorm_bwd_workspace_bytes(T, C), x.device, stream)
    _check(lib().sp_rmsnorm_bwd(_ptr(x), _ptr(w), _ptr(rstd), _ptr(dy), _ptr(dx), _ptr(dw), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), T, C, _stream(stream)), "sp_rmsnorm_bwd")
    return dx, dw


def sp_rope(x, cos_table, sin_table, conjugate: bool = False, out=None, stream=None):
    """x [T, H, D] bf16, cos/sin tables [T, D/2] fp32 -> rotated tensor (out may be x)."""
    T, H, D = x.shape
    _expect(x, (T, H, D), torch.bfloat16, "x")
    _expect(cos_table, (T, D // 2), torch.float32, "cos_table"); _expect(sin_table, (T, D // 2), torch.float32, "sin_table")
    out = _new(stream, x.shape, x.dtype, x.device) if out is None else out
    _check(lib().sp_rope(_ptr(x), _ptr(cos_table), _ptr(sin_table), _ptr(out), T, H, D, int(bool(conjugate)),
                         _stream(stream)), "sp_rope")
    return out


def sp_swiglu_fwd(g, u, y=None, stream=None):
    _expect(g, g.shape, torch.bfloat16, "g"); _expect(u, g.shape, torch.bfloat16, "u")
    y = _new(stream, g.shape, g.dtype, g.device) if y is None else y
    _check(lib().sp_swiglu_fwd(_ptr(g), _ptr(u), _ptr(y), g.numel(), _stream(stream)), "sp_swiglu_fwd")
    return y


def sp_swiglu_bwd(g, u, dy, dg=None, du=None, stream=None):
    _expect(g, g.shape, torch.bfloat16, "g"); _expect(u, g.shape, torch.bfloat16, "u"); _expect(dy, g.shape, torch.bfloat16, "dy")
    dg = _new(stream, g.shape, g.dtype, g.device) if dg is None else dg
    du = _new(stream, u.shape, u.dtype, u.device) if du is None else du
    _check(lib().sp_swiglu_bwd(_ptr(g), _ptr(u), _ptr(dy), _ptr(dg), _ptr(du), g.numel(), _stream(stream)), "sp_swiglu_bwd")
    return dg, du


# --------------------------------------------------------------------------- 8-bit linear layers
# An 8-bit operand of R rows and K columns: q [R, Kp] float8, scale [Kp/128, Rp] float8_e8m0fnu, Kp = K rounded up to 128,
# Rp = R rounded up to 16; it stands for q[r, k] * scale[k // 128, r].
_E8M0 = torch.float8_e8m0fnu
_FP8_TYPES = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}
_OUT_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _operand_shapes(R: int, K: int):
    blocks = (K + 127) // 128
    return (R, blocks * 128), (blocks, (R + 15) // 16 * 16)


_BF16, _F32, _E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _refuse(*args):
    """Raises for the first of the tensors, given as (tensor or None, shape, dtype, name), that is not what is expected.  The wrappers
    below test all their tensors in one expression and come here when it fails: a call of _expect and _ptr for each takes longer
    than a single token's kernel."""
    for t, shape, dtype, name in args:
        if t is not None:
            _expect(t, shape, dtype, name)
    for t, _, _, _ in args:
        _ptr(t)
    raise AssertionError("nothing to refuse")


def sp_rmsnorm_fp8_fwd(x, w, eps: float, res=None, h=None, q=None, q_scale=None, rstd=None, stream=None):
    """x, res [T, C], w [C] bf16 -> (h = x + res [T, C] bf16, q, q_scale: the e4m3 operand of norm(h) [T, C], rstd [T] fp32).
    Without res, h is x itself.  h may be x or res (in place)."""
    rows = T, C = x.shape
    shape, scale_shape = _operand_shapes(T, C)
    if h is None and res is not None:
        h = _new(stream, rows, _BF16, x.device)
    if q is None:
        q = _new(stream, shape, _E4M3, x.device)
    if q_scale is None:
        q_scale = _new(stream, scale_shape, _E8M0, x.device)
    if rstd is None:
        rstd = _new(stream, (T,), _F32, x.device)
    if not (x.dtype is _BF16 and x.is_cuda and x.is_contiguous() and w.dtype is _BF16 and w.shape == (C,) and w.is_cuda and w.is_contiguous()
            and q.dtype is _E4M3 and q.shape == shape and q.is_cuda and q.is_contiguous()
            and q_scale.dtype is _E8M0 and q_scale.shape == scale_shape and q_scale.is_cuda and q_scale.is_contiguous()
            and rstd.dtype is _F32 and rstd.shape == (T,) and rstd.is_cuda and rstd.is_contiguous()
            and (res is None or (res.dtype is _BF16 and res.shape == rows and res.is_cuda and res.is_contiguous()
                                 and h.dtype is _BF16 and h.shape == rows and h.is_cuda and h.is_contiguous()))):
        _refuse((x, rows, _BF16, "x"), (res, rows, _BF16, "res"), (w, (C,), _BF16, "w"), (None if res is None else h, rows, _BF16, "h"),
                (q, shape, _E4M3, "q"), (q_scale, scale_shape, _E8M0, "q_scale"), (rstd, (T,), _F32, "rstd"))
    if res is None:
        h, r_ptr, h_ptr = x, None, None
    else:
        r_ptr, h_ptr = res.data_ptr(), h.data_ptr()
    code = (_lib or lib()).sp_rmsnorm_fp8_fwd(x.data_ptr(), r_ptr, w.data_ptr(), h_ptr, q.data_ptr(), q_scale.data_ptr(), rstd.data_ptr(),
                                              T, C, eps, _stream(stream))
    if code:
        _check(code, "sp_rmsnorm_fp8_fwd")
    return h, q, q_scale, rstd


def sp_rmsnorm_res_bwd(h, w, rstd, dy, dres, dh=None, dw=None, workspace=None, stream=None):
    """Gradients behind a residual norm: (dh [T, C], the gradient of x and of res alike, dw [C]) bf16.  dh may be dres or dy."""
    rows = T, C = h.shape
    if dh is None:
        dh = _new(stream, rows, _BF16, h.device)
    if dw is None:
        dw = _new(stream, (C,), _BF16, h.device)
    if workspace is None:
        workspace = _workspace(sp_rmsnorm_bwd_workspace_bytes(T, C), h.device, stream)
    if not (h.dtype is _BF16 and h.is_cuda and h.is_contiguous() and w.dtype is _BF16 and w.shape == (C,) and w.is_cuda and w.is_contiguous()
            and rstd.dtype is _F32 and rstd.shape == (T,) and rstd.is_cuda and rstd.is_contiguous()
            and dy.dtype is _BF16 and dy.shape == rows and dy.is_cuda and dy.is_contiguous()
            and dres.dtype is _BF16 and dres.shape == rows and dres.is_cuda and dres.is_contiguous()
            and dh.dtype is _BF16 and dh.shape == rows and dh.is_cuda and dh.is_contiguous()
            and dw.dtype is _BF16 and dw.shape == (C,) and dw.is_cuda and dw.is_contiguous() and workspace.is_cuda and workspace.is_contiguous()):
        _refuse((h, rows, _BF16, "h"), (w, (C,), _BF16, "w"), (rstd, (T,), _F32, "rstd"), (dy, rows, _BF16, "dy"), (dres, rows, _BF16, "dres"),
                (dh, rows, _BF16, "dh"), (dw, (C,), _BF16, "dw"), (workspace, workspace.shape, workspace.dtype, "workspace"))
    code = (_lib or lib()).sp_rmsnorm_res_bwd(h.data_ptr(), w.data_ptr(), rstd.data_ptr(), dy.data_ptr(), dres.data_ptr(), dh.data_ptr(),
                                              dw.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(), T, C,
                                              _stream(stream))
    if code:
        _check(code, "sp_rmsnorm_res_bwd")
    return dh, dw


def sp_fp8_quant(x, dtype=torch.float8_e4m3fn, rows: bool = True, cols: bool = False, rstd=None, w=None, q=None, q_scale=None,
                 qt=None, qt_scale=None, stream=None):
    """x [T, C] bf16 (times rstd [T] fp32 and w [C] bf16, if given) -> (q, q_scale, qt, qt_scale): the operand of x [T, C] if
    `rows`, that of its transpose [C, T] if `cols`; None for a side that is not asked for."""
    T, C = x.shape
    kind = _FP8_TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"dtype: expected float8_e4m3fn or float8_e5m2, got {dtype}")
    if not (rows or cols):
        raise ValueError("nothing asked for: rows and cols are both false")
    if (rstd is None) != (w is None):
        raise ValueError("rstd and w come together")
    fine = x.dtype is _BF16 and x.is_cuda and x.is_contiguous()
    r_ptr = w_ptr = q_ptr = qs_ptr = qt_ptr = qts_ptr = None
    shape = scale_shape = shape_t = scale_shape_t = None
    if rows:
        shape, scale_shape = _operand_shapes(T, C)
        if q is None:
            q = _new(stream, shape, dtype, x.device)
        if q_scale is None:
            q_scale = _new(stream, scale_shape, _E8M0, x.device)
        fine = (fine and q.dtype is dtype and q.shape == shape and q.is_cuda and q.is_contiguous()
                and q_scale.dtype is _E8M0 and q_scale.shape == scale_shape and q_scale.is_cuda and q_scale.is_contiguous())
        q_ptr, qs_ptr = q.data_ptr(), q_scale.data_ptr()
    else:
        q = q_scale = None
    if cols:
        shape_t, scale_shape_t = _operand_shapes(C, T)
        if qt is None:
            qt = _new(stream, shape_t, dtype, x.device)
        if qt_scale is None:
            qt_scale = _new(stream, scale_shape_t, _E8M0, x.device)
        fine = (fine and qt.dtype is dtype and qt.shape == shape_t and qt.is_cuda and qt.is_contiguous()
                and qt_scale.dtype is _E8M0 and qt_scale.shape == scale_shape_t and qt_scale.is_cuda and qt_scale.is_contiguous())
        qt_ptr, qts_ptr = qt.data_ptr(), qt_scale.data_ptr()
    else:
        qt = qt_scale = None
    if w is not None:
        fine = (fine and w.dtype is _BF16 and w.shape == (C,) and w.is_cuda and w.is_contiguous()
                and rstd.dtype is _F32 and rstd.shape == (T,) and rstd.is_cuda and rstd.is_contiguous())
        r_ptr, w_ptr = rstd.data_ptr(), w.data_ptr()
    if not fine:
        _refuse((x, (T, C), _BF16, "x"), (rstd, (T,), _F32, "rstd"), (w, (C,), _BF16, "w"), (q, shape, dtype, "q"), (q_scale, scale_shape, _E8M0, "q_scale"),
                (qt, shape_t, dtype, "qt"), (qt_scale, scale_shape_t, _E8M0, "qt_scale"))
    code = (_lib or lib()).sp_fp8_quant(x.data_ptr(), r_ptr, w_ptr, q_ptr, qs_ptr, qt_ptr, qts_ptr, T, C, kind, _stream(stream))
    if code:
        _check(code, "sp_fp8_quant")
    return q, q_scale, qt, qt_scale


@functools.lru_cache(maxsize=4096)
def sp_fp8_matmul_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().sp_fp8_matmul_workspace_bytes(M, N, K))


def sp_fp8_matmul(a, a_scale, b, b_scale, out_dtype=torch.bfloat16, out=None, accumulate: bool = False, workspace=None, stream=None):
    """Operands a [M, K] (e4m3 or e5m2) and b [N, K] (e4m3) -> out [M, N] = a b^T in bf16 or fp32 (out's type, if it is given);
    accumulate adds to what an fp32 `out` holds.  In bf16 the contraction is shared out (sp_fp8_matmul_split) where
    sp_fp8_matmul_workspace_bytes(M, N, K) is not 0; the workspace is allocated if it is not given.
    bf16 results are made by an instruction that sums eight products at a time with 13 binary places below the largest one: 1.5e-5 of
    a sum over normal values, but where large products cancel each of the other seven may be off by 2^-13 of the largest.  fp32
    results are sums in fp32 of exact products."""
    M, K = a.shape
    N = b.shape[0]
    kind = _FP8_TYPES.get(a.dtype)
    if kind is None:
        raise ValueError(f"a: expected float8_e4m3fn or float8_e5m2, got {a.dtype}")
    if K % 128 != 0:
        raise ValueError(f"a: {K} columns, not a multiple of 128")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensor to add to")
        if out_dtype not in _OUT_TYPES:
            raise ValueError(f"out: bfloat16 or float32 expected, got {out_dtype}")
        out = _new(stream, (M, N), out_dtype, a.device)
    out_kind = _OUT_TYPES.get(out.dtype)
    if out_kind is None or (accumulate and out.dtype is not _F32):
        raise ValueError(f"out: {'torch.float32' if accumulate else 'bfloat16 or float32'} expected, got {out.dtype}")
    a_shape, b_shape = (K // 128, (M + 15) // 16 * 16), (K // 128, (N + 15) // 16 * 16)
    if not (a.is_cuda and a.is_contiguous() and a_scale.dtype is _E8M0 and a_scale.shape == a_shape and a_scale.is_cuda and a_scale.is_contiguous()
            and b.dtype is _E4M3 and b.shape == (N, K) and b.is_cuda and b.is_contiguous()
            and b_scale.dtype is _E8M0 and b_scale.shape == b_shape and b_scale.is_cuda and b_scale.is_contiguous()
            and out.shape == (M, N) and out.is_cuda and out.is_contiguous()):
        _refuse((a, (M, K), a.dtype, "a"), (b, (N, K), _E4M3, "b"), (a_scale, a_shape, _E8M0, "a_scale"), (b_scale, b_shape, _E8M0, "b_scale"),
                (out, (M, N), out.dtype, "out"))
    need = sp_fp8_matmul_workspace_bytes(M, N, K) if out_kind == 0 else 0
    if need:
        if workspace is None:
            workspace = _workspace(need, a.device, stream)
        elif not (workspace.is_cuda and workspace.is_contiguous()):
            raise ValueError("workspace: a contiguous device tensor expected")
        code = (_lib or lib()).sp_fp8_matmul_split(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), out.data_ptr(),
                                                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), M, N, K, kind, _stream(stream))
        if code:
            _check(code, "sp_fp8_matmul_split")
        return out
    code = (_lib or lib()).sp_fp8_matmul(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), out.data_ptr(), M, N, K, kind, out_kind,
                                         1 if accumulate else 0, _stream(stream))
    if code:
        _check(code, "sp_fp8_matmul")
    return out


def default_scale(D: int) -> float:
    return 1.0 / math.sqrt(D)
