"""MI355X-native exact O(N)-memory attention (forward + backward) behind a C ABI.

`attn_fwd`, `attn_bwd`, `attn_bwd_workspace_bytes`, `attn_fwd_qkvpacked`, ... mirror the entry points
of `include/avion_attn.h` one to one.  This module only marshals arguments (device pointers, sizes,
the current HIP stream); every step of the computation runs in the HIP kernels of
`libavion_attn.so`.  There is no CPU or PyTorch fallback: if the library is missing, loading fails.
PyTorch is used for device memory and streams only.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libavion_attn.so")

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP, ESCRATCH = 0, -1, -2, -3, -4, -5
FLAG_F16, FLAG_CAUSAL, FLAG_QKVPACKED, FLAG_WIDE_F32, FLAG_TOKENS_I32 = 1, 2, 4, 8, 16

_lib = None


class AvionError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"avion_attn error {code}: {text}")
        self.code = code


def load_library() -> ctypes.CDLL:
    """Load the HIP library built in-tree. Raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
                "or python paper_2309_16669_amd/build.py); there is no fallback path")
        lib = ctypes.CDLL(LIB_PATH)
        p, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        lib.avion_version.restype = i
        lib.avion_version.argtypes = []
        lib.avion_strerror.restype = ctypes.c_char_p
        lib.avion_strerror.argtypes = [i]
        lib.avion_last_hip_error.restype = ctypes.c_char_p
        lib.avion_last_hip_error.argtypes = []
        lib.avion_attn_fwd.restype = i
        lib.avion_attn_fwd.argtypes = [p, p, p, p, p, i, i, i, i, f, p]
        lib.avion_attn_bwd_workspace_bytes.restype = sz
        lib.avion_attn_bwd_workspace_bytes.argtypes = [i, i, i, i]
        lib.avion_attn_bwd.restype = i
        lib.avion_attn_bwd.argtypes = [p, p, p, p, p, p, p, p, p, i, i, i, i, f, p, sz, p]
        lib.avion_attn_bwd_dq.restype = i
        lib.avion_attn_bwd_dq.argtypes = [p, p, p, p, p, p, p, i, i, i, i, f, p, sz, p]
        lib.avion_attn_bwd_dkdv.restype = i
        lib.avion_attn_bwd_dkdv.argtypes = [p, p, p, p, p, p, p, i, i, i, i, f, p, sz, p]
        lib.avion_attn_fwd_qkvpacked.restype = i
        lib.avion_attn_fwd_qkvpacked.argtypes = [p, p, p, i, i, i, i, f, p]
        lib.avion_attn_bwd_qkvpacked.restype = i
        lib.avion_attn_bwd_qkvpacked.argtypes = [p, p, p, p, p, i, i, i, i, f, p, sz, p]
        lib.avion_attn_fwd_f16.restype = i
        lib.avion_attn_fwd_f16.argtypes = lib.avion_attn_fwd.argtypes
        lib.avion_attn_bwd_f16.restype = i
        lib.avion_attn_bwd_f16.argtypes = lib.avion_attn_bwd.argtypes
        lib.avion_attn_fwd_causal.restype = i
        lib.avion_attn_fwd_causal.argtypes = lib.avion_attn_fwd.argtypes
        lib.avion_attn_bwd_causal.restype = i
        lib.avion_attn_bwd_causal.argtypes = lib.avion_attn_bwd.argtypes
        u = ctypes.c_uint
        lib.avion_attn_fwd_ex.restype = i
        lib.avion_attn_fwd_ex.argtypes = [p, p, p, p, p, i, i, i, i, f, u, p]
        lib.avion_attn_bwd_ex.restype = i
        lib.avion_attn_bwd_ex.argtypes = [p, p, p, p, p, p, p, p, p, i, i, i, i, f, u, p, sz, p]
        ll = ctypes.c_longlong
        lib.avion_layernorm_fwd.restype = i
        lib.avion_layernorm_fwd.argtypes = [p, p, p, p, p, p, ll, i, f, u, p]
        lib.avion_layernorm_bwd_workspace_bytes.restype = sz
        lib.avion_layernorm_bwd_workspace_bytes.argtypes = [ll, i]
        lib.avion_layernorm_bwd.restype = i
        lib.avion_layernorm_bwd.argtypes = [p, p, p, p, p, p, p, p, ll, i, u, p, sz, p]
        lib.avion_bias_gelu_fwd.restype = i
        lib.avion_bias_gelu_fwd.argtypes = [p, p, p, ll, i, u, p]
        lib.avion_bias_gelu_bwd_workspace_bytes.restype = sz
        lib.avion_bias_gelu_bwd_workspace_bytes.argtypes = [ll, i]
        lib.avion_bias_gelu_bwd.restype = i
        lib.avion_bias_gelu_bwd.argtypes = [p, p, p, p, p, ll, i, u, p, sz, p]
        lib.avion_bias_gelu_bwd_y.restype = i
        lib.avion_bias_gelu_bwd_y.argtypes = [p, p, p, p, p, p, ll, i, u, p, sz, p]
        lib.avion_column_sum_workspace_bytes.restype = sz
        lib.avion_column_sum_workspace_bytes.argtypes = [ll, i]
        lib.avion_column_sum.restype = i
        lib.avion_column_sum.argtypes = [p, p, ll, i, u, p, sz, p]
        lib.avion_attn_bwd_noalloc.restype = i
        lib.avion_attn_bwd_noalloc.argtypes = [p, p, p, p, p, p, p, p, p, i, i, i, i, f, p]
        lib.avion_embedding_fwd.restype = i
        lib.avion_embedding_fwd.argtypes = [p, p, p, ll, ll, i, f, u, p]
        lib.avion_embedding_bwd_workspace_bytes.restype = sz
        lib.avion_embedding_bwd_workspace_bytes.argtypes = [ll, ll, i]
        lib.avion_embedding_bwd.restype = i
        lib.avion_embedding_bwd.argtypes = [p, p, p, ll, ll, i, f, u, p, sz, p]
        lib.avion_rmsnorm_fwd.restype = i
        lib.avion_rmsnorm_fwd.argtypes = [p, p, p, p, p, p, ll, i, f, u, p]
        lib.avion_rmsnorm_bwd_workspace_bytes.restype = sz
        lib.avion_rmsnorm_bwd_workspace_bytes.argtypes = [ll, i]
        lib.avion_rmsnorm_bwd.restype = i
        lib.avion_rmsnorm_bwd.argtypes = [p, p, p, p, p, p, p, p, ll, i, u, p, sz, p]
        lib.avion_rmsnorm_fwd_fp8.restype = i
        lib.avion_rmsnorm_fwd_fp8.argtypes = [p, p, p, p, p, p, ll, i, f, u, p]
        lib.avion_quantize_rows.restype = i
        lib.avion_quantize_rows.argtypes = [p, p, p, ll, i, u, p]
        lib.avion_linear_fp8.restype = i
        lib.avion_linear_fp8.argtypes = [p, p, p, p, p, p, ll, i, i, u, p]
        _lib = lib
    return _lib


def version() -> int:
    return int(load_library().avion_version())


def strerror(code: int) -> str:
    return load_library().avion_strerror(int(code)).decode()


def _check(rc: int):
    if rc != OK:
        lib = load_library()
        text = strerror(rc)
        if rc == EHIP:
            text += ": " + lib.avion_last_hip_error().decode()
        raise AvionError(rc, text)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def _stream_handle(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _require(t, name, dtype, shape=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def attn_bwd_workspace_bytes(B: int, H: int, N: int, d: int) -> int:
    return int(load_library().avion_attn_bwd_workspace_bytes(B, H, N, d))


def _fwd(entry, dt, q, k, v, o, lse, scale, stream):
    import torch
    B, N, H, d = q.shape
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o")):
        _require(t, n, dt, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _check(entry(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, N, d, float(scale), _stream_handle(stream)))


def _bwd(entry, dt, q, k, v, o, lse, dO, dq, dk, dv, scale, workspace, stream):
    import torch
    B, N, H, d = q.shape
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dO, "dO"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        _require(t, n, dt, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _require(workspace, "workspace", torch.uint8)
    _check(entry(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, d,
                 float(scale), _ptr(workspace), workspace.numel(), _stream_handle(stream)))


def attn_fwd(q, k, v, o, lse, scale: float, stream=None) -> None:
    """avion_attn_fwd on torch tensors: q,k,v,o bf16 [B,N,H,d] on the GPU; lse fp32 [B,H,N]."""
    import torch
    _fwd(load_library().avion_attn_fwd, torch.bfloat16, q, k, v, o, lse, scale, stream)


def attn_fwd_f16(q, k, v, o, lse, scale: float, stream=None) -> None:
    """avion_attn_fwd_f16: the same on fp16 tensors."""
    import torch
    _fwd(load_library().avion_attn_fwd_f16, torch.float16, q, k, v, o, lse, scale, stream)


def attn_bwd(q, k, v, o, lse, dO, dq, dk, dv, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd on torch tensors; `workspace` is a uint8 GPU tensor of at least
    attn_bwd_workspace_bytes(B,H,N,d) bytes."""
    import torch
    _bwd(load_library().avion_attn_bwd, torch.bfloat16, q, k, v, o, lse, dO, dq, dk, dv, scale, workspace, stream)


def attn_bwd_noalloc(q, k, v, o, lse, dO, dq, dk, dv, scale: float, stream=None) -> None:
    """avion_attn_bwd_noalloc: avion_attn_bwd without a workspace argument (the library's built-in
    32 MiB scratch takes its place; larger problems raise AvionError with code ESCRATCH)."""
    import torch
    B, N, H, d = q.shape
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dO, "dO"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        _require(t, n, torch.bfloat16, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _check(load_library().avion_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq),
                                                 _ptr(dk), _ptr(dv), B, H, N, d, float(scale), _stream_handle(stream)))


def attn_bwd_f16(q, k, v, o, lse, dO, dq, dk, dv, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd_f16: the same on fp16 tensors."""
    import torch
    _bwd(load_library().avion_attn_bwd_f16, torch.float16, q, k, v, o, lse, dO, dq, dk, dv, scale, workspace, stream)


def attn_fwd_causal(q, k, v, o, lse, scale: float, stream=None) -> None:
    """avion_attn_fwd_causal: bf16 tensors, query i attends to keys 0..i."""
    import torch
    _fwd(load_library().avion_attn_fwd_causal, torch.bfloat16, q, k, v, o, lse, scale, stream)


def attn_bwd_causal(q, k, v, o, lse, dO, dq, dk, dv, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd_causal: gradients of the causal forward."""
    import torch
    _bwd(load_library().avion_attn_bwd_causal, torch.bfloat16, q, k, v, o, lse, dO, dq, dk, dv, scale, workspace,
         stream)


def attn_bwd_dq(q, k, v, o, lse, dO, dq, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd_dq: first phase of the backward (delta into the workspace, and dQ)."""
    import torch
    B, N, H, d = q.shape
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (dO, "dO"), (dq, "dq")):
        _require(t, n, torch.bfloat16, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_attn_bwd_dq(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq),
                                            B, H, N, d, float(scale), _ptr(workspace), workspace.numel(),
                                            _stream_handle(stream)))


def attn_bwd_dkdv(q, k, v, lse, dO, dk, dv, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd_dkdv: second phase of the backward (dK, dV; reads delta from the workspace)."""
    import torch
    B, N, H, d = q.shape
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (dO, "dO"), (dk, "dk"), (dv, "dv")):
        _require(t, n, torch.bfloat16, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_attn_bwd_dkdv(_ptr(q), _ptr(k), _ptr(v), _ptr(lse), _ptr(dO), _ptr(dk), _ptr(dv),
                                              B, H, N, d, float(scale), _ptr(workspace), workspace.numel(),
                                              _stream_handle(stream)))


def attn_fwd_qkvpacked(qkv, o, lse, scale: float, stream=None) -> None:
    """avion_attn_fwd_qkvpacked: qkv bf16 [B,N,3,H,d] (the joint projection's output), o bf16 [B,N,H,d],
    lse fp32 [B,H,N]."""
    import torch
    B, N, three, H, d = qkv.shape
    _require(qkv, "qkv", torch.bfloat16, (B, N, 3, H, d))
    _require(o, "o", torch.bfloat16, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _check(load_library().avion_attn_fwd_qkvpacked(_ptr(qkv), _ptr(o), _ptr(lse), B, H, N, d, float(scale),
                                                   _stream_handle(stream)))


def attn_bwd_qkvpacked(qkv, o, lse, dO, dqkv, scale: float, workspace, stream=None) -> None:
    """avion_attn_bwd_qkvpacked: gradients of the packed tensor, in the same packing."""
    import torch
    B, N, three, H, d = qkv.shape
    for t, n in ((qkv, "qkv"), (dqkv, "dqkv")):
        _require(t, n, torch.bfloat16, (B, N, 3, H, d))
    for t, n in ((o, "o"), (dO, "dO")):
        _require(t, n, torch.bfloat16, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_attn_bwd_qkvpacked(_ptr(qkv), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dqkv), B, H, N, d,
                                                   float(scale), _ptr(workspace), workspace.numel(),
                                                   _stream_handle(stream)))


def _flags(dtype, causal: bool, packed: bool) -> int:
    import torch
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"tensors must be bf16 or fp16, got {dtype}")
    return (FLAG_F16 if dtype == torch.float16 else 0) | (FLAG_CAUSAL if causal else 0) | (FLAG_QKVPACKED if packed else 0)


def attn_fwd_ex(q, k, v, o, lse, scale: float, causal: bool = False, stream=None) -> None:
    """avion_attn_fwd_ex: any combination of format (bf16 / fp16, taken from q.dtype), masking (`causal`)
    and packing (k is None and v is None: q is the packed [B,N,3,H,d] tensor)."""
    import torch
    packed = k is None and v is None
    dt = q.dtype
    if packed:
        B, N, three, H, d = q.shape
        _require(q, "qkv", dt, (B, N, 3, H, d))
    else:
        B, N, H, d = q.shape
        for t, n in ((q, "q"), (k, "k"), (v, "v")):
            _require(t, n, dt, (B, N, H, d))
    _require(o, "o", dt, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    none = ctypes.c_void_p(None)
    _check(load_library().avion_attn_fwd_ex(_ptr(q), none if packed else _ptr(k), none if packed else _ptr(v), _ptr(o),
                                            _ptr(lse), B, H, N, d, float(scale), _flags(dt, causal, packed),
                                            _stream_handle(stream)))


def attn_bwd_ex(q, k, v, o, lse, dO, dq, dk, dv, scale: float, workspace, causal: bool = False, stream=None) -> None:
    """avion_attn_bwd_ex: the gradients for avion_attn_fwd_ex with the same format, masking and packing
    (packed: k, v, dk, dv are None, q and dq are the packed tensors)."""
    import torch
    packed = k is None and v is None
    dt = q.dtype
    if packed:
        B, N, three, H, d = q.shape
        for t, n in ((q, "qkv"), (dq, "dqkv")):
            _require(t, n, dt, (B, N, 3, H, d))
        if dk is not None or dv is not None:
            raise ValueError("packed call: dk and dv must be None (dq receives the packed gradient)")
    else:
        B, N, H, d = q.shape
        for t, n in ((q, "q"), (k, "k"), (v, "v"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
            _require(t, n, dt, (B, N, H, d))
    for t, n in ((o, "o"), (dO, "dO")):
        _require(t, n, dt, (B, N, H, d))
    _require(lse, "lse", torch.float32, (B, H, N))
    _require(workspace, "workspace", torch.uint8)
    none = ctypes.c_void_p(None)
    opt = lambda t: none if t is None else _ptr(t)
    _check(load_library().avion_attn_bwd_ex(_ptr(q), opt(k), opt(v), _ptr(o), _ptr(lse), _ptr(dO), _ptr(dq), opt(dk),
                                            opt(dv), B, H, N, d, float(scale), _flags(dt, causal, packed),
                                            _ptr(workspace), workspace.numel(), _stream_handle(stream)))


def layernorm_bwd_workspace_bytes(M: int, D: int) -> int:
    return int(load_library().avion_layernorm_bwd_workspace_bytes(M, D))


def layernorm_fwd(x, gamma, beta, y, mean, rstd, eps: float, stream=None) -> None:
    """avion_layernorm_fwd: x, y bf16 or fp16 [M, D]; gamma, beta fp32 [D]; mean, rstd fp32 [M] (saved for the backward)."""
    import torch
    M, D = x.shape
    _require(x, "x", x.dtype, (M, D))
    _require(y, "y", x.dtype, (M, D))
    for t, n in ((gamma, "gamma"), (beta, "beta")):
        _require(t, n, torch.float32, (D,))
    for t, n in ((mean, "mean"), (rstd, "rstd")):
        _require(t, n, torch.float32, (M,))
    _check(load_library().avion_layernorm_fwd(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(y), _ptr(mean), _ptr(rstd), M, D,
                                              float(eps), _flags(x.dtype, False, False), _stream_handle(stream)))


def layernorm_bwd(x, gamma, mean, rstd, dy, dx, dgamma, dbeta, workspace, stream=None) -> None:
    """avion_layernorm_bwd: dx [M, D] in the format of x; dgamma, dbeta fp32 [D]."""
    import torch
    M, D = x.shape
    for t, n in ((x, "x"), (dy, "dy"), (dx, "dx")):
        _require(t, n, x.dtype, (M, D))
    for t, n in ((gamma, "gamma"), (dgamma, "dgamma"), (dbeta, "dbeta")):
        _require(t, n, torch.float32, (D,))
    for t, n in ((mean, "mean"), (rstd, "rstd")):
        _require(t, n, torch.float32, (M,))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_layernorm_bwd(_ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd), _ptr(dy), _ptr(dx), _ptr(dgamma),
                                              _ptr(dbeta), M, D, _flags(x.dtype, False, False), _ptr(workspace),
                                              workspace.numel(), _stream_handle(stream)))


def bias_gelu_bwd_workspace_bytes(M: int, F: int) -> int:
    return int(load_library().avion_bias_gelu_bwd_workspace_bytes(M, F))


def bias_gelu_fwd(x, bias, y, stream=None) -> None:
    """avion_bias_gelu_fwd: x, y bf16 or fp16 [M, F]; bias fp32 [F]."""
    import torch
    M, F = x.shape
    _require(x, "x", x.dtype, (M, F))
    _require(y, "y", x.dtype, (M, F))
    _require(bias, "bias", torch.float32, (F,))
    _check(load_library().avion_bias_gelu_fwd(_ptr(x), _ptr(bias), _ptr(y), M, F, _flags(x.dtype, False, False),
                                              _stream_handle(stream)))


def bias_gelu_bwd(x, bias, dy, dx, dbias, workspace, stream=None) -> None:
    """avion_bias_gelu_bwd: dx [M, F] in the format of x; dbias fp32 [F]."""
    import torch
    M, F = x.shape
    for t, n in ((x, "x"), (dy, "dy"), (dx, "dx")):
        _require(t, n, x.dtype, (M, F))
    for t, n in ((bias, "bias"), (dbias, "dbias")):
        _require(t, n, torch.float32, (F,))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_bias_gelu_bwd(_ptr(x), _ptr(bias), _ptr(dy), _ptr(dx), _ptr(dbias), M, F,
                                              _flags(x.dtype, False, False), _ptr(workspace), workspace.numel(),
                                              _stream_handle(stream)))


def bias_gelu_bwd_y(x, bias, dy, dx, y, dbias, workspace, stream=None) -> None:
    """avion_bias_gelu_bwd_y: bias_gelu_bwd that also writes y = GELU(x + bias); dx may be dy."""
    import torch
    M, F = x.shape
    for t, n in ((x, "x"), (dy, "dy"), (dx, "dx"), (y, "y")):
        _require(t, n, x.dtype, (M, F))
    for t, n in ((bias, "bias"), (dbias, "dbias")):
        _require(t, n, torch.float32, (F,))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_bias_gelu_bwd_y(_ptr(x), _ptr(bias), _ptr(dy), _ptr(dx), _ptr(y), _ptr(dbias), M, F,
                                                _flags(x.dtype, False, False), _ptr(workspace), workspace.numel(),
                                                _stream_handle(stream)))


def column_sum_workspace_bytes(M: int, F: int) -> int:
    return int(load_library().avion_column_sum_workspace_bytes(M, F))


def column_sum(x, out, workspace, stream=None) -> None:
    """avion_column_sum: out [F] = sum over the rows of x [M, F], both bf16 or fp16."""
    import torch
    M, F = x.shape
    _require(x, "x", x.dtype, (M, F))
    _require(out, "out", x.dtype, (F,))
    _require(workspace, "workspace", torch.uint8)
    _check(load_library().avion_column_sum(_ptr(x), _ptr(out), M, F, _flags(x.dtype, False, False), _ptr(workspace),
                                           workspace.numel(), _stream_handle(stream)))


def _opt(t):
    return ctypes.c_void_p(None) if t is None else _ptr(t)


def _one_device(*tensors):
    """The device of all of them (None: absent).  The calls below run with it as the current device, on its current stream
    unless another is given."""
    device = tensors[0].device
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors must live on one GPU, got {device} and {t.device}")
    return device


def _launch(device, entry, args, stream):
    import torch
    for a, kind in zip(args, entry.argtypes):
        if kind is ctypes.c_int and not -(1 << 31) <= a < 1 << 31:   # (ctypes would take it modulo 2^32)
            raise ValueError(f"{a} does not fit 32 bits")
    with torch.cuda.device(device):
        _check(entry(*args, _stream_handle(stream)))


def _tokens_flag(tokens) -> int:
    import torch
    if tokens.dtype not in (torch.int64, torch.int32):
        raise ValueError(f"tokens must be int64 or int32, got {tokens.dtype}")
    return FLAG_TOKENS_I32 if tokens.dtype == torch.int32 else 0


def _wide_flag(t, dtype, name) -> int:
    """FLAG_WIDE_F32 for an fp32 tensor, 0 for one of `dtype`."""
    import torch
    if t.dtype not in (torch.float32, dtype):
        raise ValueError(f"{name} must be {dtype} or torch.float32, got {t.dtype}")
    return FLAG_WIDE_F32 if t.dtype == torch.float32 else 0


def embedding_fwd(tokens, table, y, scale: float, stream=None) -> None:
    """avion_embedding_fwd: tokens int64 or int32 [n], table [V, D] in the format of y or fp32, y bf16 or fp16 [n, D]."""
    (n,), (V, D) = tokens.shape, table.shape
    flags = _tokens_flag(tokens) | _flags(y.dtype, False, False) | _wide_flag(table, y.dtype, "table")
    _require(tokens, "tokens", tokens.dtype, (n,))
    _require(table, "table", table.dtype, (V, D))
    _require(y, "y", y.dtype, (n, D))
    _launch(_one_device(table, tokens, y), load_library().avion_embedding_fwd,
            (_ptr(tokens), _ptr(table), _ptr(y), n, V, D, float(scale), flags), stream)


def embedding_bwd_workspace_bytes(n: int, V: int, D: int) -> int:
    return int(load_library().avion_embedding_bwd_workspace_bytes(n, V, D))


def embedding_bwd(tokens, dy, dtable, scale: float, workspace, stream=None) -> None:
    """avion_embedding_bwd: dy bf16 or fp16 [n, D]; dtable [V, D] in that format or fp32."""
    import torch
    (n,), (V, D) = tokens.shape, dtable.shape
    flags = _tokens_flag(tokens) | _flags(dy.dtype, False, False) | _wide_flag(dtable, dy.dtype, "dtable")
    _require(tokens, "tokens", tokens.dtype, (n,))
    _require(dy, "dy", dy.dtype, (n, D))
    _require(dtable, "dtable", dtable.dtype, (V, D))
    _require(workspace, "workspace", torch.uint8)
    _launch(_one_device(dtable, tokens, dy, workspace), load_library().avion_embedding_bwd,
            (_ptr(tokens), _ptr(dy), _ptr(dtable), n, V, D, float(scale), flags, _ptr(workspace), workspace.numel()), stream)


def _rms_inputs(x, residual, weight, h):
    import torch
    M, D = x.shape
    flags = _flags(x.dtype, False, False)
    _require(x, "x", x.dtype, (M, D))
    _require(weight, "weight", torch.float32, (D,))
    if (residual is None) != (h is None):
        raise ValueError("residual and h are given together or not at all")
    if residual is not None:
        flags |= _wide_flag(residual, x.dtype, "residual")
        _require(residual, "residual", residual.dtype, (M, D))
        _require(h, "h", residual.dtype, (M, D))
    return M, D, flags


def rmsnorm_fwd(x, residual, weight, y, h, rstd, eps: float, stream=None) -> None:
    """avion_rmsnorm_fwd: x, y bf16 or fp16 [M, D]; residual and h (both None: no addition) in that format or fp32; weight fp32
    [D]; rstd fp32 [M], or None where no backward follows."""
    import torch
    M, D, flags = _rms_inputs(x, residual, weight, h)
    _require(y, "y", x.dtype, (M, D))
    if rstd is not None:
        _require(rstd, "rstd", torch.float32, (M,))
    _launch(_one_device(x, residual, weight, y, h, rstd), load_library().avion_rmsnorm_fwd,
            (_ptr(x), _opt(residual), _ptr(weight), _ptr(y), _opt(h), _opt(rstd), M, D, float(eps), flags), stream)


def rmsnorm_fwd_fp8(x, residual, weight, y8, scale, h, eps: float, stream=None) -> None:
    """avion_rmsnorm_fwd_fp8: the same with y in 8 bits: y8 float8_e4m3fn [M, D], scale fp32 [M]."""
    import torch
    M, D, flags = _rms_inputs(x, residual, weight, h)
    _require(y8, "y8", torch.float8_e4m3fn, (M, D))
    _require(scale, "scale", torch.float32, (M,))
    _launch(_one_device(x, residual, weight, y8, scale, h), load_library().avion_rmsnorm_fwd_fp8,
            (_ptr(x), _opt(residual), _ptr(weight), _ptr(y8), _ptr(scale), _opt(h), M, D, float(eps), flags), stream)


def rmsnorm_bwd_workspace_bytes(M: int, D: int) -> int:
    return int(load_library().avion_rmsnorm_bwd_workspace_bytes(M, D))


def rmsnorm_bwd(h, weight, rstd, dy, dh, dx, dresidual, dweight, workspace, stream=None) -> None:
    """avion_rmsnorm_bwd: h [M, D] in the format of dy or fp32 (the residual stream's); dh like h or None; dx in the format of dy
    or None; dresidual fp32, only with an fp32 stream, or None; dweight fp32 [D]."""
    import torch
    M, D = dy.shape
    flags = _flags(dy.dtype, False, False) | _wide_flag(h, dy.dtype, "h")
    _require(h, "h", h.dtype, (M, D))
    _require(weight, "weight", torch.float32, (D,))
    _require(rstd, "rstd", torch.float32, (M,))
    _require(dy, "dy", dy.dtype, (M, D))
    for t, n, dt in ((dh, "dh", h.dtype), (dx, "dx", dy.dtype), (dresidual, "dresidual", torch.float32)):
        if t is not None:
            _require(t, n, dt, (M, D))
    _require(dweight, "dweight", torch.float32, (D,))
    _require(workspace, "workspace", torch.uint8)
    _launch(_one_device(h, weight, rstd, dy, dh, dx, dresidual, dweight, workspace), load_library().avion_rmsnorm_bwd,
            (_ptr(h), _ptr(weight), _ptr(rstd), _ptr(dy), _opt(dh), _opt(dx), _opt(dresidual), _ptr(dweight), M, D, flags,
             _ptr(workspace), workspace.numel()), stream)


def quantize_rows(x, x8, scale, stream=None) -> None:
    """avion_quantize_rows: x bf16 or fp16 [M, D] -> x8 float8_e4m3fn [M, D], scale fp32 [M]."""
    import torch
    M, D = x.shape
    _require(x, "x", x.dtype, (M, D))
    _require(x8, "x8", torch.float8_e4m3fn, (M, D))
    _require(scale, "scale", torch.float32, (M,))
    _launch(_one_device(x, x8, scale), load_library().avion_quantize_rows,
            (_ptr(x), _ptr(x8), _ptr(scale), M, D, _flags(x.dtype, False, False)), stream)


def linear_fp8(x8, x_scale, w8, w_scale, bias, y, stream=None) -> None:
    """avion_linear_fp8: x8 float8_e4m3fn [M, K] with fp32 x_scale [M], w8 [N, K] with w_scale [N], bias fp32 [N] or None, y
    bf16 or fp16 [M, N]."""
    import torch
    (M, K), N = x8.shape, w8.shape[0]
    _require(x8, "x8", torch.float8_e4m3fn, (M, K))
    _require(x_scale, "x_scale", torch.float32, (M,))
    _require(w8, "w8", torch.float8_e4m3fn, (N, K))
    _require(w_scale, "w_scale", torch.float32, (N,))
    if bias is not None:
        _require(bias, "bias", torch.float32, (N,))
    _require(y, "y", y.dtype, (M, N))
    _launch(_one_device(x8, x_scale, w8, w_scale, bias, y), load_library().avion_linear_fp8,
            (_ptr(x8), _ptr(x_scale), _ptr(w8), _ptr(w_scale), _opt(bias), _ptr(y), M, N, K, _flags(y.dtype, False, False)), stream)
