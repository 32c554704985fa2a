"""torch.autograd front end of the library, for use inside a training step.

`attention(q, k, v)` and `attention_qkvpacked(qkv)` allocate the outputs and the saved log-sum-exp with
torch and call the C-ABI entry points of `include/avion_attn.h` (the general forms, so every
combination of bf16 / fp16, causal or not, packed or not is available) through the binding in this
package.  Nothing is computed here: every step of the forward and of the backward runs in the HIP
kernels, and there is no fallback if the library is missing.

Plain calls go through the native functions of `csrc/avion_torch.cpp` (same checks, allocations, entry points
and saved tensors; the interpreter costs several times a small call's kernels).  They decline whatever is not
plain -- tensor subclasses, function transforms, modes, tracing, forward-mode tangents, arguments that do not
fit -- and those calls take the classes below, which treat or refuse them.

What is saved for the backward is O(N) per (batch, head): q, k, v, o and the fp32 log-sum-exp -- no
N x N matrix (the memory saving of Sec. 4.1 of the paper).

The classes keep the backward's workspace per (device, stream), grown on demand; backward calls on one
stream are ordered and may share it.  The native calls take theirs from torch's allocator for the length of
the call.

`layer_norm(x, gamma, beta)` and `bias_gelu(x, bias)` wrap the layer-normalisation and bias + GELU
entry points the same way (what they keep for the backward is stated in their docstrings), and so do
`embedding(tokens, weight)` and `add_rms_norm(x, residual, weight)` for the token table and for the RMS
normalisation with the residual's addition.  These two take the backward's workspace from torch's allocator for
the length of the call in either way of calling, and run on the device of their tensors.  These and the calls below take
tensors, and gradients, of any strides and at any address (what is not contiguous at a multiple of 16 bytes is copied first).
Their gradients are not differentiable: under create_graph they carry a node that raises.

`rms_norm_fp8`, `add_rms_norm_fp8`, `quantize_rows` and `linear_fp8` are the 8-bit path of a trained encoder: they
have no backward, and refuse inputs whose gradient is being recorded.
"""
from __future__ import annotations

import math
import types
import warnings

import torch

from . import (attn_bwd_ex, attn_bwd_workspace_bytes, attn_fwd_ex, bias_gelu_bwd, bias_gelu_bwd_workspace_bytes, bias_gelu_bwd_y,
               bias_gelu_fwd, column_sum, column_sum_workspace_bytes, layernorm_bwd, layernorm_bwd_workspace_bytes, layernorm_fwd, load_library)
from . import (embedding_bwd, embedding_bwd_workspace_bytes, embedding_fwd, rmsnorm_bwd, rmsnorm_bwd_workspace_bytes, rmsnorm_fwd,
               rmsnorm_fwd_fp8)
from . import linear_fp8 as _linear_fp8, quantize_rows as _quantize_rows

_native = None


def native_calls():
    """The module of native calls.  Where it is not built or does not load (another torch than it was built with) a
    stand-in that declines every call, with a warning: the classes below then serve them all."""
    global _native
    if _native is None:
        load_library()
        try:
            from . import _avion_torch
        except ImportError as e:
            warnings.warn(f"paper_2309_16669_amd/_avion_torch.so does not load ({e}); the Python classes take its calls, at "
                          "several times the host time.  Build it: python -c 'import __graft_entry__ as g; g.build()'")
            names = ("attention", "attention_qkvpacked", "layer_norm", "bias_gelu", "bias_gelu_linear", "embedding", "rms_norm",
                     "add_rms_norm", "rms_norm_fp8", "add_rms_norm_fp8", "quantize_rows", "linear_fp8")
            _avion_torch = types.SimpleNamespace(**{n: lambda *args: None for n in names})
        _native = _avion_torch
    return _native


_workspaces: dict = {}


def _workspace_of(need, device):
    key = (device, torch.cuda.current_stream(device).cuda_stream)
    ws = _workspaces.get(key)
    if ws is None or ws.numel() < need:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
        _workspaces[key] = ws
    return ws


def _workspace(B, H, N, d, device):
    return _workspace_of(attn_bwd_workspace_bytes(B, H, N, d), device)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        B, N, H, d = q.shape
        o = torch.empty_like(q)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
        attn_fwd_ex(q, k, v, o, lse, scale, causal)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.scale, ctx.causal = scale, causal
        return o

    @staticmethod
    def backward(ctx, dO):
        q, k, v, o, lse = ctx.saved_tensors
        B, N, H, d = q.shape
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        attn_bwd_ex(q, k, v, o, lse, dO.contiguous(), dq, dk, dv, ctx.scale, _workspace(B, H, N, d, q.device), ctx.causal)
        return dq, dk, dv, None, None


class _AttentionPacked(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, scale, causal):
        qkv = qkv.contiguous()
        B, N, _, H, d = qkv.shape
        o = torch.empty((B, N, H, d), dtype=qkv.dtype, device=qkv.device)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=qkv.device)
        attn_fwd_ex(qkv, None, None, o, lse, scale, causal)
        ctx.save_for_backward(qkv, o, lse)
        ctx.scale, ctx.causal = scale, causal
        return o

    @staticmethod
    def backward(ctx, dO):
        qkv, o, lse = ctx.saved_tensors
        B, N, _, H, d = qkv.shape
        dqkv = torch.empty_like(qkv)
        attn_bwd_ex(qkv, None, None, o, lse, dO.contiguous(), dqkv, None, None, ctx.scale,
                    _workspace(B, H, N, d, qkv.device), ctx.causal)
        return dqkv, None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, eps):
        shape = x.shape
        x2 = x.contiguous().view(-1, shape[-1])
        M = x2.shape[0]
        y = torch.empty_like(x2)
        mean = torch.empty((M,), dtype=torch.float32, device=x.device)
        rstd = torch.empty((M,), dtype=torch.float32, device=x.device)
        layernorm_fwd(x2, gamma.contiguous(), beta.contiguous(), y, mean, rstd, eps)
        ctx.save_for_backward(x2, gamma, mean, rstd)   # the input and two floats per token; not y
        ctx.shape = shape
        return y.view(shape)

    @staticmethod
    def backward(ctx, dy):
        x2, gamma, mean, rstd = ctx.saved_tensors
        M, D = x2.shape
        dx = torch.empty_like(x2)
        dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
        layernorm_bwd(x2, gamma.contiguous(), mean, rstd, dy.contiguous().view(M, D), dx, dgamma, dbeta,
                      _workspace_of(layernorm_bwd_workspace_bytes(M, D), x2.device))
        return dx.view(ctx.shape), dgamma, dbeta, None


class _BiasGelu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, bias):
        shape = x.shape
        x2 = x.contiguous().view(-1, shape[-1])
        y = torch.empty_like(x2)
        bias_gelu_fwd(x2, bias.contiguous(), y)
        ctx.save_for_backward(x2, bias)                # the pre-activation only; the derivative is rebuilt from it
        ctx.shape = shape
        return y.view(shape)

    @staticmethod
    def backward(ctx, dy):
        x2, bias = ctx.saved_tensors
        M, F = x2.shape
        dx, dbias = torch.empty_like(x2), torch.empty_like(bias)
        bias_gelu_bwd(x2, bias.contiguous(), dy.contiguous().view(M, F), dx, dbias,
                      _workspace_of(bias_gelu_bwd_workspace_bytes(M, F), x2.device))
        return dx.view(ctx.shape), dbias


def _column_sum(d):
    """d.sum(0); torch's where the rows are no multiple of 16 bytes, and where the sum is to be differentiated itself
    (create_graph, a tangent): it is linear in d."""
    need = column_sum_workspace_bytes(*d.shape)
    recorded = torch.is_grad_enabled() and d.requires_grad
    if need == 0 or d.data_ptr() % 16 != 0 or recorded or torch.autograd.forward_ad.unpack_dual(d).tangent is not None:
        return d.sum(0)
    out = torch.empty((d.shape[1],), dtype=d.dtype, device=d.device)
    column_sum(d, out, _workspace_of(need, d.device))
    return out


class _BiasGeluLinear(torch.autograd.Function):
    """linear(GELU(x + bias), weight, out_bias) that keeps x only: the activation's output is rebuilt by the
    backward pass (avion_bias_gelu_bwd_y) for the weight gradient.  The two matrix products per
    direction are torch's (library GEMMs)."""

    @staticmethod
    def forward(ctx, x, bias, weight, out_bias):
        shape = x.shape
        x2 = x.contiguous().view(-1, shape[-1])
        y = torch.empty_like(x2)
        bias_gelu_fwd(x2, bias.contiguous(), y)
        out = torch.addmm(out_bias, y, weight.t()) if out_bias is not None else y @ weight.t()
        ctx.save_for_backward(x2, bias, weight)
        ctx.shape, ctx.has_out_bias = shape, out_bias is not None
        return out.view(*shape[:-1], weight.shape[0])

    @staticmethod
    def backward(ctx, dout):
        x2, bias, weight = ctx.saved_tensors
        M, F = x2.shape
        d2 = dout.contiguous().view(M, weight.shape[0])
        # with respect to the activation's output; then, in its place, to x: .data, as neither the product's node
        # (create_graph) nor its tangent is that of the gradient of x
        dx = (d2 @ weight).data
        y, dbias = torch.empty_like(x2), torch.empty_like(bias)
        bias_gelu_bwd_y(x2, bias.contiguous(), dx, dx, y, dbias, _workspace_of(bias_gelu_bwd_workspace_bytes(M, F), x2.device))
        return dx.view(ctx.shape), dbias, d2.t() @ y, (_column_sum(d2) if ctx.has_out_bias else None)


def bias_gelu_linear(x, bias, weight, out_bias=None):
    """linear(GELU(x + bias), weight, out_bias): the second half of the encoder's MLP, keeping only x (the
    first matrix product's output) for the backward; x bf16 or fp16 [..., F], bias fp32 [F], weight
    [out, F] and out_bias [out] in the format of x."""
    out = (_native or native_calls()).bias_gelu_linear(x, bias, weight, out_bias)
    return _BiasGeluLinear.apply(x, bias, weight, out_bias) if out is None else out


def layer_norm(x, gamma, beta, eps: float = 1e-5):
    """Layer normalisation over the last axis of x (bf16 or fp16, any leading shape, width <= 2048 and a
    multiple of 8) with fp32 gain and bias.  Differentiable in x, gamma and beta; keeps x and two floats
    per token for the backward."""
    y = (_native or native_calls()).layer_norm(x, gamma, beta, float(eps))
    return _LayerNorm.apply(x, gamma, beta, float(eps)) if y is None else y


def bias_gelu(x, bias):
    """GELU(x + bias) (exact erf form) over the last axis of x (bf16 or fp16, width a multiple of 8) with
    an fp32 bias.  Differentiable in x and bias; keeps only x for the backward."""
    y = (_native or native_calls()).bias_gelu(x, bias)
    return _BiasGelu.apply(x, bias) if y is None else y


def attention(q, k, v, scale: float | None = None, causal: bool = False):
    """softmax(scale * q k^T) v per (batch, head) for q, k, v of shape [B, N, H, d], bf16 or fp16,
    d in {64, 80}; `causal`: query i attends to keys 0..i.  Differentiable.  scale defaults to 1/sqrt(d)."""
    scale, causal = 1.0 / math.sqrt(q.shape[-1]) if scale is None else float(scale), bool(causal)
    o = (_native or native_calls()).attention(q, k, v, scale, causal)
    return _Attention.apply(q, k, v, scale, causal) if o is None else o


def attention_qkvpacked(qkv, scale: float | None = None, causal: bool = False):
    """The same for the [B, N, 3, H, d] output of a joint QKV projection (bf16 or fp16); the gradient
    comes back in the same packing."""
    scale, causal = 1.0 / math.sqrt(qkv.shape[-1]) if scale is None else float(scale), bool(causal)
    o = (_native or native_calls()).attention_qkvpacked(qkv, scale, causal)
    return _AttentionPacked.apply(qkv, scale, causal) if o is None else o


# ------------------------------------------------------------------- token table, RMS normalisation, 8-bit path
def _bytes_on(device, need):
    if need == 0:
        raise ValueError("unsupported shape")
    return torch.empty(need, dtype=torch.uint8, device=device)


def _dense(t):
    """Contiguous and at a multiple of 16 bytes, as the C entries ask: a piece of a larger tensor (a gradient that comes out of a
    concatenation) may begin at any element, and its place is not the caller's to choose."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _NoSecondDerivative(torch.autograd.Function):
    """The node of a gradient that a kernel has written: it leads to the tensors that the gradient depends on, and says that the
    way back through it does not exist.  Without it a second derivative would silently miss this operator's part."""

    @staticmethod
    def forward(ctx, what, gradient, *inputs):
        ctx.what = what
        return gradient[0]

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError(f"{ctx.what} has no second derivative")


def _depends_on(gradient, what, *inputs):
    """`gradient` with that node, where the backward itself is recorded (create_graph)."""
    inputs = [t for t in inputs if t is not None and t.requires_grad]
    if gradient is None or not inputs or not torch.is_grad_enabled():
        return gradient
    return _NoSecondDerivative.apply(what, (gradient,), *inputs)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, dtype):
        t = tokens.contiguous().view(-1)
        V, D = weight.shape
        y = torch.empty((t.shape[0], D), dtype=dtype, device=weight.device)
        embedding_fwd(t, _dense(weight), y, scale)
        ctx.save_for_backward(t)
        ctx.scale, ctx.shape, ctx.dtype = scale, (V, D), weight.dtype
        return y.view(*tokens.shape, D)

    @staticmethod
    def backward(ctx, dy):
        (t,) = ctx.saved_tensors
        V, D = ctx.shape
        dweight = torch.empty((V, D), dtype=ctx.dtype, device=dy.device)
        embedding_bwd(t, _dense(dy).view(-1, D), dweight, ctx.scale,
                      _bytes_on(dy.device, embedding_bwd_workspace_bytes(t.shape[0], V, D)))
        return None, _depends_on(dweight, "embedding", dy), None, None


class _AddRmsNorm(torch.autograd.Function):
    """residual None: the norm of x itself, y alone."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        shape = x.shape
        D = shape[-1]
        x = _dense(x)
        x2 = x.view(-1, D)
        r2 = None if residual is None else _dense(residual).view(-1, D)
        y, h = torch.empty_like(x2), None if residual is None else torch.empty_like(r2)
        rstd = torch.empty((x2.shape[0],), dtype=torch.float32, device=x.device)
        rmsnorm_fwd(x2, r2, _dense(weight), y, h, rstd, eps)
        ctx.set_materialize_grads(False)
        h = x if h is None else h.view(shape)
        ctx.save_for_backward(h, weight, rstd)         # the residual stream, kept anyway, and one float per token; not y
        ctx.dtype, ctx.alone, ctx.vary = x.dtype, residual is None, any(ctx.needs_input_grad[:2])
        return y.view(shape) if residual is None else (y.view(shape), h)

    @staticmethod
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        if dy is None and dh is None:
            return None, None, None, None
        D = h.shape[-1]
        given = dy, dh
        h2 = _dense(h).view(-1, D)
        dy = torch.zeros(h2.shape, dtype=ctx.dtype, device=h.device) if dy is None else _dense(dy).view(-1, D)
        dh = None if dh is None else _dense(dh).view(-1, D)
        wide = h.dtype != ctx.dtype
        dx = torch.empty_like(dy) if ctx.needs_input_grad[0] or not wide else None
        dr = torch.empty_like(h2) if wide and ctx.needs_input_grad[1] else None
        dweight = torch.empty_like(weight, memory_format=torch.contiguous_format)
        rmsnorm_bwd(h2, _dense(weight), rstd, dy, dh, dx, dr, dweight,
                    _bytes_on(h.device, rmsnorm_bwd_workspace_bytes(*h2.shape)))
        what = "rms_norm" if ctx.alone else "add_rms_norm"
        dx = None if dx is None else _depends_on(dx.view(h.shape), what, *given, h, weight)
        dr = dx if not wide else None if dr is None else _depends_on(dr.view(h.shape), what, *given, h, weight)
        dweight = _depends_on(dweight, what, given[0], h if ctx.vary else None)
        return dx, (None if ctx.alone else dr), dweight, None


def _check_residual(x, residual):
    if residual.shape != x.shape:
        raise ValueError(f"residual must have the shape of x, {tuple(x.shape)}, got {tuple(residual.shape)}")


def _no_backward(name, *tensors):
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError(f"{name} has no backward: call it under torch.no_grad(), or detach its inputs")


def embedding(tokens, weight, scale: float = 1.0, dtype=None):
    """scale * weight[tokens] for tokens (int64 or int32, any shape) of a table [V, D] in bf16, fp16 or fp32, D a multiple of 8;
    the result is bf16 or fp16 (`dtype`; the table's own format, bf16 for an fp32 table, if None).  A token outside [0, V)
    gives a row of zeros and adds to no gradient.  Differentiable once in weight (the gradient has the table's format; fp32 sums in
    a fixed order); keeps the tokens for the backward."""
    if dtype is None:
        dtype = torch.bfloat16 if weight.dtype == torch.float32 else weight.dtype
    y = (_native or native_calls()).embedding(tokens, weight, float(scale), dtype == torch.float16, dtype == torch.bfloat16)
    return _Embedding.apply(tokens, weight, float(scale), dtype) if y is None else y


def rms_norm(x, weight, eps: float = 1e-6):
    """Root-mean-square normalisation over the last axis of x (bf16 or fp16, any leading shape, width <= 16384 and a multiple of
    8) with fp32 gains.  Differentiable once in x and weight; keeps x and one float per token for the backward."""
    y = (_native or native_calls()).rms_norm(x, weight, float(eps))
    return _AddRmsNorm.apply(_dense(x), None, weight, float(eps)) if y is None else y


def add_rms_norm(x, residual, weight, eps: float = 1e-6):
    """(y, h): h = x + residual, the residual stream behind a layer's branch, and y = rms_norm(h, weight), what the next branch
    reads.  x bf16 or fp16 [..., D]; residual, of the same shape, in the format of x or fp32, and h like it (y is the norm of h
    as stored).  Differentiable once in x, residual and weight; keeps h and one float per token."""
    _check_residual(x, residual)
    out = (_native or native_calls()).add_rms_norm(x, residual, weight, float(eps))
    return _AddRmsNorm.apply(x, residual, weight, float(eps)) if out is None else out


def _rms_norm_fp8(x, residual, weight, eps):
    shape = x.shape
    x2 = _dense(x).view(-1, shape[-1])
    r2 = None if residual is None else _dense(residual).view(-1, shape[-1])
    y8 = torch.empty(x2.shape, dtype=torch.float8_e4m3fn, device=x.device)
    scale = torch.empty((x2.shape[0],), dtype=torch.float32, device=x.device)
    h = None if r2 is None else torch.empty_like(r2)
    rmsnorm_fwd_fp8(x2, r2, _dense(weight), y8, scale, h, eps)
    return y8.view(shape), scale.view(shape[:-1]), None if h is None else h.view(shape)


def rms_norm_fp8(x, weight, eps: float = 1e-6):
    """(y8, scale): rms_norm(x, weight) in 8 bits, y ~ y8 * scale[..., None] with y8 float8_e4m3fn [..., D] and one fp32 scale a
    row, max|y| / 448.  D a multiple of 16.  No backward."""
    _no_backward("rms_norm_fp8", x, weight)
    out = (_native or native_calls()).rms_norm_fp8(x, weight, float(eps))
    return _rms_norm_fp8(x, None, weight, float(eps))[:2] if out is None else out


def add_rms_norm_fp8(x, residual, weight, eps: float = 1e-6):
    """(y8, scale, h): add_rms_norm with y in 8 bits, as rms_norm_fp8 gives it.  No backward."""
    _check_residual(x, residual)
    _no_backward("add_rms_norm_fp8", x, residual, weight)
    out = (_native or native_calls()).add_rms_norm_fp8(x, residual, weight, float(eps))
    return _rms_norm_fp8(x, residual, weight, float(eps)) if out is None else out


def quantize_rows(x):
    """(x8, scale) with x ~ x8 * scale[..., None]: the rows (last axis, a multiple of 16) of a bf16 or fp16 tensor in 8 bits
    (float8_e4m3fn) with one fp32 scale a row, max|x| / 448.  For a weight [N, K] that linear_fp8 reads, and for activations
    that no norm produces.  No backward."""
    _no_backward("quantize_rows", x)
    out = (_native or native_calls()).quantize_rows(x)
    if out is not None:
        return out
    x2 = _dense(x).view(-1, x.shape[-1])
    x8 = torch.empty(x2.shape, dtype=torch.float8_e4m3fn, device=x.device)
    scale = torch.empty((x2.shape[0],), dtype=torch.float32, device=x.device)
    _quantize_rows(x2, x8, scale)
    return x8.view(x.shape), scale.view(x.shape[:-1])


def linear_fp8(x8, x_scale, w8, w_scale, bias=None, dtype=torch.bfloat16):
    """linear(x, w, bias) of rows in 8 bits: x ~ x8 * x_scale[..., None] with x8 [..., K], w ~ w8 * w_scale[:, None] with w8
    [N, K] (both float8_e4m3fn, scales fp32, as rms_norm_fp8 and quantize_rows give them), bias fp32 [N] or None.  The
    result [..., N] is bf16 or fp16 (`dtype`), summed in fp32 and rounded once.  K a multiple of 16, N of 8.  No backward."""
    _no_backward("linear_fp8", x8, x_scale, w8, w_scale, bias)
    y = (_native or native_calls()).linear_fp8(x8, x_scale, w8, w_scale, bias, dtype == torch.float16, dtype == torch.bfloat16)
    if y is not None:
        return y
    K = x8.shape[-1]
    if w8.dim() != 2 or w8.shape[1] != K:
        raise ValueError(f"w8 must have shape (N, {K}), got {tuple(w8.shape)}")
    if x_scale.shape != x8.shape[:-1]:
        raise ValueError(f"x_scale must have shape {tuple(x8.shape[:-1])}, got {tuple(x_scale.shape)}")
    x2 = _dense(x8).view(-1, K)
    y = torch.empty((x2.shape[0], w8.shape[0]), dtype=dtype, device=x8.device)
    _linear_fp8(x2, x_scale.contiguous().view(-1), _dense(w8), _dense(w_scale), None if bias is None else _dense(bias), y)
    return y.view(*x8.shape[:-1], w8.shape[0])
