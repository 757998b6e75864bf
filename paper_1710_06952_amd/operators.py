"""Operators of a worker's own training step on torch tensors: dense layers, gated projections and layer norm,
log-probabilities and losses over a vocabulary, AdamW over many tensors.  The same entry points as include/adpsgd.h; every computation runs in the HIP
library, on the current stream of the tensors' device.

    y = dense(x, w, bias, residual=r, activation="gelu")           # differentiable
    h = gated(layer_norm(x, scale, shift), w2, activation="silu")  # differentiable
    lp = token_log_probs(logits, tokens)                           # of a frozen model, or to sample with
    r = policy_loss_and_gradient(logits, tokens, old, advantages, ref, clip=(0.2, 0.2), kl_coef=0.05)
    r = preference_loss_and_gradient(logits, tokens, offsets, ref, beta=0.1)
    r = distillation_loss_and_gradient(logits, tokens, teacher_tokens, teacher_logits, temperature=2.0)
    logits.backward(r.dlogits)                                     # or torch.autograd.grad
    opt = AdamW(params, grads, lr=1e-3, state_bits=8);  opt.step(max_norm=1.0)

A gradient function of model "external" evaluates loss and gradient with these and hands the engine an AdamW direction
(``out``) where the engine expects a gradient: the event averages and steps along it.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple

import numpy as np
import torch
from torch.autograd import forward_ad

from . import binding as B

_TYPES = {torch.float32: B.TYPE_F32, torch.bfloat16: B.TYPE_BF16, torch.float16: B.TYPE_F16}
_ACTIVATIONS = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}

PolicyLoss = namedtuple("PolicyLoss", "loss dlogits log_probs")
DistillationLoss = namedtuple("DistillationLoss", "loss dlogits divergences log_probs")
PreferenceLoss = namedtuple("PreferenceLoss", "loss dlogits log_probs margins")


def _call(device, fn, *args):
    """One library call on the device's current stream.  The stream is asked for as the number it is: a Stream object takes
    2.5 us to make, a sixth of what the smallest calls take in all."""
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc != B.OK:
        raise B.AdpsgdError(rc, (B.lib().adpsgd_last_error(None) or b"").decode())


def _refuse_capture(name):
    """Of a differentiable form and of its backward pass: what autograd does around them depends on graphs of the same leaves that live outside."""
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("%s with gradients cannot be captured: capture %s_forward and %s_gradients" % (name, name, name))


def _on_gpu(name, t, device=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:      # read through its address, it would lose the tangent
        raise NotImplementedError("%s has a tangent: the operators have no derivatives in forward mode" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU: the HIP library is the only implementation" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, the other tensors on %s" % (name, t.device, device))


def _vector(name, t, n, dtype, device):
    _on_gpu(name, t, device)
    if t.dtype != dtype or t.shape != (n,):
        raise ValueError("%s must be a vector of %d %s, is %s %s" % (name, n, dtype, tuple(t.shape), t.dtype))
    return t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- dense layers -----------------------------------------------------------------------------------------------

_REACH = 1 << 22        # elements from one row of a dense operand to the next, at most


def _as_rows(t, reach=_REACH):
    """t as a matrix whose last dimension is contiguous, and its leading dimension.  The stride of a dimension of size 1 says nothing."""
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    n, (step, inner) = t.shape[1], t.stride()
    if t.shape[0] <= 1:
        step = n
    if (inner != 1 and n > 1) or not n <= step <= reach:
        t, step = t.contiguous(), n
    return t, step


def _as_weights(w):
    """w (out x in) as it is stored: the tensor, its leading dimension, and whether it lies in x out."""
    (N, K), (out, inner) = w.shape, w.stride()
    if (inner == 1 or K == 1) and (N == 1 or K <= out <= _REACH):
        return w, K if N == 1 else out, 0
    if (out == 1 or N == 1) and (K == 1 or N <= inner <= _REACH):
        return w, N if K == 1 else inner, 1
    return w.contiguous(), K, 0


def _check_dense(x, w, b, r, activation):
    _on_gpu("x", x)
    for name, t in (("w", w), ("bias", b), ("residual", r)):
        if t is None and name != "w":
            continue
        _on_gpu(name, t, x.device)
        if t.dtype != x.dtype:
            raise TypeError("x is %s, %s is %s" % (x.dtype, name, t.dtype))
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("dense takes bfloat16 or float16, not %s" % x.dtype)
    if activation not in _ACTIVATIONS:
        raise ValueError("activation must be one of %s" % ", ".join(_ACTIVATIONS))
    if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1] or w.shape[0] < 1 or w.shape[1] < 1:
        raise ValueError("x is %s, w %s: w must be out x in" % (tuple(x.shape), tuple(w.shape)))
    if b is not None and b.shape != (w.shape[0],):
        raise ValueError("bias is %s, w %s" % (tuple(b.shape), tuple(w.shape)))
    if r is not None and r.shape != (*x.shape[:-1], w.shape[0]):
        raise ValueError("residual is %s, must have the shape of the result" % (tuple(r.shape),))


def _dense_args(x, ldx, w, ldw, transposed, activation, backward):
    M, K, N = x.shape[0], x.shape[1], w.shape[0]
    size = B.lib().adpsgd_dense_workspace_bytes(M, N, K, backward)
    if size < 0:
        raise B.AdpsgdError(B.ERR_ARG, "dense: M = %d, N = %d, K = %d is too large" % (M, N, K))
    space = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    args = B.Dense(_TYPES[x.dtype], _ACTIVATIONS[activation], M, N, K, x.data_ptr(), ldx, w.data_ptr(), ldw, transposed, 0, None, None, 0,
                   _ptr(space), size)
    return args, space


def _forward(x, w, b, r, activation, want_slope):
    xm, ldx = _as_rows(x)
    ws, ldw, transposed = _as_weights(w)
    M, N = xm.shape[0], w.shape[0]
    args, space = _dense_args(xm, ldx, ws, ldw, transposed, activation, 0)
    y = torch.empty(*x.shape[:-1], N, dtype=x.dtype, device=x.device)
    slope = torch.empty(M, N, dtype=torch.int16, device=x.device) if want_slope and activation != "none" else None
    if b is not None:
        b = b.contiguous()
        args.b = b.data_ptr()
    if r is not None:
        r, args.ldr = _as_rows(r)
        args.r = r.data_ptr()
    if M:
        _call(x.device, B.lib().adpsgd_dense_forward, C.byref(args), y.data_ptr(), _ptr(slope))
    del space
    return y, slope


def _backward(dy, x, w, slope, activation, need_dx, need_dw, need_db):
    xm, ldx = _as_rows(x)
    ws, ldw, transposed = _as_weights(w)
    dym, lddy = _as_rows(dy)
    M, K, N = xm.shape[0], xm.shape[1], w.shape[0]
    args, space = _dense_args(xm, ldx, ws, ldw, transposed, activation, 1)
    new = lambda *shape: torch.empty(*shape, dtype=x.dtype, device=x.device)  # noqa: E731
    dx = new(*x.shape) if need_dx else None
    dw = (new(K, N).t() if transposed else new(N, K)) if need_dw else None
    db = new(N) if need_db else None
    _call(x.device, B.lib().adpsgd_dense_backward, C.byref(args), dym.data_ptr(), lddy, _ptr(slope), _ptr(dx), _ptr(dw), _ptr(db))
    del space
    return dx, dw, db


class _Dense(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, r, activation):
        y, slope = _forward(x, w, b, r, activation, True)
        ctx.save_for_backward(x, w, slope)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, w, slope = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = db = None
        if need[0] or need[1] or need[2]:
            dx, dw, db = _backward(dy, x, w, slope, ctx.activation, *need[:3])
        return dx, dw, db, dy if need[3] else None, None


def dense(x, w, bias=None, *, residual=None, activation="none"):
    """act(x w^T + bias) + residual in one pass, differentiable (once, in reverse mode) in all four.

    x (..., in), w (out, in) as it is or as the transpose of an (in, out) tensor, bias (out), residual (..., out), all
    bfloat16 or all float16; activation "none", "relu", "gelu" (z Phi(z)) or "silu".  Products are added in 32 bits and
    the result is rounded once.  With gradients, 2 bytes an output are kept for the backward pass (the slope).

    Under capture of a HIP graph the differentiable form is refused: what autograd does around it depends on graphs of
    the same leaves that live outside.  dense_forward and dense_gradients can be captured."""
    _check_dense(x, w, bias, residual, activation)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, w, bias, residual)):
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("dense with gradients cannot be captured: capture dense_forward and dense_gradients")
        return _Dense.apply(x, w, bias, residual, activation)
    return _forward(x, w, bias, residual, activation, False)[0]


def dense_forward(x, w, bias=None, *, residual=None, activation="none"):
    """(y, slope): the forward pass without autograd, and what dense_gradients needs (None without an activation)."""
    _check_dense(x, w, bias, residual, activation)
    with torch.no_grad():
        return _forward(x, w, bias, residual, activation, True)


def dense_gradients(dy, x, w, slope, *, activation="none", need=(True, True, True)):
    """(dx, dw, dbias) for dy; None where ``need`` says so.  The residual's gradient is dy."""
    _check_dense(x, w, None, dy, activation)
    if activation != "none":
        _on_gpu("slope", slope, x.device)
        if slope.dtype != torch.int16 or slope.numel() != dy.numel() or not slope.is_contiguous():
            raise ValueError("slope must be what dense_forward returned")
    if not any(need):
        return None, None, None
    with torch.no_grad():
        return _backward(dy, x, w, slope if activation != "none" else None, activation, *need)


# ---- gated projections ------------------------------------------------------------------------------------------

_SLOPE_BYTES = {torch.bfloat16: 2, torch.float16: 3}      # of adpsgd_gated_slopes_bytes


def _check_gated(x, w, b, activation):
    _on_gpu("x", x)
    T, device = x.dtype, x.device
    for name, t in (("w", w), ("bias", b)):
        if t is None and name != "w":
            continue
        _on_gpu(name, t, device)
        if t.dtype != T:
            raise TypeError("x is %s, %s is %s" % (T, name, t.dtype))
    if T not in _SLOPE_BYTES:
        raise TypeError("gated takes bfloat16 or float16, not %s" % T)
    if activation not in _ACTIVATIONS:
        raise ValueError("activation must be one of %s" % ", ".join(_ACTIVATIONS))
    rows, inner = w.shape if w.dim() == 2 else (0, 0)
    if x.dim() < 1 or x.shape[-1] != inner or rows < 2 or rows % 2 or inner < 1:
        raise ValueError("x is %s, w %s: w must be 2 out x in, the gates' rows and then their partners'" % (tuple(x.shape), tuple(w.shape)))
    if b is not None and (b.dim() != 1 or b.numel() != rows):
        raise ValueError("bias is %s, w %s" % (tuple(b.shape), tuple(w.shape)))


def _gated_args(x, w, activation, backward):
    xm, ldx = _as_rows(x)
    ws, ldw, transposed = _as_weights(w)
    M, K, N = xm.shape[0], xm.shape[1], w.shape[0] // 2
    size = B.lib().adpsgd_gated_workspace_bytes(M, N, K, backward)
    if size < 0:
        raise B.AdpsgdError(B.ERR_ARG, "gated: M = %d, N = %d, K = %d is too large" % (M, N, K))
    space = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    args = B.Dense(_TYPES[x.dtype], _ACTIVATIONS[activation], M, N, K, xm.data_ptr(), ldx, ws.data_ptr(), ldw, transposed, 0, None, None, 0, _ptr(space),
                   size)
    return args, (xm, ws, space)


def _gated_forward(x, w, b, activation, want_slopes):
    args, keep = _gated_args(x, w, activation, 0)
    h = torch.empty(*x.shape[:-1], args.N, dtype=x.dtype, device=x.device)
    slopes = torch.empty(_SLOPE_BYTES[x.dtype] * 2 * args.N * args.M, dtype=torch.uint8, device=x.device) if want_slopes else None
    if b is not None:
        b = b.contiguous()
        args.b = b.data_ptr()
    if args.M:
        _call(x.device, B.lib().adpsgd_gated_forward, C.byref(args), h.data_ptr(), _ptr(slopes))
    del keep
    return h, slopes


def _gated_backward(dh, x, w, slopes, need_dx, need_dw, need_db):
    args, keep = _gated_args(x, w, "none", 1)
    dhm, lddh = _as_rows(dh)
    M, N, K = args.M, args.N, args.K
    new = lambda *shape: torch.empty(*shape, dtype=x.dtype, device=x.device)  # noqa: E731
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need_dx else None
    dw = torch.empty_strided((2 * N, K), (1, 2 * N) if args.w_transposed else (K, 1), dtype=x.dtype, device=x.device) if need_dw else None
    db = new(2 * N) if need_db else None
    _call(x.device, B.lib().adpsgd_gated_backward, C.byref(args), dhm.data_ptr(), lddh, slopes.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db))
    del keep
    return dx, dw, db


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, activation):
        h, slopes = _gated_forward(x, w, b, activation, True)
        ctx.save_for_backward(x, w, slopes)
        return h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        _refuse_capture("gated")
        return (*_gated_backward(dh, *ctx.saved_tensors, *ctx.needs_input_grad[:3]), None)


def gated(x, w, bias=None, *, activation="silu"):
    """act(x wg^T + bg) (x wu^T + bu) in one pass, the first half of a feed-forward block; differentiable (once, in reverse mode) in
    all three.  Its second half is dense(h, w2, residual=...).

    x (..., in), w (2 out, in) the rows of wg and then those of wu, as it is or as the transpose of an (in, 2 out) tensor, bias (2 out)
    likewise, all bfloat16 or all float16; the result is (..., out).  Activations as dense's.  Both products and theirs are in 32 bits and
    the result is rounded once.  With gradients, 4 bytes an output (float16: 6) are kept for the backward pass: its slopes for the two projections, in
    bfloat16 within 2^-10 from 2^-28 to 65504^2, 0 below 2^-50 and within 3.4 % above 65504^2 (float16: within 2^-16).  Under capture of a HIP graph the
    differentiable form is refused, as dense's is: gated_forward and gated_gradients can be captured."""
    _check_gated(x, w, bias, activation)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, w, bias)):
        _refuse_capture("gated")
        return _Gated.apply(x, w, bias, activation)
    return _gated_forward(x, w, bias, activation, False)[0]


def gated_forward(x, w, bias=None, *, activation="silu"):
    """(h, slopes): the forward pass without autograd, and what gated_gradients needs.  With relu h is gated's but for gates next to 0, whose sums are added again in
    64 bits for their slopes: there it may differ by what a sum in 32 bits is rounded by.  (gated with gradients keeps slopes too.)"""
    _check_gated(x, w, bias, activation)
    return _gated_forward(x, w, bias, activation, True)


def gated_gradients(dh, x, w, slopes, *, need=(True, True, True)):
    """(dx, dw, dbias) for dh; None where ``need`` says so.  The activation is in the slopes."""
    _check_gated(x, w, None, "none")
    _on_gpu("dh", dh, x.device)
    _on_gpu("slopes", slopes, x.device)
    if dh.dtype != x.dtype or dh.shape != (*x.shape[:-1], w.shape[0] // 2):
        raise ValueError("dh is %s %s, must be as the result" % (tuple(dh.shape), dh.dtype))
    if slopes.dtype != torch.uint8 or slopes.shape != (_SLOPE_BYTES[x.dtype] * dh.numel() * 2,) or not slopes.is_contiguous():
        raise ValueError("slopes must be what gated_forward returned")
    if not any(need):
        return None, None, None
    return _gated_backward(dh, x, w, slopes, *need)


# ---- layer norm -------------------------------------------------------------------------------------------------

_FAR = 1 << 40          # elements from one row to the next, at most, where rows are walked one by one


def _check_norm(x, w, b, dy=None):
    _on_gpu("x", x)
    T, device = x.dtype, x.device
    if T not in _TYPES:
        raise TypeError("layer_norm takes float32, bfloat16 or float16, not %s" % T)
    n = x.shape[-1] if x.dim() else 0
    if n < 1:
        raise ValueError("x is %s: the last dimension is what is normalised" % (tuple(x.shape),))
    if b is not None and w is None:
        raise ValueError("a bias without a weight")
    for name, t in (("weight", w), ("bias", b)):
        if t is None:
            continue
        _on_gpu(name, t, device)
        if (t.dtype != T and t.dtype != torch.float32) or t.dtype != w.dtype:
            raise TypeError("x is %s, %s is %s: weight and bias are both of that type or both float32" % (T, name, t.dtype))
        if t.dim() != 1 or t.numel() != n:
            raise ValueError("%s is %s, x %s" % (name, tuple(t.shape), tuple(x.shape)))
    if dy is not None:
        _on_gpu("dy", dy, device)
        if dy.dtype != T or dy.shape != x.shape:
            raise ValueError("dy is %s %s, must be as x, %s %s" % (tuple(dy.shape), dy.dtype, tuple(x.shape), T))


def _norm_args(x, w, b, eps):
    xm, ldx = _as_rows(x, _FAR)
    rows, n = xm.shape
    kind = _TYPES[x.dtype]
    w, b = (None if t is None else t.contiguous() for t in (w, b))
    return B.LayerNorm(kind, kind if w is None else _TYPES[w.dtype], rows, n, xm.data_ptr(), ldx, _ptr(w), _ptr(b), eps, None, 0), (xm, w, b)


def _norm_forward(x, w, b, eps, want_stats):
    args, keep = _norm_args(x, w, b, eps)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    stats = torch.empty(3, args.rows, dtype=torch.float32, device=x.device) if want_stats else None
    _call(x.device, B.lib().adpsgd_layer_norm_forward, C.byref(args), y.data_ptr(), _ptr(stats))
    del keep
    return y, stats


def _norm_backward(dy, x, w, stats, need_dx, need_dw, need_db):
    args, keep = _norm_args(x, w, None, 1.0)
    dym, lddy = _as_rows(dy, _FAR)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need_dx else None
    dw, db = (torch.empty_like(w, memory_format=torch.contiguous_format) if needed and w is not None else None for needed in (need_dw, need_db))
    space = None
    if dw is not None or db is not None:
        size = B.lib().adpsgd_layer_norm_workspace_bytes(args.type, args.rows, args.n)
        if size > 0:
            space = torch.empty(size, dtype=torch.uint8, device=x.device)
            args.workspace, args.workspace_bytes = space.data_ptr(), size
    _call(x.device, B.lib().adpsgd_layer_norm_backward, C.byref(args), dym.data_ptr(), lddy, stats.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db))
    del keep, space
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, eps):
        y, stats = _norm_forward(x, w, b, eps, True)
        ctx.save_for_backward(x, w, stats)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        _refuse_capture("layer_norm")
        x, w, stats = ctx.saved_tensors
        return (*_norm_backward(dy, x, w, stats, *ctx.needs_input_grad[:3]), None)


def layer_norm(x, weight=None, bias=None, *, eps=1e-5):
    """(x - mean) / sqrt(var + eps) weight + bias over the last dimension, differentiable (once, in reverse mode) in all three.

    x (..., n) float32, bfloat16 or float16; weight and bias (n) both of that type or both float32, bias only with a weight.  Means,
    variances and sums are in 32 bits or more, results are rounded once.  With gradients, 12 bytes a row are kept for the
    backward pass.  Under capture of a HIP graph the differentiable form is refused, as dense's is: layer_norm_forward and
    layer_norm_gradients can be captured."""
    _check_norm(x, weight, bias)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias)):
        _refuse_capture("layer_norm")
        return _LayerNorm.apply(x, weight, bias, eps)
    return _norm_forward(x, weight, bias, eps, False)[0]


def layer_norm_forward(x, weight=None, bias=None, *, eps=1e-5):
    """(y, stats): the forward pass without autograd, and what layer_norm_gradients needs."""
    _check_norm(x, weight, bias)
    return _norm_forward(x, weight, bias, eps, True)


def layer_norm_gradients(dy, x, weight, stats, *, need=(True, True, True)):
    """(dx, dweight, dbias) for dy; None where ``need`` says so, and without a weight for the last two."""
    _check_norm(x, weight, None, dy)
    _on_gpu("stats", stats, x.device)
    if stats.dtype != torch.float32 or stats.shape != (3, x.numel() // x.shape[-1]) or not stats.is_contiguous():
        raise ValueError("stats must be what layer_norm_forward returned")
    need = (need[0], need[1] and weight is not None, need[2] and weight is not None)
    if not any(need):
        return None, None, None
    return _norm_backward(dy, x, weight, stats, *need)


# ---- losses over a vocabulary -----------------------------------------------------------------------------------

def _logits(logits, tokens, workspace_bytes=None):
    _on_gpu("logits", logits)
    if logits.dtype not in _TYPES:
        raise TypeError("logits must be float32, bfloat16 or float16, not %s" % logits.dtype)
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be rows x vocabulary, are %s" % (tuple(logits.shape),))
    rows, vocab = logits.shape
    device = logits.device
    tokens = _vector("tokens", tokens, rows, torch.int64, device)
    z, ld = _as_rows(logits, 1 << 40)
    size = (workspace_bytes or B.lib().adpsgd_loss_workspace_bytes)(rows, vocab)
    if size < 0:
        raise B.AdpsgdError(B.ERR_ARG, "logits: %d rows of %d are too many%s" % (rows, vocab, ", or more than 1024 entries" if workspace_bytes else ""))
    space = torch.empty(size, dtype=torch.uint8, device=device)
    return (B.Logits(_TYPES[z.dtype], 0, rows, vocab, z.data_ptr(), ld, tokens.data_ptr(), space.data_ptr(), size), rows, device, (z, tokens, space))


def token_log_probs(logits, tokens):
    """log softmax(logits)[i, tokens[i]] as float32, without autograd; 0 where tokens[i] is negative (that row is not read)."""
    args, rows, dev, keep = _logits(logits, tokens)
    out = torch.empty(rows, dtype=torch.float32, device=dev)
    _call(dev, B.lib().adpsgd_token_log_probs, C.byref(args), out.data_ptr())
    del keep
    return out


def policy_loss_and_gradient(logits, tokens, old_log_probs, advantages, ref_log_probs=None, *, clip=(0.2, 0.2), kl_coef=0.0):
    """Clipped policy loss with a KL term (see adpsgd_policy_loss), a mean over the rows whose token is not negative, and its
    gradient for the logits.  loss is a scalar tensor; dlogits has the logits' shape and type; log_probs is float32."""
    args, rows, dev, keep = _logits(logits, tokens)
    old = _vector("old_log_probs", old_log_probs, rows, torch.float32, dev)
    adv = _vector("advantages", advantages, rows, torch.float32, dev)
    ref = None if ref_log_probs is None else _vector("ref_log_probs", ref_log_probs, rows, torch.float32, dev)
    loss, logp = torch.empty((), dtype=torch.float32, device=dev), torch.empty(rows, dtype=torch.float32, device=dev)
    dz = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    _call(dev, B.lib().adpsgd_policy_loss, C.byref(args), old.data_ptr(), adv.data_ptr(), _ptr(ref), clip[0], clip[1], kl_coef, loss.data_ptr(),
          dz.data_ptr(), logp.data_ptr())
    del keep
    return PolicyLoss(loss, dz, logp)


def preference_loss_and_gradient(logits, tokens, offsets, ref_log_probs, *, beta=0.1, label_smoothing=0.0):
    """Preference loss of paired answers (see adpsgd_preference_loss) and its gradient for the logits.  The rows of sequence q are
    offsets[q] .. offsets[q + 1]; the first half of the sequences are the chosen answers, the other half their rejected ones in
    the same order.  ref_log_probs: sums over each sequence under the reference model.  log_probs are those sums under this one."""
    args, rows, dev, keep = _logits(logits, tokens)
    _on_gpu("offsets", offsets, dev)
    if offsets.dim() != 1 or offsets.dtype != torch.int64 or offsets.numel() < 3 or offsets.numel() % 2 == 0:
        raise ValueError("offsets must be 2 pairs + 1 int64, are %s %s" % (tuple(offsets.shape), offsets.dtype))
    pairs = offsets.numel() // 2
    offsets = offsets.contiguous()
    ref = _vector("ref_log_probs", ref_log_probs, 2 * pairs, torch.float32, dev)
    new = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)  # noqa: E731
    loss, sums, margins = new(), new(2 * pairs), new(pairs)
    dz = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    _call(dev, B.lib().adpsgd_preference_loss, C.byref(args), offsets.data_ptr(), pairs, ref.data_ptr(), beta, label_smoothing, loss.data_ptr(),
          dz.data_ptr(), sums.data_ptr(), margins.data_ptr())
    del keep
    return PreferenceLoss(loss, dz, sums, margins)


def _teacher_rows(name, t, rows, device):
    """t as rows x k with a contiguous last dimension, and its leading dimension."""
    _on_gpu(name, t, device)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < 1:
        raise ValueError("%s is %s, must be rows x entries of %d rows" % (name, tuple(t.shape), rows))
    return _as_rows(t, _FAR)


def distillation_loss_and_gradient(logits, tokens, teacher_tokens, teacher_logits, *, temperature=1.0, hard_weight=0.0, loss_scale=1.0):
    """(1 - hard_weight) T^2 KL(teacher || softmax(logits / T)) - hard_weight log softmax(logits)[token] (see adpsgd_distillation_loss), a mean over the
    rows whose token is not negative, and its gradient for the logits.

    The teacher of a row is the softmax of teacher_logits / T (rows x k, any of the types) over its entries teacher_tokens (rows x k,
    int64): its k <= 1024 largest logits, say; an entry with a negative token is not used.  loss is a scalar tensor; dlogits has the logits'
    shape and type, and is the gradient of loss_scale times the loss, for logits in float16 (AdamW.step's grad_scale takes it off again); divergences
    (KL of each row) and log_probs (of the tokens; None where hard_weight is 0) are float32."""
    _on_gpu("logits", logits)
    tt, ld_tokens = _teacher_rows("teacher_tokens", teacher_tokens, logits.shape[0] if logits.dim() else 0, logits.device)
    tz, ld = _teacher_rows("teacher_logits", teacher_logits, tt.shape[0], logits.device)
    if tt.dtype != torch.int64 or tz.dtype not in _TYPES or tz.shape != tt.shape:
        raise TypeError("teacher_tokens must be int64 and teacher_logits of the same shape, float32, bfloat16 or float16: they are %s %s, %s %s"
                        % (tuple(tt.shape), tt.dtype, tuple(tz.shape), tz.dtype))
    k = tt.shape[1]
    args, rows, dev, keep = _logits(logits, tokens, lambda rows, vocab: B.lib().adpsgd_distillation_workspace_bytes(rows, vocab, k))
    teacher = B.Teacher(_TYPES[tz.dtype], 0, k, tt.data_ptr(), ld_tokens, tz.data_ptr(), ld)
    new = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)  # noqa: E731
    loss, kl, logp = new(), new(rows), new(rows) if hard_weight else None
    dz = torch.empty_like(logits, memory_format=torch.contiguous_format)
    _call(dev, B.lib().adpsgd_distillation_loss, C.byref(args), C.byref(teacher), temperature, hard_weight, loss_scale, loss.data_ptr(), dz.data_ptr(),
          kl.data_ptr(), _ptr(logp))
    del keep
    return DistillationLoss(loss, dz, kl, logp)


# ---- AdamW ------------------------------------------------------------------------------------------------------

class AdamW:
    """AdamW over all tensors of a model in one or two launches a step (see adpsgd_adamw_opts_t).

    params, grads: lists of contiguous tensors, each list of one type; they are read and written where they lie, for the life of
    the object.  masters: float32 copies that are stepped, with the params as their roundings.  out: float32 tensors that
    receive the direction u + weight_decay p in place of a step.  weight_decay: a number, or one for each tensor.  state_bits 32 or
    8.  ``lr`` may be changed between steps.  A step raises the versions of the tensors that it writes, as other changes in place do."""

    def __init__(self, params, grads, *, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, state_bits=32, masters=None, out=None, seed=0):
        self._h = None
        params, grads = list(params), list(grads)
        if not params or len(params) != len(grads):
            raise ValueError("params and grads must be lists of the same length, not empty")
        dev = params[0].device if isinstance(params[0], torch.Tensor) else None
        lists = [("params", params, None), ("grads", grads, None), ("masters", masters, torch.float32), ("out", out, torch.float32)]
        self._tensors = []                      # what the library reads and writes stays alive
        for name, ts, dtype in lists:
            if ts is None:
                self._tensors.append(None)
                continue
            ts = list(ts)
            if len(ts) != len(params):
                raise ValueError("%s has %d tensors, params %d" % (name, len(ts), len(params)))
            for t, p in zip(ts, params):
                _on_gpu(name, t, dev)
                if t.dtype not in _TYPES or t.dtype != (dtype or ts[0].dtype):
                    raise TypeError("%s must be %s" % (name, dtype or "float32, bfloat16 or float16, all the same"))
                if not t.is_contiguous() or t.numel() != p.numel():
                    raise ValueError("%s must be contiguous, of as many elements as params" % name)
            self._tensors.append([t.detach() for t in ts])
        n = len(params)
        decay = np.ascontiguousarray(np.broadcast_to(np.asarray(weight_decay, dtype=np.float32), (n,)))
        sizes = (C.c_int64 * n)(*(t.numel() for t in params))
        length = B.lib().adpsgd_adamw_state_length(sizes, n)
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        kind = torch.float32 if state_bits == 32 else torch.uint8
        self.lr, self.state_bits, self.device, self.state_length = lr, state_bits, dev, length
        self._m, self._v = (torch.zeros(length, dtype=kind, device=dev) for _ in range(2))
        self._exponents = torch.zeros(2 * (length // 256), dtype=torch.int8, device=dev) if state_bits == 8 else None
        pointers = lambda ts: None if ts is None else (C.c_void_p * n)(*(t.data_ptr() for t in ts))  # noqa: E731
        p, g, ma, o = (pointers(ts) for ts in self._tensors)
        opts = B.AdamwOpts(n, _TYPES[params[0].dtype], _TYPES[grads[0].dtype], state_bits, sizes, p, g, ma, o,
                           decay.ctypes.data_as(C.POINTER(C.c_float)), betas[0], betas[1], eps, int(seed) & 0xFFFFFFFFFFFFFFFF,
                           self._m.data_ptr(), self._v.data_ptr(), _ptr(self._exponents))
        h = C.c_void_p()
        with torch.cuda.device(dev):
            torch.cuda.current_stream().synchronize()       # the state is there for whatever stream the steps are on
            rc = B.lib().adpsgd_adamw_create(C.byref(h), C.byref(opts))
        if rc != B.OK:
            raise B.AdpsgdError(rc, (B.lib().adpsgd_last_error(None) or b"").decode())
        self._h = h
        # what a step writes, for autograd's check of tensors that were saved for a backward pass
        params, _, masters, out = self._tensors
        self._written = params + (masters or []) if out is None else out

    def close(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            try:
                B.lib().adpsgd_adamw_destroy(h)
            except (AttributeError, TypeError):    # interpreter shutdown: the module globals are already gone
                pass

    __del__ = close

    def _open(self):
        if not self._h:
            raise RuntimeError("the optimizer is closed")
        return self._h

    @property
    def steps(self):
        out = C.c_int64()
        B.lib().adpsgd_adamw_get_steps(self._open(), C.byref(out))
        return out.value

    def step(self, *, max_norm=0.0, grad_scale=1.0):
        """One step on the current stream.  max_norm: gradients times grad_scale are scaled down to this norm over all tensors;
        the norm before that is returned as a scalar tensor (None with 0: no clipping, no norm)."""
        norm = torch.empty((), dtype=torch.float32, device=self.device) if max_norm else None
        _call(self.device, B.lib().adpsgd_adamw_step, self._open(), self.lr, max_norm, grad_scale, _ptr(norm))
        torch.autograd.graph.increment_version(self._written)
        return norm

    def moments(self):
        """(m, v), each tensor's from a multiple of 256 on.  state_bits 32: the state itself; 8: what it stands for, as bfloat16,
        which holds those values exactly."""
        if self.state_bits == 32:
            return self._m, self._v
        m, v = (torch.empty(self.state_length, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        _call(self.device, B.lib().adpsgd_adamw_get_moments, self._open(), m.data_ptr(), v.data_ptr())
        return m, v

    def load_moments(self, m, v, steps):
        """Continue from stored moments (any float type; 8 bits: rounded to the nearest) after ``steps`` steps."""
        for name, t in (("m", m), ("v", v)):
            _on_gpu(name, t, self.device)
            if t.shape != (self.state_length,):
                raise ValueError("%s must have %d elements" % (name, self.state_length))
        if int(steps) < 0:
            raise ValueError("steps must not be negative")
        if self.state_bits == 32:
            self._m.copy_(m)
            self._v.copy_(v)
        else:
            m, v = m.float().contiguous(), v.float().contiguous()
            _call(self.device, B.lib().adpsgd_adamw_set_moments, self._open(), m.data_ptr(), v.data_ptr())
        B.lib().adpsgd_adamw_set_steps(self._open(), int(steps))

    def state_dict(self):
        """A copy of the state as it is kept, and the number of steps."""
        parts = {"m": self._m, "v": self._v, "exponents": self._exponents}
        return dict({k: t.clone() for k, t in parts.items() if t is not None}, steps=self.steps)

    def load_state_dict(self, state):
        """Continue from a state_dict.  One that does not fit is refused and changes nothing."""
        h = self._open()
        parts = [(k, t, state[k]) for k, t in (("m", self._m), ("v", self._v), ("exponents", self._exponents)) if t is not None]
        steps = int(state["steps"])
        for k, t, stored in parts:
            if stored.shape != t.shape or stored.dtype != t.dtype:
                raise ValueError("%s of the stored state is %s %s, here %s %s" % (k, tuple(stored.shape), stored.dtype, tuple(t.shape), t.dtype))
        if B.lib().adpsgd_adamw_set_steps(h, steps) != B.OK:
            raise ValueError("the stored state has %d steps" % steps)
        for _, t, stored in parts:
            t.copy_(stored)
