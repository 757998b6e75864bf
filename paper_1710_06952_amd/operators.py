"""Operators of a worker's own training step on torch tensors: dense layers, log-probabilities and losses over a
vocabulary, AdamW over many tensors.  The same entry points as include/adpsgd.h; every computation runs in the HIP
library, on the current stream of the tensors' device.

    y = dense(x, w, bias, residual=r, activation="gelu")           # differentiable
    lp = token_log_probs(logits, tokens)                           # of a frozen model, or to sample with
    r = policy_loss_and_gradient(logits, tokens, old, advantages, ref, clip=(0.2, 0.2), kl_coef=0.05)
    r = preference_loss_and_gradient(logits, tokens, offsets, ref, beta=0.1)
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


# ---- losses over a vocabulary -----------------------------------------------------------------------------------

def _logits(logits, tokens):
    _on_gpu("logits", logits)
    if logits.dtype not in _TYPES:
        raise TypeError("logits must be float32, bfloat16 or float16, not %s" % logits.dtype)
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be rows x vocabulary, are %s" % (tuple(logits.shape),))
    rows, vocab = logits.shape
    device = logits.device
    tokens = _vector("tokens", tokens, rows, torch.int64, device)
    z, ld = _as_rows(logits, 1 << 40)
    size = B.lib().adpsgd_loss_workspace_bytes(rows, vocab)
    if size < 0:
        raise B.AdpsgdError(B.ERR_ARG, "logits: %d rows of %d are too many" % (rows, vocab))
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
