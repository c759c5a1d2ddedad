"""Operators of a language model's training micro-batch (include/abs_llm.h) on CUDA tensors.

They are the parts of a forward and backward pass that lie around its matrix products; the flat gradient that comes out
goes to ``AbsSgd.accumulate``.  Every function checks its arguments, allocates its outputs and workspace from PyTorch's
allocator and enqueues on the current stream of the tensors' device; nothing synchronises.  Outputs that are given are
used as they are.  Refused arguments raise ``ValueError`` / ``TypeError`` here or ``binding.AbsError`` from the library.
Matrices may have any row stride; a row is contiguous.  Shapes are [tokens, width]: flatten leading dimensions with
``view``.
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as _b

_lib = _b.lib
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
_DTYPE = {_F32: _b.GRAD_F32, _BF16: _b.GRAD_BF16}
_GATE_NONE, _GATE_CHANNEL, _GATE_ELEMENT = 0, 1, 2


class PolicyLoss(NamedTuple):
    loss: torch.Tensor       # sum_t weight_t loss_t
    kl: torch.Tensor         # sum_t weight_t kl_t, without the coefficient
    clipped: torch.Tensor    # sum_t weight_t [t clipped]
    logp: torch.Tensor       # [tokens]; 0 where a token is left out
    dlogits: Optional[torch.Tensor]


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor
    pair_loss: torch.Tensor  # [pairs]
    seq_logp: torch.Tensor   # [2 pairs]
    dlogits: Optional[torch.Tensor]


class ResidualGrads(NamedTuple):
    dx: torch.Tensor
    dh: torch.Tensor
    dgate: Optional[torch.Tensor]
    dw_pre: torch.Tensor
    dw_post: Optional[torch.Tensor]


class Ckpt8(NamedTuple):
    """An activation [tokens, width] in 8 bits: value = q * 2**(e - 127), one e for 32 values of a row."""

    q: torch.Tensor          # int8  [tokens, width rounded up to 32]
    e: torch.Tensor          # uint8 [tokens, same / 32]
    width: int


def _refuse(rc):
    raise _b.AbsError(rc, _lib.abs_last_error(None).decode())


def _matrix(t, name, dtype=None, shape=None):
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of two dimensions")
    if t.dtype not in _DTYPE if dtype is None else t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}" + (f", {dtype} is wanted" if dtype else ", float32 or bfloat16 is wanted"))
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {tuple(shape)} is wanted")
    if t.stride(1) != 1 and t.shape[1] > 1 or t.stride(0) < t.shape[1] and t.shape[0] > 1:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap")
    return t


def _vector(t, name, n, dtype, device):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device:
        raise TypeError(f"{name} must be a {dtype} tensor on {device}")
    if t.dim() != 1 or t.shape[0] != n or n > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous with {n} elements")
    return t


def _same_device(device, *ts):
    for t in ts:
        if t is not None and t.device != device:
            raise ValueError("the tensors are on different devices")


def _ld(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _addr(t):
    return None if t is None else t.data_ptr()


def _call(device, fn, *args):
    """fn(*args, stream) with `device` current, on its current stream."""
    stream = torch.cuda.current_stream(device).cuda_stream
    if device.index == torch.cuda.current_device():
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream)
    if rc != _b.OK:
        _refuse(rc)


def _workspace(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device)


def _dlogits(logits, dlogits, need_grad):
    if not need_grad:
        if dlogits is not None:
            raise ValueError("dlogits is given but need_grad is False")
        return None
    if dlogits is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _matrix(dlogits, "dlogits", logits.dtype, logits.shape)
    _same_device(logits.device, dlogits)
    return dlogits


def policy_loss(logits, labels, logp_old, advantage, weight, logp_ref=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, dlogits=None, need_grad: bool = True) -> PolicyLoss:
    """Clipped policy loss with a KL term to a reference model, with the gradient of the logits (``abs_policy_loss``).

    logits [tokens, vocab] float32 / bfloat16; labels int32; logp_old, advantage, weight, logp_ref float32 [tokens].
    weight is a token's share of the loss (1 / n for the mean over n tokens); tokens of weight 0 or with a label outside
    [0, vocab) are left out.  dlogits may be the logits themselves."""
    T, V = _matrix(logits, "logits").shape
    dev = logits.device
    _vector(labels, "labels", T, _I32, dev)
    for t, name in ((logp_old, "logp_old"), (advantage, "advantage"), (weight, "weight")):
        _vector(t, name, T, _F32, dev)
    if logp_ref is not None:
        _vector(logp_ref, "logp_ref", T, _F32, dev)
    d = _dlogits(logits, dlogits, need_grad)
    out = torch.empty(T + 3, dtype=_F32, device=dev)
    n = _POLICY_WORKSPACE
    ws = _workspace(n, dev)
    at = out.data_ptr()
    _call(dev, _lib.abs_policy_loss, logits.data_ptr(), _DTYPE[logits.dtype], T, V, _ld(logits), labels.data_ptr(), logp_old.data_ptr(),
          _addr(logp_ref), advantage.data_ptr(), weight.data_ptr(), clip_low, clip_high, kl_coef, at, at + 12, _addr(d),
          _ld(d) if d is not None else 0, ws.data_ptr(), n)
    return PolicyLoss(out[0], out[1], out[2], out[3:], d)


_POLICY_WORKSPACE = int(_lib.abs_policy_loss_workspace())


def preference_loss(logits, labels, offsets, logp_ref, beta: float = 0.1, smoothing: float = 0.0, scale: Optional[float] = None,
                    dlogits=None, need_grad: bool = True) -> PreferenceLoss:
    """Paired preference loss with the gradient of the logits (``abs_preference_loss``).

    logits [tokens, vocab]: the rows of the answers one after the other, answers 2 p and 2 p + 1 the preferred and the
    other one of pair p; offsets int32 [2 pairs + 1]: their first rows; labels int32 [tokens], outside [0, vocab) for rows
    that do not count; logp_ref float32 [2 pairs]: the reference model's log-probabilities.  scale: 1 / pairs if not given."""
    T, V = _matrix(logits, "logits").shape
    dev = logits.device
    _vector(labels, "labels", T, _I32, dev)
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] % 2 != 1:
        raise ValueError("offsets must have 2 pairs + 1 elements")
    pairs = offsets.shape[0] // 2
    _vector(offsets, "offsets", 2 * pairs + 1, _I32, dev)
    _vector(logp_ref, "logp_ref", 2 * pairs, _F32, dev)
    d = _dlogits(logits, dlogits, need_grad)
    out = torch.empty(3 * pairs + 1, dtype=_F32, device=dev)
    n = int(_lib.abs_preference_loss_workspace(T))
    ws = _workspace(n, dev)
    at = out.data_ptr()
    _call(dev, _lib.abs_preference_loss, logits.data_ptr(), _DTYPE[logits.dtype], T, V, _ld(logits), labels.data_ptr(), offsets.data_ptr(),
          pairs, logp_ref.data_ptr(), beta, smoothing, (1.0 / pairs if pairs else 0.0) if scale is None else scale, at, at + 4,
          at + 4 + 4 * pairs, _addr(d), _ld(d) if d is not None else 0, ws.data_ptr(), n)
    return PreferenceLoss(out[0], out[1:1 + pairs], out[1 + pairs:], d)


def _gate_kind(gate, like, width):
    if gate is None:
        return _GATE_NONE
    if isinstance(gate, torch.Tensor) and gate.dim() == 1:
        _vector(gate, "gate", width, _F32, like.device)
        return _GATE_CHANNEL
    _matrix(gate, "gate", like.dtype, like.shape)
    _same_device(like.device, gate)
    return _GATE_ELEMENT


def _out_matrix(t, name, like):
    if t is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    _matrix(t, name, like.dtype, like.shape)
    _same_device(like.device, t)
    return t


def residual_norm(x, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, y=None, n=None):
    """(y, n): y = scale x + G u, u = h / rms(h) w_post (h without w_post), n = y / rms(y) w_pre (``abs_residual_norm``).

    x, h [tokens, width] float32 / bfloat16; w_pre, w_post float32 [width].  gate: None (G = 1), float32 [width] (G = gate)
    or [tokens, width] of x's dtype (G = sigmoid(gate)).  y may be x, n may be h."""
    T, D = _matrix(x, "x").shape
    dev = x.device
    _matrix(h, "h", x.dtype, x.shape)
    _same_device(dev, h)
    _vector(w_pre, "w_pre", D, _F32, dev)
    if w_post is not None:
        _vector(w_post, "w_post", D, _F32, dev)
    kind = _gate_kind(gate, x, D)
    y, n = _out_matrix(y, "y", x), _out_matrix(n, "n", x)
    _call(dev, _lib.abs_residual_norm, x.data_ptr(), _ld(x), h.data_ptr(), _ld(h), _addr(gate), _ld(gate) if kind == _GATE_ELEMENT else 0, kind,
          _addr(w_post), w_pre.data_ptr(), scale, eps, _DTYPE[x.dtype], T, D, y.data_ptr(), _ld(y), n.data_ptr(), _ld(n))
    return y, n


def residual_norm_backward(dn, dy, y, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, dx=None, dh=None,
                           dgate=None, dw_pre=None, dw_post=None, accumulate: bool = False) -> ResidualGrads:
    """Gradients of ``residual_norm`` from dn and dy (None: nothing else reads y) at the stored y and h.

    dw_pre, dw_post and a channel gate's dgate (float32 [width]) may be slices of a flat gradient; with accumulate the
    sums are added to what the given ones hold (those that are not given start at zero)."""
    T, D = _matrix(y, "y").shape
    dev, dt, shape = y.device, y.dtype, y.shape
    _matrix(dn, "dn", dt, shape)
    _matrix(h, "h", dt, shape)
    if dy is not None:
        _matrix(dy, "dy", dt, shape)
    _same_device(dev, dn, h, dy)
    _vector(w_pre, "w_pre", D, _F32, dev)
    if w_post is not None:
        _vector(w_post, "w_post", D, _F32, dev)
    kind = _gate_kind(gate, y, D)
    dx, dh = _out_matrix(dx, "dx", y), _out_matrix(dh, "dh", y)
    fresh = torch.zeros if accumulate else torch.empty

    def column(t, name):
        return fresh(D, dtype=_F32, device=dev) if t is None else _vector(t, name, D, _F32, dev)

    dw_pre = column(dw_pre, "dw_pre")
    if w_post is not None:
        dw_post = column(dw_post, "dw_post")
    elif dw_post is not None:
        raise ValueError("dw_post without w_post")
    if kind == _GATE_CHANNEL:
        dgate = column(dgate, "dgate")
    elif kind == _GATE_ELEMENT:
        dgate = _out_matrix(dgate, "dgate", y)
    elif dgate is not None:
        raise ValueError("dgate without a gate")
    n = int(_lib.abs_residual_norm_workspace(T, D))
    ws = _workspace(n, dev)
    element = kind == _GATE_ELEMENT
    _call(dev, _lib.abs_residual_norm_backward, dn.data_ptr(), _ld(dn), _addr(dy), _ld(dy) if dy is not None else 0, y.data_ptr(), _ld(y),
          h.data_ptr(), _ld(h), _addr(gate), _ld(gate) if element else 0, kind, _addr(w_post), w_pre.data_ptr(), scale, eps, _DTYPE[dt], T, D,
          dx.data_ptr(), _ld(dx), dh.data_ptr(), _ld(dh), _addr(dgate), _ld(dgate) if element else 0, dw_pre.data_ptr(), _addr(dw_post),
          int(accumulate), ws.data_ptr(), n)
    return ResidualGrads(dx, dh, dgate, dw_pre, dw_post)


def ckpt8_quantize(x) -> Ckpt8:
    """An activation [tokens, width] (float32 / bfloat16) in 8 bits (``abs_ckpt8_quantize``)."""
    T, D = _matrix(x, "x").shape
    W = (D + 31) // 32 * 32
    q = torch.empty((T, W), dtype=torch.int8, device=x.device)
    e = torch.empty((T, W // 32), dtype=torch.uint8, device=x.device)
    _call(x.device, _lib.abs_ckpt8_quantize, x.data_ptr(), _ld(x), _DTYPE[x.dtype], T, D, q.data_ptr(), e.data_ptr())
    return Ckpt8(q, e, D)


def _ckpt(c):
    W = (c.width + 31) // 32 * 32
    q, e = c.q, c.e
    if q.dtype != torch.int8 or e.dtype != torch.uint8 or not q.is_cuda or q.device != e.device:
        raise TypeError("a Ckpt8 holds an int8 and a uint8 tensor on one CUDA device")
    if q.dim() != 2 or q.shape[1] != W or e.shape != (q.shape[0], W // 32) or not q.is_contiguous() or not e.is_contiguous():
        raise ValueError("a Ckpt8 holds q [tokens, width rounded up to 32] and e [tokens, same / 32], contiguous")
    return q, e


def ckpt8_dequantize(c: Ckpt8, dtype=torch.bfloat16, out=None):
    """The values that a Ckpt8 stands for, [tokens, width]."""
    q, e = _ckpt(c)
    if out is None:
        out = torch.empty((q.shape[0], c.width), dtype=dtype, device=q.device)
    _matrix(out, "out", dtype, (q.shape[0], c.width))
    _same_device(q.device, out)
    if dtype not in _DTYPE:
        raise TypeError("dtype must be float32 or bfloat16")
    _call(q.device, _lib.abs_ckpt8_dequantize, q.data_ptr(), e.data_ptr(), q.shape[0], c.width, out.data_ptr(), _ld(out), _DTYPE[dtype])
    return out


def ckpt8_wgrad(c: Ckpt8, dy, out=None, accumulate: bool = False):
    """x^T dy of the activation x that `c` stands for: the gradient of a weight stored [in, out] (``abs_ckpt8_wgrad``).

    dy bfloat16 [tokens, out].  out float32 [width, out], for instance a view of a flat gradient; accumulate adds to it."""
    q, e = _ckpt(c)
    T, N = _matrix(dy, "dy", _BF16).shape
    if T != q.shape[0]:
        raise ValueError(f"dy has {T} rows, the checkpoint {q.shape[0]}")
    dev = q.device
    _same_device(dev, dy)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out to add to")
        out = torch.empty((c.width, N), dtype=_F32, device=dev)
    else:
        _matrix(out, "out", _F32, (c.width, N))
        _same_device(dev, out)
    ld = _ld(dy)
    n = int(_lib.abs_ckpt8_wgrad_workspace(T, c.width, N, dy.data_ptr(), ld))
    ws = _workspace(n, dev) if n else None
    _call(dev, _lib.abs_ckpt8_wgrad, q.data_ptr(), e.data_ptr(), dy.data_ptr(), ld, T, c.width, N, out.data_ptr(), _ld(out), int(accumulate),
          _addr(ws), n)
    return out


def check(device=None):
    """Blocks until the current stream has finished; raises if a kernel of this module gave up a bounded wait."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    _call(device, _lib.abs_llm_check)
