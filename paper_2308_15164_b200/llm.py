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


_empty, _empty_like, _Tensor = torch.empty, torch.empty_like, torch.Tensor
_stream_of = torch._C._cuda_getCurrentRawStream      # what torch.cuda.current_stream(d).cuda_stream returns, 2 us sooner


def _first(t, name):
    """(dtype code, rows, columns, device index) of the matrix that the others have to agree with."""
    if not isinstance(t, _Tensor) or not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name} must be a CUDA tensor of two dimensions")
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} has dtype {t.dtype}, float32 or bfloat16 is wanted")
    rows, cols = t.shape
    return code, rows, cols, t.get_device()


def _matrix(t, name, dtype, rows, cols, index):
    """(address, leading dimension) of a [rows, cols] matrix on CUDA device `index`."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.get_device() != index:
        raise TypeError(f"{name} must be a {dtype} tensor on cuda:{index}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {(rows, cols)} is wanted")
    if t.is_contiguous():
        return t.data_ptr(), cols
    down, along = t.stride()
    if along != 1 and cols > 1 or down < cols and rows > 1:
        raise ValueError(f"{name}: rows must be contiguous and must not overlap")
    return t.data_ptr(), max(down, cols)


def _vector(t, name, n, dtype, index):
    """Address of a contiguous vector of n elements on CUDA device `index`."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.get_device() != index:
        raise TypeError(f"{name} must be a {dtype} tensor on cuda:{index}")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} elements")
    return t.data_ptr()


def _call(index, fn, *args):
    """fn(*args, stream) with device `index` current, on its current stream."""
    if index == torch._C._cuda_getDevice():
        rc = fn(*args, _stream_of(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _stream_of(index))
    if rc:
        _refuse(rc)


def _workspace(n, like):
    return _empty(n, dtype=torch.uint8, device=like.device)


def _out(t, name, like, index):
    """(tensor, address, leading dimension) of an output of `like`'s type and shape; made if not given."""
    if t is None:
        t = _empty_like(like) if like.is_contiguous() else like.new_empty(like.shape)
        return t, t.data_ptr(), like.shape[1]
    rows, cols = like.shape
    return (t, *_matrix(t, name, like.dtype, rows, cols, index))


def _dlogits(logits, dlogits, need_grad, index):
    if need_grad:
        return _out(dlogits, "dlogits", logits, index)
    if dlogits is not None:
        raise ValueError("dlogits is given but need_grad is False")
    return None, None, 0


def policy_loss(logits, labels, logp_old, advantage, weight, logp_ref=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, dlogits=None, need_grad: bool = True) -> PolicyLoss:
    """Clipped policy loss with a KL term to a reference model, with the gradient of the logits (``abs_policy_loss``).

    logits [tokens, vocab] float32 / bfloat16; labels int32; logp_old, advantage, weight, logp_ref float32 [tokens].
    weight is a token's share of the loss (1 / n for the mean over n tokens); tokens of weight 0 or with a label outside
    [0, vocab) are left out.  dlogits may be the logits themselves."""
    code, T, V, dev = _first(logits, "logits")
    z, ld = _matrix(logits, "logits", logits.dtype, T, V, dev)
    y = _vector(labels, "labels", T, _I32, dev)
    old = _vector(logp_old, "logp_old", T, _F32, dev)
    adv = _vector(advantage, "advantage", T, _F32, dev)
    w = _vector(weight, "weight", T, _F32, dev)
    ref = None if logp_ref is None else _vector(logp_ref, "logp_ref", T, _F32, dev)
    d, da, ld_d = _dlogits(logits, dlogits, need_grad, dev)
    logp = _empty_like(weight)
    stats = weight.new_empty(3)
    ws = _workspace(_POLICY_WORKSPACE, logits)
    _call(dev, _lib.abs_policy_loss, z, code, T, V, ld, y, old, ref, adv, w, clip_low, clip_high, kl_coef, stats.data_ptr(), logp.data_ptr(), da,
          ld_d, ws.data_ptr(), _POLICY_WORKSPACE)
    return PolicyLoss(*stats.unbind(), logp, d)


_POLICY_WORKSPACE = int(_lib.abs_policy_loss_workspace())


def preference_loss(logits, labels, offsets, logp_ref, beta: float = 0.1, smoothing: float = 0.0, scale: Optional[float] = None,
                    dlogits=None, need_grad: bool = True) -> PreferenceLoss:
    """Paired preference loss with the gradient of the logits (``abs_preference_loss``).

    logits [tokens, vocab]: the rows of the answers one after the other, answers 2 p and 2 p + 1 the preferred and the
    other one of pair p; offsets int32 [2 pairs + 1]: their first rows; labels int32 [tokens], outside [0, vocab) for rows
    that do not count; logp_ref float32 [2 pairs]: the reference model's log-probabilities.  scale: 1 / pairs if not given."""
    code, T, V, dev = _first(logits, "logits")
    z, ld = _matrix(logits, "logits", logits.dtype, T, V, dev)
    y = _vector(labels, "labels", T, _I32, dev)
    if not isinstance(offsets, _Tensor) or offsets.dim() != 1 or offsets.shape[0] % 2 != 1:
        raise ValueError("offsets must have 2 pairs + 1 elements")
    pairs = offsets.shape[0] // 2
    off = _vector(offsets, "offsets", 2 * pairs + 1, _I32, dev)
    ref = _vector(logp_ref, "logp_ref", 2 * pairs, _F32, dev)
    d, da, ld_d = _dlogits(logits, dlogits, need_grad, dev)
    seq_logp = _empty_like(logp_ref)
    pair_loss, loss = logp_ref.new_empty(pairs), logp_ref.new_empty(())
    n = _lib.abs_preference_loss_workspace(T)
    ws = _workspace(n, logits)
    if scale is None:
        scale = 1.0 / pairs if pairs else 0.0
    _call(dev, _lib.abs_preference_loss, z, code, T, V, ld, y, off, pairs, ref, beta, smoothing, scale, loss.data_ptr(), pair_loss.data_ptr(),
          seq_logp.data_ptr(), da, ld_d, ws.data_ptr(), n)
    return PreferenceLoss(loss, pair_loss, seq_logp, d)


def _gate(gate, like, rows, cols, index):
    """(kind, address, leading dimension)"""
    if gate is None:
        return _GATE_NONE, None, 0
    if isinstance(gate, _Tensor) and gate.dim() == 1:
        return _GATE_CHANNEL, _vector(gate, "gate", cols, _F32, index), 0
    return (_GATE_ELEMENT, *_matrix(gate, "gate", like.dtype, rows, cols, index))


def residual_norm(x, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, y=None, n=None):
    """(y, n): y = scale x + G u, u = h / rms(h) w_post (h without w_post), n = y / rms(y) w_pre (``abs_residual_norm``).

    x, h [tokens, width] float32 / bfloat16; w_pre, w_post float32 [width].  gate: None (G = 1), float32 [width] (G = gate)
    or [tokens, width] of x's dtype (G = sigmoid(gate)).  y may be x, n may be h."""
    code, T, D, dev = _first(x, "x")
    dt = x.dtype
    xa, ld_x = _matrix(x, "x", dt, T, D, dev)
    ha, ld_h = _matrix(h, "h", dt, T, D, dev)
    pre = _vector(w_pre, "w_pre", D, _F32, dev)
    post = None if w_post is None else _vector(w_post, "w_post", D, _F32, dev)
    kind, ga, ld_g = _gate(gate, x, T, D, dev)
    y, ya, ld_y = _out(y, "y", x, dev)
    n, na, ld_n = _out(n, "n", x, dev)
    _call(dev, _lib.abs_residual_norm, xa, ld_x, ha, ld_h, ga, ld_g, kind, post, pre, scale, eps, code, T, D, ya, ld_y, na, ld_n)
    return y, n


def residual_norm_backward(dn, dy, y, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, dx=None, dh=None,
                           dgate=None, dw_pre=None, dw_post=None, accumulate: bool = False) -> ResidualGrads:
    """Gradients of ``residual_norm`` from dn and dy (None: nothing else reads y) at the stored y and h.

    dw_pre, dw_post and a channel gate's dgate (float32 [width]) may be slices of a flat gradient; with accumulate the
    sums are added to what the given ones hold (those that are not given start at zero)."""
    code, T, D, dev = _first(y, "y")
    dt = y.dtype
    ya, ld_y = _matrix(y, "y", dt, T, D, dev)
    dna, ld_dn = _matrix(dn, "dn", dt, T, D, dev)
    ha, ld_h = _matrix(h, "h", dt, T, D, dev)
    dya, ld_dy = (None, 0) if dy is None else _matrix(dy, "dy", dt, T, D, dev)
    pre = _vector(w_pre, "w_pre", D, _F32, dev)
    post = None if w_post is None else _vector(w_post, "w_post", D, _F32, dev)
    kind, ga, ld_g = _gate(gate, y, T, D, dev)
    dx, dxa, ld_dx = _out(dx, "dx", y, dev)
    dh, dha, ld_dh = _out(dh, "dh", y, dev)

    def column(t, name):
        if t is None:
            t = torch.zeros_like(w_pre) if accumulate else _empty_like(w_pre)
            return t, t.data_ptr()
        return t, _vector(t, name, D, _F32, dev)

    dw_pre, dpre = column(dw_pre, "dw_pre")
    dpost, dga, ld_dg = None, None, 0
    if post is not None:
        dw_post, dpost = column(dw_post, "dw_post")
    elif dw_post is not None:
        raise ValueError("dw_post without w_post")
    if kind == _GATE_CHANNEL:
        dgate, dga = column(dgate, "dgate")
    elif kind == _GATE_ELEMENT:
        dgate, dga, ld_dg = _out(dgate, "dgate", y, dev)
    elif dgate is not None:
        raise ValueError("dgate without a gate")
    n = _lib.abs_residual_norm_workspace(T, D)
    ws = _workspace(n, y)
    _call(dev, _lib.abs_residual_norm_backward, dna, ld_dn, dya, ld_dy, ya, ld_y, ha, ld_h, ga, ld_g, kind, post, pre, scale, eps, code, T, D,
          dxa, ld_dx, dha, ld_dh, dga, ld_dg, dpre, dpost, bool(accumulate), ws.data_ptr(), n)
    return ResidualGrads(dx, dh, dgate, dw_pre, dw_post)


def ckpt8_quantize(x) -> Ckpt8:
    """An activation [tokens, width] (float32 / bfloat16) in 8 bits (``abs_ckpt8_quantize``)."""
    code, T, D, dev = _first(x, "x")
    xa, ld = _matrix(x, "x", x.dtype, T, D, dev)
    W = (D + 31) // 32 * 32
    q = _empty((T, W), dtype=torch.int8, device=x.device)
    e = _empty((T, W // 32), dtype=torch.uint8, device=x.device)
    _call(dev, _lib.abs_ckpt8_quantize, xa, ld, code, T, D, q.data_ptr(), e.data_ptr())
    return Ckpt8(q, e, D)


def _ckpt(c):
    """(address of q, address of e, tokens, device index)"""
    q, e = c.q, c.e
    W = (c.width + 31) // 32 * 32
    dev = q.get_device()
    if q.dtype is not torch.int8 or e.dtype is not torch.uint8 or dev < 0 or e.get_device() != dev:
        raise TypeError("a Ckpt8 holds an int8 and a uint8 tensor on one CUDA device")
    if q.dim() != 2 or q.shape[1] != W or e.shape != (q.shape[0], W // 32) or not q.is_contiguous() or not e.is_contiguous():
        raise ValueError("a Ckpt8 holds q [tokens, width rounded up to 32] and e [tokens, same / 32], contiguous")
    return q.data_ptr(), e.data_ptr(), q.shape[0], dev


def ckpt8_dequantize(c: Ckpt8, dtype=torch.bfloat16, out=None):
    """The values that a Ckpt8 stands for, [tokens, width]."""
    qa, ea, T, dev = _ckpt(c)
    code = _DTYPE.get(dtype)
    if code is None:
        raise TypeError("dtype must be float32 or bfloat16")
    if out is None:
        out = _empty((T, c.width), dtype=dtype, device=c.q.device)
    oa, ld = _matrix(out, "out", dtype, T, c.width, dev)
    _call(dev, _lib.abs_ckpt8_dequantize, qa, ea, T, c.width, oa, ld, code)
    return out


def ckpt8_wgrad(c: Ckpt8, dy, out=None, accumulate: bool = False):
    """x^T dy of the activation x that `c` stands for: the gradient of a weight stored [in, out] (``abs_ckpt8_wgrad``).

    dy bfloat16 [tokens, out].  out float32 [width, out], for instance a view of a flat gradient; accumulate adds to it."""
    qa, ea, T, dev = _ckpt(c)
    if not isinstance(dy, _Tensor) or dy.dim() != 2:
        raise TypeError("dy must be a CUDA tensor of two dimensions")
    N = dy.shape[1]
    ya, ld = _matrix(dy, "dy", _BF16, T, N, dev)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out to add to")
        out = _empty((c.width, N), dtype=_F32, device=dy.device)
    oa, ld_o = _matrix(out, "out", _F32, c.width, N, dev)
    n = _lib.abs_ckpt8_wgrad_workspace(T, c.width, N, ya, ld)
    ws = _workspace(n, dy) if n else None
    _call(dev, _lib.abs_ckpt8_wgrad, qa, ea, ya, ld, T, c.width, N, oa, ld_o, bool(accumulate), ws.data_ptr() if n else None, n)
    return out


def check(device=None):
    """Blocks until the current stream has finished; raises if a kernel of this module gave up a bounded wait."""
    index = torch.cuda.current_device() if device is None else torch.device(device).index
    _call(torch.cuda.current_device() if index is None else index, _lib.abs_llm_check)
