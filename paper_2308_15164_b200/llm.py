"""Operators of a language model's training micro-batch (include/abs_llm.h) on CUDA tensors.

They are the parts of a forward and backward pass that lie around its matrix products; the flat gradient that comes out
goes to ``AbsSgd.accumulate``.  Every function checks its arguments, allocates its outputs and workspace from PyTorch's
allocator and enqueues on the current stream of the tensors' device; nothing synchronises.  Outputs that are given are
used as they are, and count as modified in place where autograd has saved them.  Refused arguments raise ``ValueError`` / ``TypeError`` here or ``binding.AbsError`` from the library.
Matrices may have any row stride; a row is contiguous.  Shapes are [tokens, width]: flatten leading dimensions with
``view``.
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as _b

try:
    from . import _llm as _t
except ImportError as e:
    raise ImportError(f"{e}: build the package with `python -m paper_2308_15164_b200.build`.  There is no fallback.") from e

_t.set_errors(_b.AbsError, torch.OutOfMemoryError)


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


class LayerNormGrads(NamedTuple):
    dx: torch.Tensor
    dw: torch.Tensor
    db: Optional[torch.Tensor]


class Linear(NamedTuple):
    y: torch.Tensor
    z: Optional[torch.Tensor]  # bfloat16: what the activation was taken of


class LinearGrads(NamedTuple):
    dw: torch.Tensor
    db: Optional[torch.Tensor]


class Recurrence(NamedTuple):
    y: torch.Tensor
    last: torch.Tensor       # [sequences, width] float32: the state behind each sequence


class RecurrenceGrads(NamedTuple):
    dx: torch.Tensor
    dg: torch.Tensor
    dh0: Optional[torch.Tensor]


ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}       # ABS_ACT_*
RECURRENCES = {"blend": 0, "add": 1}                             # ABS_RECURRENCE_*


def _choice(table, value, name):
    try:
        return table[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {', '.join(table)}") from None


def _is_bf16(dtype) -> bool:
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise TypeError("dtype must be float32 or bfloat16")
    return dtype is torch.bfloat16


def policy_loss(logits, labels, logp_old, advantage, weight, logp_ref=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, dlogits=None, need_grad: bool = True) -> PolicyLoss:
    """Clipped policy loss with a KL term to a reference model, with the gradient of the logits (``abs_policy_loss``).

    logits [tokens, vocab] float32 / bfloat16; labels int32; logp_old, advantage, weight, logp_ref float32 [tokens].
    weight is a token's share of the loss (1 / n for the mean over n tokens); tokens of weight 0 or with a label outside
    [0, vocab) are left out.  dlogits may be the logits themselves."""
    return PolicyLoss(*_t.policy_loss(logits, labels, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, dlogits, need_grad))


def preference_loss(logits, labels, offsets, logp_ref, beta: float = 0.1, smoothing: float = 0.0, scale: Optional[float] = None,
                    dlogits=None, need_grad: bool = True) -> PreferenceLoss:
    """Paired preference loss with the gradient of the logits (``abs_preference_loss``).

    logits [tokens, vocab]: the rows of the answers one after the other, answers 2 p and 2 p + 1 the preferred and the
    other one of pair p; offsets int32 [2 pairs + 1]: their first rows; labels int32 [tokens], outside [0, vocab) for rows
    that do not count; logp_ref float32 [2 pairs]: the reference model's log-probabilities.  scale: 1 / pairs if not given."""
    return PreferenceLoss(*_t.preference_loss(logits, labels, offsets, logp_ref, beta, smoothing, scale, dlogits, need_grad))


def residual_norm(x, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, y=None, n=None):
    """(y, n): y = scale x + G u, u = h / rms(h) w_post (h without w_post), n = y / rms(y) w_pre (``abs_residual_norm``).

    x, h [tokens, width] float32 / bfloat16; w_pre, w_post float32 [width].  gate: None (G = 1), float32 [width] (G = gate)
    or [tokens, width] of x's dtype (G = sigmoid(gate)).  y may be x, n may be h."""
    return _t.residual_norm(x, h, w_pre, w_post, gate, scale, eps, y, n)


def residual_norm_backward(dn, dy, y, h, w_pre, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, dx=None, dh=None,
                           dgate=None, dw_pre=None, dw_post=None, accumulate: bool = False) -> ResidualGrads:
    """Gradients of ``residual_norm`` from dn and dy (None: nothing else reads y) at the stored y and h.

    dw_pre, dw_post and a channel gate's dgate (float32 [width]) may be slices of a flat gradient; with accumulate the
    sums are added to what the given ones hold (those that are not given start at zero)."""
    return ResidualGrads(*_t.residual_norm_backward(dn, dy, y, h, w_pre, w_post, gate, scale, eps, dx, dh, dgate, dw_pre, dw_post, accumulate))


def ckpt8_quantize(x) -> Ckpt8:
    """An activation [tokens, width] (float32 / bfloat16) in 8 bits (``abs_ckpt8_quantize``)."""
    return Ckpt8(*_t.ckpt8_quantize(x), x.shape[1])


def ckpt8_dequantize(c: Ckpt8, dtype=torch.bfloat16, out=None):
    """The values that a Ckpt8 stands for, [tokens, width]."""
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise TypeError("dtype must be float32 or bfloat16")
    return _t.ckpt8_dequantize(*c, dtype is torch.bfloat16, out)


def ckpt8_wgrad(c: Ckpt8, dy, out=None, accumulate: bool = False):
    """x^T dy of the activation x that `c` stands for: the gradient of a weight stored [in, out] (``abs_ckpt8_wgrad``).

    dy bfloat16 [tokens, out].  out float32 [width, out], for instance a view of a flat gradient; accumulate adds to it."""
    return _t.ckpt8_wgrad(*c, dy, out, accumulate)


def embed(ids, table, scale: float = 1.0, dtype=torch.bfloat16, y=None):
    """y[t] = scale table[ids[t]], zeros where an id lies outside the table (``abs_embed``).

    ids int32 [tokens]; table float32 [vocab, width], for instance a view of the flat parameters; y [tokens, width] of `dtype`."""
    return _t.embed(ids, table, scale, _is_bf16(dtype), y)


def embed_backward(dy, ids, vocab: int, scale: float = 1.0, out=None, accumulate: bool = False):
    """The gradient of ``embed``'s table, float32 [vocab, width]: rows of no token are zero (``abs_embed_backward``).

    dy [tokens, width] float32 / bfloat16.  out: for instance a view of a flat gradient; with accumulate the rows of the tokens that
    occur are added to and no other is touched."""
    return _t.embed_backward(dy, ids, vocab, scale, out, accumulate)


def layer_norm(x, w, b=None, eps: float = 1e-5, n=None):
    """(x - mean) / sqrt(var + eps) w + b of every row (``abs_layer_norm``).  x [tokens, width] float32 / bfloat16; w, b float32 [width]; n
    may be x."""
    return _t.layer_norm(x, w, b, eps, n)


def layer_norm_backward(dn, x, w, dskip=None, bias: bool = True, eps: float = 1e-5, dx=None, dw=None, db=None,
                        accumulate: bool = False) -> LayerNormGrads:
    """Gradients of ``layer_norm`` from dn at the stored x; dskip (what reaches x around the norm) is added to dx
    (``abs_layer_norm_backward``).

    dw, db (float32 [width]; db with bias) may be slices of a flat gradient; with accumulate the sums are added to what the given
    ones hold (those that are not given start at zero).  dx may be dn, x or dskip."""
    return LayerNormGrads(*_t.layer_norm_backward(dn, x, w, dskip, bias, eps, dx, dw, db, accumulate))


def linear(x, w, b=None, act: str = "none", residual=None, keep: bool = False, dtype=torch.bfloat16, y=None, z=None) -> Linear:
    """z = x w + b, y = act(z) + residual (``abs_linear``).

    x bfloat16 [tokens, in], w bfloat16 [in, out], b float32 [out]; act "none", "relu", "gelu" or "silu"; y and residual
    [tokens, out] of `dtype` (y may be the residual).  keep: z is returned too, bfloat16, for the way back."""
    return Linear(*_t.linear(x, w, b, _choice(ACTIVATIONS, act, "act"), residual, keep, _is_bf16(dtype), y, z))


def linear_dgrad(dy, w, act: str = "none", z=None, residual=None, dtype=torch.bfloat16, dx=None):
    """dx = (dy w^T) act'(z) + residual: the gradient of a linear layer's input, and through the activation that made this input
    from z (``abs_linear_dgrad``).

    dy bfloat16 [tokens, out], w bfloat16 [in, out]; z bfloat16 [tokens, in], given exactly with an activation; dx and residual [tokens, in] of
    `dtype`; dx may be the residual or z."""
    return _t.linear_dgrad(dy, w, _choice(ACTIVATIONS, act, "act"), z, residual, _is_bf16(dtype), dx)


def linear_wgrad(x, dy, bias: bool = False, dw=None, db=None, accumulate: bool = False) -> LinearGrads:
    """dw = x^T dy and, with bias, db = the column sums of dy (``abs_linear_wgrad``).

    x [tokens, in], dy [tokens, out] bfloat16; dw [in, out], db [out] float32, for instance views of a flat gradient; accumulate adds to them
    (both have to be given then)."""
    return LinearGrads(*_t.linear_wgrad(x, dy, bias, dw, db, accumulate))


def activation_backward(dy, z, act: str, dz=None):
    """dz = dy act'(z), bfloat16, for an activation whose gradient no ``linear_dgrad`` forms (``abs_activation_backward``).  dy float32 /
    bfloat16, z bfloat16 [tokens, width]; dz may be z, or dy if that is bfloat16."""
    return _t.activation_backward(dy, z, _choice(ACTIVATIONS, act, "act"), dz)


def gated_recurrence(x, g, offsets=None, h0=None, kind: str = "blend", y=None, last=None) -> Recurrence:
    """h_t = a_t h_{t-1} + (1 - a_t) x_t ("blend") or + x_t ("add"), a = sigmoid(g), channel by channel over packed sequences
    (``abs_recurrence``).

    x, g [tokens, width] float32 / bfloat16: the rows of the sequences one after the other; offsets int32 [sequences + 1]: their first
    rows (None: one sequence); h0 float32 [sequences, width]: the states in front (None: zero).  y: h_t, zeros in rows of no sequence; y may
    be x or g."""
    return Recurrence(*_t.recurrence(x, g, offsets, h0, _choice(RECURRENCES, kind, "kind"), y, last))


def gated_recurrence_backward(dy, x, g, y, offsets=None, h0=None, dlast=None, kind: str = "blend", dx=None, dg=None,
                              dh0=None) -> RecurrenceGrads:
    """Gradients of ``gated_recurrence`` from dy and dlast (None: nothing reads last) at the stored x, g and y
    (``abs_recurrence_backward``).  dh0 is formed where h0 or dh0 is given.  dx and dg may be dy, x or g (not the same one)."""
    return RecurrenceGrads(*_t.recurrence_backward(dy, x, g, y, offsets, h0, dlast, _choice(RECURRENCES, kind, "kind"), dx, dg, dh0))


def gated_recurrence_step(x, g, h, kind: str = "blend", y=None, out=None) -> Recurrence:
    """One row for each sequence: the new state from h (float32 [sequences, width]), as y of x's dtype and as `last`, which is `out` (may be h)
    if that is given (``abs_recurrence_step``)."""
    return Recurrence(*_t.recurrence_step(x, g, h, _choice(RECURRENCES, kind, "kind"), y, out))


def check(device=None):
    """Blocks until the current stream has finished; raises if a kernel of this module gave up a bounded wait."""
    with torch.cuda.device(device):
        rc = _b.lib.abs_llm_check(torch.cuda.current_stream().cuda_stream)
    if rc:
        raise _b.AbsError(rc, _b.lib.abs_last_error(None).decode())
