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


def check(device=None):
    """Blocks until the current stream has finished; raises if a kernel of this module gave up a bounded wait."""
    with torch.cuda.device(device):
        rc = _b.lib.abs_llm_check(torch.cuda.current_stream().cuda_stream)
    if rc:
        raise _b.AbsError(rc, _b.lib.abs_last_error(None).decode())
