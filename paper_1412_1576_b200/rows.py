"""Operators on rows of logits or probabilities, for callers that hold torch tensors.

What a neural model of the sampler's words needs beside the sampler: a teacher's lists (``top_logits``), a drafter's loss
against them (``distill_loss``, ``distill_loss_and_grad``), and the test that accepts the drafter's tokens (``verify_drafts``).
Argument checks and outputs only: the work is done by the entry points of the same purpose in ``include/lda_b200.h``, queued on
the current stream of the tensors' device.  There is no fallback: tensors that are not on a GPU are refused, and so is tracing
(``torch.compile`` leaves the calls outside of its graphs).
"""

from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version
from torch.fx.experimental.proxy_tensor import get_proxy_mode

from . import binding as _b

# (whether torch.jit, a dispatch mode or a tracer before dispatch is at work: a quarter of a microsecond together)
_jit_tracing, _modes = torch._C._is_tracing, torch._C._len_torch_dispatch_stack
_before_dispatch = torch._ops.mode_stack_state_for_pre_dispatch().get
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
_DTYPES = {torch.float32: _b.LDA_F32, torch.float16: _b.LDA_F16, torch.bfloat16: _b.LDA_BF16}


def _rows(x, name):
    """Checks a matrix whose rows are consecutive in memory; returns (dtype code, rows, V, row stride)."""
    code = _DTYPES.get(x.dtype)
    shape = x.shape
    if code is None or len(shape) != 2 or shape[1] < 1:
        if code is None:
            raise TypeError(f"{name}: float32, float16 or bfloat16 is needed, not {x.dtype}")
        raise ValueError(f"{name}: a matrix with at least one column is needed, not {tuple(shape)}")
    return code, shape[0], shape[1], _row_stride(x, shape, name)


def _row_stride(x, shape, name):
    between, step = x.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError(f"{name}: the words of a row must be consecutive in memory")
    return between if shape[0] > 1 else shape[1]


def _vector(x, name, dtype, n, device):
    """Checks a contiguous vector; returns its address."""
    if x.dtype is dtype and x.shape == (n,) and x.device == device and x.is_contiguous():
        return x.data_ptr()
    if x.dtype is not dtype:
        raise TypeError(f"{name}: {dtype} is needed, not {x.dtype}")
    if x.shape != (n,):
        raise ValueError(f"{name}: {n} values are needed, not {tuple(x.shape)}")
    _here(x, name, device)
    raise ValueError(f"{name}: must be contiguous")


def _optional(x, name, n, device):
    """The same of a float32 vector that may be None, as NULL."""
    if x is None:
        return None
    address = _vector(x, name, torch.float32, n, device)
    if not address and n:  # (torch's functional wrappers; the library would take it for `not given`)
        raise ValueError(f"{name}: a tensor without memory of its own")
    return address


def _here(x, name, device):
    if x.device != device:
        raise ValueError(f"{name}: on {x.device}, the rows are on {device}")


def _cuda(x, name):
    # (a tracer sees the outputs' allocation, not the library's call that fills them)
    if _jit_tracing() or (_modes() or _before_dispatch(0)) and get_proxy_mode() is not None:
        raise RuntimeError(f"{name}: operators on rows cannot be traced")
    if not x.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed (there is no CPU fallback)")
    return x.device


def _call(name, device, *args):
    """One library call on the device's current stream."""
    fn = getattr(_b.load_library(), name)
    index = device.index
    # (two microseconds less than torch.cuda.current_stream(device).cuda_stream, which is a fifth of a small call)
    stream = _raw_stream(index)
    if _current_device() == index:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream)
    if rc:
        raise _b.LdaError(rc, name)


def top_logits(logits, top: int, temperature: float = 1.0):
    """The `top` largest logits of every row: (ids int32 [rows, top], values [rows, top], lse float32 [rows]).

    Values descend, equal ones by the lower word.  Words at minus infinity are masked: never listed, and places that no word
    is left for have id -1 and value minus infinity.  ``lse`` is log sum exp(x / temperature) of the whole row.  None of the
    three is followed by autograd.
    """
    device = _cuda(logits, "logits")
    code, rows, V, stride = _rows(logits, "logits")
    if not 1 <= top <= _b.LDA_TOP_MAX:
        raise ValueError(f"top: 1 to {_b.LDA_TOP_MAX}, not {top}")
    values = logits.new_empty((rows, top))
    ids = logits.new_empty((rows, top), dtype=torch.int32)
    lse = logits.new_empty(rows, dtype=torch.float32)
    _call("lda_top_logits", device, logits.data_ptr(), code, rows, V, stride, top, temperature, ids.data_ptr(),
          values.data_ptr(), lse.data_ptr())
    return ids, values, lse


def _list(ids, values, lse, rows, device):
    """Checks a teacher's lists; returns the library's arguments for them."""
    code = _DTYPES.get(values.dtype)
    shape = ids.shape
    if ids.dtype is not torch.int32:
        raise TypeError(f"ids: int32 is needed, not {ids.dtype}")
    if code is None:
        raise TypeError(f"values: float32, float16 or bfloat16 is needed, not {values.dtype}")
    if len(shape) != 2 or shape[0] != rows or shape != values.shape:
        raise ValueError(f"ids and values: one list per row, {rows} of them, not {tuple(shape)} and {tuple(values.shape)}")
    top = shape[1]
    if not 1 <= top <= _b.LDA_TOP_MAX:
        raise ValueError(f"ids: lists of 1 to {_b.LDA_TOP_MAX} words, not {top}")
    between = ids.stride()
    if between != values.stride() or between[1] != 1:
        if top > 1 and (between[1] != 1 or values.stride(1) != 1):
            raise ValueError("ids and values: the places of a list must be consecutive in memory")
        if rows > 1 and between[0] != values.stride(0):
            raise ValueError("ids and values: their rows must lie equally far apart")
    if ids.device != device or values.device != device:
        _here(ids, "ids", device)
        _here(values, "values", device)
    return ids.data_ptr(), values.data_ptr(), code, top, between[0] if rows > 1 else top, _optional(lse, "lse", rows, device)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, values, lse, temperature):
        ctx.save_for_backward(logits, ids, values, lse)
        ctx.temperature = temperature
        return _loss(logits, ids, values, lse, temperature)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, ids, values, lse = ctx.saved_tensors
        grad = _grad(logits.detach(), ids, values, lse, ctx.temperature, dloss.contiguous(), None, None)
        return grad, None, None, None, None


def _loss(logits, ids, values, lse, temperature):
    device = _cuda(logits, "logits")
    code, rows, V, stride = _rows(logits, "logits")
    lists = _list(ids, values, lse, rows, device)
    loss = logits.new_empty(rows, dtype=torch.float32)
    _call("lda_distill_loss", device, logits.data_ptr(), code, rows, V, stride, *lists, temperature, loss.data_ptr())
    return loss


def _grad(logits, ids, values, lse, temperature, weights, loss, grad):
    """Queues the gradient; grad None: into a new tensor.  Returns it."""
    device = _cuda(logits, "logits")
    code, rows, V, stride = _rows(logits, "logits")
    lists = _list(ids, values, lse, rows, device)
    given = grad is not None
    if not given:
        grad, grad_stride = torch.empty_like(logits, memory_format=torch.contiguous_format), V
    else:
        if grad.dtype != logits.dtype or grad.shape != logits.shape:
            raise ValueError("grad: must have the logits' type and shape")
        if grad.requires_grad:
            raise ValueError("grad: a tensor that autograd follows cannot be written to (detach it)")
        grad_stride = _rows(grad, "grad")[3]
        _here(grad, "grad", device)
    w = _optional(weights, "weights", rows, device)
    _call("lda_distill_grad", device, logits.data_ptr(), code, rows, V, stride, *lists, temperature, w,
          None if loss is None else loss.data_ptr(), grad.data_ptr(), grad_stride)
    if given:
        increment_version(grad)  # (a graph that has saved what was there finds out)
    return grad


def distill_loss(logits, ids, values, lse=None, temperature: float = 1.0):
    """Loss of every row of a student's logits against a teacher's top logits: temperature^2 KL(teacher || student), float32 [rows].

    ids, values: the teacher's lists, as ``top_logits`` gives them; an id outside the vocabulary is padding.  lse None: the
    teacher's distribution is the softmax over the list.  With the teacher's log-sum-exp (taken at the same temperature) it
    is that of its whole row, and all words outside the list make one bucket more, unless the student has them all masked, with
    minus infinity (a large negative number is a logit like any other).  Differentiable once, in reverse mode, with respect to
    ``logits`` alone (the teacher is a constant); a row that gets the gradient 0 passes 0 on, whatever it holds.  A backward pass that is
    captured into a CUDA graph needs, as always with torch, that no eager graph of the same leaves is alive;
    ``distill_loss_and_grad`` does not.
    """
    # (a tangent is lost outside of autograd's function, which has no forward mode and says so)
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(logits).tangent is not None:
        raise NotImplementedError("distill_loss: forward-mode differentiation is not offered")
    if torch.is_grad_enabled() and logits.requires_grad:
        return _Distill.apply(logits, ids, values, lse, temperature)
    return _loss(logits, ids, values, lse, temperature)


def distill_loss_and_grad(logits, ids, values, lse=None, temperature: float = 1.0, weights=None, grad=None):
    """``distill_loss`` and the gradient of sum(weights * loss) with respect to the logits, in one pass over them.

    weights: float32 [rows], None for 1 each; a row of weight 0 has gradient 0.  grad: where the gradient goes, None for a
    new tensor; the logits themselves are allowed and are overwritten then.  Returns (loss, grad).  No autograd graph is made.
    """
    if logits.requires_grad:
        logits = logits.detach()
    loss = logits.new_empty(logits.shape[:1], dtype=torch.float32)
    return loss, _grad(logits, ids, values, lse, temperature, weights, loss, grad)


def verify_drafts(draft_offsets, drafts, target, draft_probs, accept_u, draw_u, tokens=None, accepted=None):
    """Which drafted tokens stand against the target's probabilities, and the token that follows them.

    draft_offsets: int64 [n + 1], sequence b has the drafts [offsets[b], offsets[b + 1]) of ``drafts`` (int32); target: one
    row per draft and one more behind each sequence's last, [drafts + n, V]; draft_probs: the drafter's rows [drafts, V] in
    the same type, or None where it put its whole mass on its draft; accept_u [drafts] and draw_u [n]: float32 uniforms.
    Returns (tokens int32 [drafts + n], accepted int32 [n]): at the places of a sequence's target rows its accepted drafts,
    the token drawn behind them, then -1.  Both may be given, apart from the inputs' memory; places of no sequence keep what they
    hold (-1 in new ones).
    """
    device = _cuda(target, "target")
    code, rows, V, stride = _rows(target, "target")
    shape = draft_offsets.shape
    if len(shape) != 1 or shape[0] < 1:
        raise ValueError("draft_offsets: one more than there are sequences is needed")
    n_seqs, n_drafts = shape[0] - 1, drafts.numel()
    if rows != n_drafts + n_seqs:
        raise ValueError(f"target: {n_drafts} drafts of {n_seqs} sequences need {n_drafts + n_seqs} rows, not {rows}")
    offsets_ptr = _vector(draft_offsets, "draft_offsets", torch.int64, n_seqs + 1, device)
    drafts_ptr = _vector(drafts, "drafts", torch.int32, n_drafts, device)
    probs_ptr, probs_stride = None, 0
    if draft_probs is not None:
        shape = draft_probs.shape
        if draft_probs.dtype is not target.dtype or shape != (n_drafts, V):
            raise ValueError(f"draft_probs: [{n_drafts}, {V}] of {target.dtype} is needed")
        probs_stride = _row_stride(draft_probs, shape, "draft_probs")
        _here(draft_probs, "draft_probs", device)
        # (without drafts there is nothing to point at; sequences then have one row each, of the target)
        probs_ptr = draft_probs.data_ptr() if n_drafts else None
        if probs_ptr == 0:
            raise ValueError("draft_probs: a tensor without memory of its own")
    accept_ptr = _vector(accept_u, "accept_u", torch.float32, n_drafts, device)
    draw_ptr = _vector(draw_u, "draw_u", torch.float32, n_seqs, device)
    given = tokens is not None or accepted is not None
    if tokens is None:
        tokens = torch.full((rows,), -1, dtype=torch.int32, device=device)
    if accepted is None:
        accepted = torch.empty(n_seqs, dtype=torch.int32, device=device)
    tokens_ptr = _vector(tokens, "tokens", torch.int32, rows, device)
    accepted_ptr = _vector(accepted, "accepted", torch.int32, n_seqs, device)
    _call("lda_verify_drafts", device, offsets_ptr, n_seqs, drafts_ptr, n_drafts, target.data_ptr(), stride, probs_ptr,
          probs_stride, code, V, accept_ptr, draw_ptr, tokens_ptr, accepted_ptr)
    if given:
        increment_version((tokens, accepted))  # (a graph that has saved them, as an embedding's indices, finds out)
    return tokens, accepted
