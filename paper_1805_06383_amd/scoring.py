"""Operators of a learned scorer of label sequences, on the GPU.

A composed transducer is a set of hypotheses; a scorer embeds their labels,
mixes them over the sequence, gives each label a log-probability (an arc's
weight, or a hypothesis' score), and is trained from which of two hypotheses
was better.  These are its operators, bound to the kernels of libfstc.so
(declared in include/fstc.h):

    embed                   rows of a table, scaled; gradient of the table
    linear_attention        decayed linear attention over whole sequences, gradients
    linear_attention_step   the same for one label of many hypotheses, which
                            continue (fork) their parents' states
    label_logprob           log softmax at given labels; gradient of the logits
    preference_loss         loss of pairs of sequences; gradient of the logits

Tensors are float32, bfloat16 or float16 on one GPU; labels are int32 (the
bits of the u32 labels of a transducer) or int64, and a label outside its
alphabet, such as -1, marks padding.  Work is enqueued on the current stream of
the tensors' device.  Arguments that an operator does not take raise
``FstcError`` before anything is enqueued, and so do derivatives that it does not have
(second ones, those of forward mode, those in a decay or a reference).
"""
from __future__ import annotations

import ctypes
import struct

import torch
from torch.autograd import forward_ad

from .fstc import (FSTC_ERR_INVALID_ARG, FSTC_ERR_RANGE, FstcError, FstcLinattnArgs, _check,
                   load_library)

__all__ = ["embed", "label_logprob", "linear_attention", "linear_attention_step",
           "preference_loss"]

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_LABEL_BYTES = {torch.int32: 4, torch.int64: 8}
_I64x3 = ctypes.c_int64 * 3
_PROXY = torch._C._TorchDispatchModeKey.PROXY  # (of a trace by torch.fx)


def _refuse(msg: str):
    raise FstcError(FSTC_ERR_INVALID_ARG, msg)


def _values(name: str, x, ndim: int, like: torch.Tensor | None = None) -> int:
    """Checks a value tensor (its last dimension consecutive); its type's code."""
    code = _DTYPE.get(x.dtype)
    if code is None or x.ndim != ndim or not x.is_cuda:
        _refuse(f"{name}: a {ndim}-dimensional float32, bfloat16 or float16 tensor on the GPU, "
                f"not {x.dtype} {tuple(x.shape)} on {x.device}")
    if like is not None and (x.dtype != like.dtype or x.device != like.device):
        _refuse(f"{name}: {x.dtype} on {x.device}, but {like.dtype} on {like.device} before it")
    return code


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x itself where its last dimension is consecutive, else a contiguous copy."""
    return x if x.stride(-1) == 1 or x.shape[-1] <= 1 else x.contiguous()


def _labels(name: str, x, like: torch.Tensor) -> tuple[torch.Tensor, int]:
    size = _LABEL_BYTES.get(x.dtype)
    if size is None or x.device != like.device:
        _refuse(f"{name}: int32 or int64 on {like.device}, not {x.dtype} on {x.device}")
    return x.contiguous(), size


def _f32(name: str, x, shape, like: torch.Tensor) -> torch.Tensor:
    if x.dtype != torch.float32 or x.shape != shape or x.device != like.device:
        _refuse(f"{name}: float32 {tuple(shape)} on {like.device}, "
                f"not {x.dtype} {tuple(x.shape)} on {x.device}")
    return x.contiguous()


def _call(name: str, device: torch.device, *args):
    """The entry point `name` with the device's current stream as the last
    argument, the device made current."""
    f = getattr(load_library(), name)
    index = device.index
    if torch._C._cuda_getDevice() == index:
        rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(device):
            rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if rc:
        _check(rc)


def _refuse_lost(*tensors):
    """Refuses what would lose an operator without a word: a tangent of forward-mode
    differentiation, and a trace, which records allocations and no kernel."""
    if forward_ad._current_level >= 0:
        for x in tensors:
            if x is not None and forward_ad.unpack_dual(x).tangent is not None:
                _refuse("forward-mode derivatives are not available")
    if torch._C._is_tracing() or torch._C._get_dispatch_mode(_PROXY) is not None:
        _refuse("the operators cannot be traced")


def _first_derivatives_only(*grads):
    # (a backward pass runs with gradients enabled where it is to be differentiated itself)
    if torch.is_grad_enabled():
        _refuse("second derivatives are not available")
    _refuse_lost(*grads)


def _workspace(nbytes: int, like: torch.Tensor):
    """A buffer of that size (None: none needed) and its address."""
    if nbytes == 0:
        return None, None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    return ws, ws.data_ptr()


# ---------------------------------------------------------------------------
def _embed_forward(table, labels, size, scale):
    rows, dim = table.shape
    out = table.new_empty((*labels.shape, dim))
    _call("fstc_embed", table.device, table.data_ptr(), _DTYPE[table.dtype], rows, dim,
          table.stride(0), labels.data_ptr(), size, labels.numel(), scale, out.data_ptr())
    return out


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, labels, size, scale):
        ctx.save_for_backward(labels)
        ctx.shape, ctx.size, ctx.scale = table.shape, size, scale
        return _embed_forward(table, labels, size, scale)

    @staticmethod
    def backward(ctx, grad):
        _first_derivatives_only(grad)
        labels = ctx.saved_tensors[0].contiguous()
        (rows, dim), n = ctx.shape, labels.numel()
        grad = _rows(grad.reshape(n, dim))
        if n and grad.stride(0) < dim:  # a broadcast gradient
            grad = grad.contiguous()
        out = grad.new_empty((rows, dim))
        size = load_library().fstc_embed_grad_workspace(n, dim)
        ws, at = _workspace(size, grad)
        _call("fstc_embed_grad", grad.device, grad.data_ptr(), _DTYPE[grad.dtype],
              max(grad.stride(0), dim), labels.data_ptr(), ctx.size, n, rows, dim, ctx.scale,
              out.data_ptr(), at, size)
        return out, None, None, None


def embed(table: torch.Tensor, labels: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """scale * table[labels]: [*labels.shape, dim] of the table's type; zero
    rows for labels outside [0, len(table)).  Differentiable in the table; the
    gradient's sums have a fixed order (equal inputs give equal bits)."""
    _refuse_lost(table)
    _values("table", table, 2)
    table = _rows(table)
    if table.shape[0] > 1 and table.stride(0) < table.shape[1]:
        table = table.contiguous()
    elif table.shape[0] <= 1 and table.stride(0) < table.shape[1]:
        table = table.as_strided(table.shape, (table.shape[1], 1))
    labels, size = _labels("labels", labels, table)
    if table.requires_grad and torch.is_grad_enabled():
        if max(table.shape[0], labels.numel()) >= 1 << 28:
            raise FstcError(FSTC_ERR_RANGE, "rows and labels must be below 2^28 for the gradient")
        return _Embed.apply(table, labels, size, float(scale))
    return _embed_forward(table, labels, size, float(scale))


# ---------------------------------------------------------------------------
_ARGS = struct.Struct("=5IifI5Q9qQ")  # FstcLinattnArgs, built at once


def _linattn_args(shape, dv, dtype, log_decay, scale, init, lengths, q, k, v, qs, ks, vs):
    """The call's FstcLinattnArgs; qs, ks, vs: strides of the batch, the position, the head."""
    B, T, H, dk = shape
    return FstcLinattnArgs.from_buffer_copy(_ARGS.pack(
        B, T, H, dk, dv, _DTYPE[dtype], scale, 0, log_decay.data_ptr(),
        lengths.data_ptr() if lengths is not None else 0, q.data_ptr(), k.data_ptr(), v.data_ptr(),
        *qs, *ks, *vs, init.data_ptr() if init is not None else 0))


def _sequence_args(q, k, v, log_decay, scale, init, lengths):
    return _linattn_args(q.shape, v.shape[3], q.dtype, log_decay, scale, init, lengths, q, k, v,
                         q.stride()[:3], k.stride()[:3], v.stride()[:3])


def _linattn_forward(q, k, v, log_decay, init, lengths, scale):
    B, T, H, dk = q.shape
    dv = v.shape[3]
    device = q.device
    out = q.new_empty((B, T, H, dv))
    final = torch.empty((B, H, dk, dv), dtype=torch.float32, device=device)
    args = _sequence_args(q, k, v, log_decay, scale, init, lengths)
    size = load_library().fstc_linattn_workspace(args, 0)
    ws, at = _workspace(size, q)
    _call("fstc_linattn", device, args, out.data_ptr(), final.data_ptr(), at, size)
    return out, final


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, init, lengths, scale):
        ctx.save_for_backward(q, k, v, log_decay, init, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return _linattn_forward(q, k, v, log_decay, init, lengths, scale)

    @staticmethod
    def backward(ctx, dout, dfinal):
        _first_derivatives_only(dout, dfinal)
        # (hooks may give back what was saved laid out otherwise)
        q, k, v, *rest = ctx.saved_tensors
        q, k, v = _rows(q), _rows(k), _rows(v)
        log_decay, init, lengths = (x if x is None else x.contiguous() for x in rest)
        if dout is None:
            dout = torch.zeros((), dtype=q.dtype, device=q.device).expand(*q.shape[:3], v.shape[3])
        dout = _rows(dout)
        if dfinal is not None:
            dfinal = dfinal.contiguous()
        dq, dk, dv = (x.new_empty(x.shape) for x in (q, k, v))
        dinit = None
        if init is not None and ctx.needs_input_grad[4]:
            dinit = init.new_empty(init.shape)
        args = _sequence_args(q, k, v, log_decay, ctx.scale, init, lengths)
        size = load_library().fstc_linattn_workspace(args, 1)
        ws, at = _workspace(size, q)
        _call("fstc_linattn_grad", q.device, args, dout.data_ptr(), _I64x3(*dout.stride()[:3]),
              dfinal.data_ptr() if dfinal is not None else None, dq.data_ptr(), dk.data_ptr(),
              dv.data_ptr(), dinit.data_ptr() if dinit is not None else None, at, size)
        return dq, dk, dv, None, dinit, None, None


def _attention_inputs(q, k, v, log_decay, ndim):
    """q, k, v with consecutive last dimensions, checked against each other;
    the heads' decays."""
    _values("q", q, ndim)
    shape, vs, dtype, device = q.shape, v.shape, q.dtype, q.device
    if k.dtype != dtype or k.device != device or v.dtype != dtype or v.device != device:
        _values("k", k, ndim, q)
        _values("v", v, ndim, q)
    if k.shape != shape or len(vs) != ndim or vs[:-1] != shape[:-1]:
        _refuse(f"q, k and v have shapes {tuple(q.shape)}, {tuple(k.shape)} and {tuple(v.shape)}: "
                "all but the last of v have to agree")
    if log_decay.requires_grad and torch.is_grad_enabled():
        _refuse("log_decay is a fixed schedule: it has no gradient (pass it detached)")
    log_decay = _f32("log_decay", log_decay, shape[-2:-1], q)
    return _rows(q), _rows(k), _rows(v), log_decay


def linear_attention(q, k, v, log_decay, scale: float = 1.0, initial_state=None, lengths=None):
    """Linear attention with a decay for each head over whole sequences:
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T, out_t = scale * S_t^T q_t.

    q, k [batch, length, heads, dim_k], v [batch, length, heads, dim_v] (any
    strides; dims at most 256), log_decay float32 [heads] (<= 0, a fixed
    schedule without gradient), initial_state float32 [batch, heads, dim_k, dim_v]
    (None: zero), lengths int32 [batch] (None: all positions).  Returns (out,
    final_state): out has q's type, zero at and beyond a row's length;
    final_state is float32, the state after the row's last position, from which
    linear_attention_step goes on.  Differentiable in q, k, v and initial_state.
    Nothing beyond a length is read; within it a value that is not finite may reach outputs
    up to 63 positions before it, as well as all after it, and an infinity may end as NaN."""
    _refuse_lost(q, k, v, log_decay, initial_state)
    q, k, v, log_decay = _attention_inputs(q, k, v, log_decay, 4)
    B, T, H, dk = q.shape
    if initial_state is not None:
        initial_state = _f32("initial_state", initial_state, (B, H, dk, v.shape[3]), q)
    if lengths is not None:
        if lengths.dtype != torch.int32 or tuple(lengths.shape) != (B,) or lengths.device != q.device:
            _refuse(f"lengths: int32 ({B},) on {q.device}, not {lengths.dtype} "
                    f"{tuple(lengths.shape)} on {lengths.device}")
        lengths = lengths.contiguous()
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or (
            initial_state is not None and initial_state.requires_grad)):
        return _LinearAttention.apply(q, k, v, log_decay, initial_state, lengths, float(scale))
    return _linattn_forward(q, k, v, log_decay, initial_state, lengths, float(scale))


def linear_attention_step(q, k, v, log_decay, state, scale: float = 1.0, parents=None,
                          out_state=None):
    """One label of linear_attention for each of a batch of hypotheses.

    q, k [batch, heads, dim_k], v [batch, heads, dim_v]; state float32
    [rows, heads, dim_k, dim_v].  Hypothesis b goes on from state[parents[b]]
    (parents int32 [batch]; one outside [0, rows), such as -1, starts from a zero
    state), or from state[b] without parents (rows = batch).  Returns (out
    [batch, heads, dim_v], new states [batch, heads, dim_k, dim_v]).  out_state
    receives the new states, as an in-place operation does; it may be `state` itself
    when there are no parents.  Not differentiable (train with linear_attention)."""
    _refuse_lost(q, k, v, log_decay, state, out_state)
    q, k, v, log_decay = _attention_inputs(q, k, v, log_decay, 3)
    B, H, dk = q.shape
    dv = v.shape[2]
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad
                                    or state.requires_grad):
        _refuse("a step has no gradient: call it under torch.no_grad(), or linear_attention")
    rows = state.shape[0] if state.ndim else 0
    state = _f32("state", state, (rows, H, dk, dv), q)
    if parents is not None:
        if parents.dtype != torch.int32 or tuple(parents.shape) != (B,) or parents.device != q.device:
            _refuse(f"parents: int32 ({B},) on {q.device}, not {parents.dtype} "
                    f"{tuple(parents.shape)} on {parents.device}")
        parents = parents.contiguous()
    versioned = False
    if out_state is None:
        out_state = state.new_empty((B, H, dk, dv))
    else:
        if not out_state.is_contiguous():
            _refuse("out_state has to be contiguous")
        _f32("out_state", out_state, (B, H, dk, dv), q)
        if out_state.requires_grad and torch.is_grad_enabled():
            _refuse("out_state wants a gradient, which a step does not have: call it under torch.no_grad()")
        versioned = not out_state.is_inference()
    out = q.new_empty((B, H, dv))
    (qb, qh, _), (kb, kh, _), (vb, vh, _) = q.stride(), k.stride(), v.stride()
    args = _linattn_args((B, 1, H, dk), dv, q.dtype, log_decay, scale, state, None, q, k, v,
                         (qb, 0, qh), (kb, 0, kh), (vb, 0, vh))
    _call("fstc_linattn_step", q.device, args, parents.data_ptr() if parents is not None else None,
          rows, out_state.data_ptr(), out.data_ptr())
    if versioned:  # (a backward pass that has kept it must not use it as it is now)
        torch.autograd.graph.increment_version(out_state)
    return out, out_state


# ---------------------------------------------------------------------------
def _logit_rows(logits):
    """logits, or a copy of them, as evenly spaced rows: (tensor, rows, vocab, row stride)."""
    vocab = logits.shape[-1] if logits.ndim else 0
    if vocab == 0:
        _refuse("logits: at least one logit a row")
    if logits.is_contiguous():
        return logits, logits.numel() // vocab, vocab, vocab
    x = _rows(logits.reshape(-1, vocab))
    if x.shape[0] > 1 and x.stride(0) < vocab:
        x = x.contiguous()
    return x, x.shape[0], vocab, max(x.stride(0), vocab)


def _saved_logits(ctx):
    """Logits that a forward pass kept, their rows, the labels and the rows' statistics (hooks
    may give them back laid out otherwise, so the rows are measured again)."""
    x, labels, kept = ctx.saved_tensors
    x, *rows = _logit_rows(x)
    return x, rows, labels.contiguous(), kept.contiguous()


def _logprob_forward(x, n, vocab, stride, labels, size, extra=0):
    """Log-probabilities, and a buffer that starts with what the gradient needs of each
    row (2 n values) and has `extra` more."""
    lp = torch.empty(labels.shape, dtype=torch.float32, device=x.device)
    kept = torch.empty(2 * n + extra, dtype=torch.float32, device=x.device)
    _call("fstc_label_logprob", x.device, x.data_ptr(), _DTYPE[x.dtype], n, vocab, stride,
          labels.data_ptr(), size, lp.data_ptr(), kept.data_ptr())
    return lp, kept


def _logprob_grad(shape, x, n, vocab, stride, labels, size, kept, weight, per, factor):
    """`weight`: an address; one value for each `per` rows."""
    d = x.new_empty(shape)
    _call("fstc_label_logprob_grad", x.device, x.data_ptr(), _DTYPE[x.dtype], n, vocab, stride,
          labels.data_ptr(), size, kept.data_ptr(), weight, per, factor, d.data_ptr())
    return d


class _LabelLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, size):
        x, *rows = _logit_rows(logits)
        lp, kept = _logprob_forward(x, *rows, labels, size)
        ctx.save_for_backward(x, labels, kept)
        ctx.size, ctx.shape = size, logits.shape
        return lp

    @staticmethod
    def backward(ctx, grad):
        _first_derivatives_only(grad)
        x, rows, labels, kept = _saved_logits(ctx)
        grad = grad.contiguous()
        return _logprob_grad(ctx.shape, x, *rows, labels, ctx.size, kept, grad.data_ptr(), 1,
                             None), None, None


def label_logprob(logits: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
    """log softmax(logits)[..., label]: float32 of labels' shape, logits
    [*labels.shape, vocab]; 0 (and no gradient) for a label outside the
    vocabulary.  Logits may be -inf (labels that a transducer does not allow);
    a row of nothing else has log-probability -inf and a zero gradient.
    Differentiable in the logits."""
    _refuse_lost(logits)
    if tuple(logits.shape[:-1]) != tuple(labels.shape):
        _refuse(f"logits {tuple(logits.shape)} for labels {tuple(labels.shape)}")
    _values("logits", logits, logits.ndim)
    labels, size = _labels("labels", labels, logits)
    if logits.requires_grad and torch.is_grad_enabled():
        return _LabelLogprob.apply(logits, labels, size)
    return _logprob_forward(*_logit_rows(logits), labels, size)[0]


def _preference_forward(x, n, vocab, stride, labels, size, ref, beta, smoothing):
    S, T = labels.shape
    device = x.device
    lp, kept = _logprob_forward(x, n, vocab, stride, labels, size, S)  # (rows, then sequences)
    loss = torch.empty((), dtype=torch.float32, device=device)
    margin = torch.empty(S // 2, dtype=torch.float32, device=device)
    seq = torch.empty(S, dtype=torch.float32, device=device)
    _call("fstc_preference_loss", device, lp.data_ptr(), S // 2, T, ref.data_ptr(), beta, smoothing,
          loss.data_ptr(), seq.data_ptr(), margin.data_ptr(), kept.data_ptr() + 8 * n)
    return kept, loss, seq, margin


class _Preference(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, size, ref, beta, smoothing):
        x, *rows = _logit_rows(logits)
        kept, loss, seq, margin = _preference_forward(x, *rows, labels, size, ref, beta, smoothing)
        ctx.save_for_backward(x, labels, kept)
        ctx.size, ctx.shape = size, logits.shape
        ctx.mark_non_differentiable(seq, margin)
        ctx.set_materialize_grads(False)  # (no zeros for what is for reading)
        return loss, seq, margin

    @staticmethod
    def backward(ctx, grad, _seq, _margin):
        _first_derivatives_only(grad)
        x, rows, labels, kept = _saved_logits(ctx)
        return _logprob_grad(ctx.shape, x, *rows, labels, ctx.size, kept,
                             kept.data_ptr() + 8 * rows[0], max(1, labels.shape[1]),
                             grad.data_ptr()), None, None, None, None, None


def preference_loss(logits: torch.Tensor, labels: torch.Tensor, ref_logprob: torch.Tensor,
                    beta: float = 0.1, label_smoothing: float = 0.0):
    """Preference loss of pairs of label sequences.

    logits [2 * pairs, length, vocab], labels [2 * pairs, length] (padding:
    labels outside the vocabulary): sequence p of the first half is preferred to
    sequence pairs + p.  ref_logprob float32 [2 * pairs]: the sequences'
    log-probabilities under a reference model (sums of label_logprob), which is fixed
    (no gradient).  Returns (loss, logprob [2 * pairs], margin [pairs]), float32: with
    L the sequences' log-probabilities, margin = beta * ((L - ref) of the preferred - (L - ref) of
    the other), loss = mean of -(1 - label_smoothing) log sigmoid(margin) -
    label_smoothing log sigmoid(-margin).  A sequence with a label of logit -inf has
    log-probability -inf and its pair an infinite margin; where infinities cancel
    (both sequences of a pair, or a sequence and its reference) the margin is NaN
    and the pair adds nothing to the loss or its gradient.  The loss is
    differentiable in the logits; logprob and margin are for reading."""
    _refuse_lost(logits, ref_logprob)
    if labels.ndim != 2 or labels.shape[0] % 2 or labels.shape[0] == 0:
        _refuse(f"labels: [2 * pairs, length], not {tuple(labels.shape)}")
    if tuple(logits.shape[:-1]) != tuple(labels.shape):
        _refuse(f"logits {tuple(logits.shape)} for labels {tuple(labels.shape)}")
    _values("logits", logits, 3)
    if not 0 <= ctypes.c_float(label_smoothing).value < 0.5:  # (as the call rounds it)
        _refuse(f"label_smoothing has to be in [0, 0.5), not {label_smoothing}")
    labels, size = _labels("labels", labels, logits)
    if ref_logprob.requires_grad and torch.is_grad_enabled():
        _refuse("ref_logprob is of a fixed model: it has no gradient (pass it detached)")
    ref = _f32("ref_logprob", ref_logprob, labels.shape[:1], logits)
    if logits.requires_grad and torch.is_grad_enabled():
        return _Preference.apply(logits, labels, size, ref, float(beta), float(label_smoothing))
    return _preference_forward(*_logit_rows(logits), labels, size, ref, float(beta),
                               float(label_smoothing))[1:]
