"""The operators between a network and a circuit's leaf weights, as differentiable PyTorch functions: log probabilities of given
tokens (:func:`token_logprobs`) and gated recurrences over sequences in the library's semirings (:func:`gated_scan`, and
:func:`gated_step` for one step).  Marshalling only, on torch's current stream of the tensors' device: the kernels are those of
``klay_tokens_*`` and ``klay_scan_*`` (include/klay.h, which says what they compute and refuse).  Results and workspaces are torch
tensors, so calls may be captured into a graph and made on several streams at once.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as _b
from .binding import KLAY_LOG, KLAY_MAXLOG, KLAY_REAL

_DTYPES = {torch.float32: _b.KLAY_F32, torch.bfloat16: _b.KLAY_BF16, torch.float16: _b.KLAY_F16}
_MOST_TOKENS, _MOST_TOP, _MOST_CHANNELS = 1024, 64, 1 << 25
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: int) -> int:
    """The handle of the device's current stream (without a Stream object where this torch has a function for it)."""
    return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device)


def _check_tensor(t, name, dtypes=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(name + " must be a CUDA tensor")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError("%s must be %s" % (name, " or ".join(str(d).replace("torch.", "") for d in dtypes)))


def _refuse_tangents(who, *tensors):
    """The operators have no forward-mode derivative, and a kernel would drop a dual tensor's tangent without a word.  (Outside of a dual level,
    where this torch tells, there is none: a look at every tensor costs the host a microsecond a call.)"""
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError(who + " has no forward-mode derivative")


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- log probabilities of given tokens ----------------------------------------------------------------------------
class TokenLogprobs(NamedTuple):
    """What :func:`token_logprobs` returns; None for what was not asked."""
    logp: Optional[torch.Tensor]
    neg: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]
    top_tokens: Optional[torch.Tensor]


def _rows_of(t):
    """(t, its leading axes as klay_rows): t itself where at most two strides describe them, else a contiguous copy."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 2:
        return t, _b.klay_rows(shape[0] or 1, 0, strides[0])
    merged = []
    for n, s in zip(shape[:-1], strides[:-1]):
        if n == 1:
            continue
        if merged and merged[-1][1] == n * s:
            merged[-1] = (merged[-1][0] * n, s)
        else:
            merged.append((n, s))
    if len(merged) > 2:
        return _rows_of(t.contiguous())
    merged = [(1, 0)] * (2 - len(merged)) + merged
    return t, _b.klay_rows(merged[1][0] or 1, merged[0][1], merged[1][1])


def _token_args(logits, tokens, top):
    vocab = logits.shape[-1]
    if logits.stride(-1) != 1 and vocab != 1:
        logits = logits.contiguous()
    logits, logit_rows = _rows_of(logits)
    k = stride = pointer = 0
    token_rows = logit_rows
    if tokens is not None:
        tokens, token_rows = _rows_of(tokens)
        k, stride, pointer = tokens.shape[-1], tokens.stride(-1), tokens.data_ptr()
    args = _b.klay_tokens_args(_DTYPES[logits.dtype], logits.get_device(), vocab, k, top, 0, logits.numel() // vocab, logits.data_ptr(),
                               logit_rows, pointer, token_rows, stride)
    return args, (logits, tokens)          # the tensors that args points into


def _tokens_forward(logits, tokens, complement, entropy, top, keep):
    args, alive = _token_args(logits, tokens, top)
    lead, new, k = tuple(logits.shape[:-1]), logits.new_empty, args.num_tokens
    logp = neg = h = top_logp = top_tokens = stats = None
    if tokens is not None:
        logp = new(lead + (k,), dtype=torch.float32)
        if complement:
            neg = new(lead + (k,), dtype=torch.float32)
    if entropy:
        h = new(lead, dtype=torch.float32)
    if top:
        top_logp, top_tokens = new(lead + (top,), dtype=torch.float32), new(lead + (top,), dtype=torch.int64)
    if keep:
        stats = new((args.rows, 4), dtype=torch.float32)
    size = _b.klay_tokens_workspace_bytes(args)
    work = new((size,), dtype=torch.uint8) if size else None
    _b.klay_tokens_forward(args, _ptr(logp), _ptr(neg), _ptr(h), _ptr(stats), _ptr(top_logp), _ptr(top_tokens), _ptr(work), size,
                           _stream(args.device))
    return logp, neg, h, top_logp, top_tokens, stats, args, alive


# What a forward call's args point into (the tensors given, or the copies made of them) is what its function saves for the reverse call, so that
# hooks on saved tensors hold all of it, and nothing else keeps it alive.  The args are used again only where every tensor comes back in its place.
def _places(*tensors):
    """Where tensors are and how they lie: what args made for them stay good for."""
    return [None if t is None else (t.data_ptr(), t.stride()) for t in tensors]


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, complement, entropy, top):
        *out, stats, ctx.args, used = _tokens_forward(logits, tokens, complement, entropy, top, True)
        ctx.places = _places(*used)
        ctx.save_for_backward(*used, stats)
        ctx.set_materialize_grads(False)
        if top:
            ctx.mark_non_differentiable(*out[3:])
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dneg, dentropy, _top_logp, _top_tokens):
        logits, tokens, stats = ctx.saved_tensors
        dlogp, dneg, dentropy = (None if t is None else t.contiguous() for t in (dlogp, dneg, dentropy))
        args = ctx.args
        if ctx.places != _places(logits, tokens):                   # what was saved has been put elsewhere
            args, (logits, tokens) = _token_args(logits, tokens, 0)
        dlogits = logits.new_empty(logits.shape)
        _b.klay_tokens_backward(args, stats.data_ptr(), _ptr(dlogp), _ptr(dneg), _ptr(dentropy), dlogits.data_ptr(),
                                _stream(args.device))
        return dlogits, None, None, None, None


def token_logprobs(logits, tokens=None, *, complement=False, entropy=False, top=0) -> TokenLogprobs:
    """Log probabilities of ``tokens[..., K]`` (int64) under ``logits[..., V]`` (float32, bfloat16 or float16): the log weights
    of the literals "the network answers t".  Everything returned is float32.

    ``logp[..., K]``; with ``complement`` also ``neg[..., K]`` = log(1 - p), the weights of the negated literals (accurate where p
    rounds to 1); with ``entropy`` the rows' entropies ``[...]``; with ``top`` = n the n most likely tokens, equal ones by their
    index, as ``top_logp[..., n]`` and ``top_tokens[..., n]``.  A logit of -inf is a token that is not allowed, a negative token
    asks for nothing (weight 1 for both literals, log 0; no gradient), a token >= V gives NaN.  ``logp``, ``neg`` and ``entropy``
    are differentiable with respect to ``logits`` (backward only: tensors with tangents are refused); of the alternatives neither is
    (ask for them as ``tokens``).

    The elements of a row should be next to each other and the rows reachable with two strides (as those of ``logits[:, :-1]``
    are); anything else is copied first.  At most 1024 tokens and 64 alternatives a row.
    """
    _check_tensor(logits, "logits", _DTYPES)
    if logits.dim() < 1 or logits.shape[-1] < 1:
        raise ValueError("logits must be [..., V] with V >= 1")
    if tokens is not None:
        _check_tensor(tokens, "tokens", (torch.int64,))
        if tokens.device != logits.device:
            raise ValueError("tokens must be on the device of logits")
        if tokens.dim() != logits.dim() or tokens.shape[:-1] != logits.shape[:-1]:
            raise ValueError("tokens must be [..., K] with the leading axes of logits, %s" % (tuple(logits.shape[:-1]),))
        if tokens.shape[-1] > _MOST_TOKENS:
            raise ValueError("tokens must be at most %d a row" % _MOST_TOKENS)
    elif complement:
        raise ValueError("complement needs tokens")
    top = int(top)
    if logits.shape[-1] >= 1 << 31 or not 0 <= top <= min(_MOST_TOP, logits.shape[-1]):
        raise ValueError("top must be 0 .. min(V, %d), and V below 2^31" % _MOST_TOP)
    _refuse_tangents("token_logprobs", logits)
    if torch.is_grad_enabled() and logits.requires_grad:
        return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, complement, entropy, top))
    return TokenLogprobs(*_tokens_forward(logits, tokens, complement, entropy, top, False)[:5])


# ---- gated recurrence ---------------------------------------------------------------------------------------------
def _channels_last(t):
    """(t, its strides), or those of a copy where its channels lie apart (or its time steps further than the kernels reach; the stride of a
    single step, which contiguous() would leave as it is, is of no account)"""
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] != 1:
        t = t.contiguous()
        strides = t.stride()
    elif strides[-2] > _MOST_CHANNELS:
        if t.shape[-2] > 1:
            t = t.contiguous()
            strides = t.stride()
        else:
            strides = strides[:-2] + (0, 1)
    return t, strides


def _scan_args(gates, inputs, initial, semiring, offsets, row_info):
    (gates, gs), (inputs, xs) = _channels_last(gates), _channels_last(inputs)
    shape = gates.shape
    initial = None if initial is None else initial.contiguous()
    if offsets is None:
        batch, time, channels = shape
        args = _b.klay_scan_args(_DTYPES[gates.dtype], semiring, gates.get_device(), channels, batch, time, 0, gates.data_ptr(),
                                 inputs.data_ptr(), gs[0], gs[1], xs[0], xs[1], None, None, _ptr(initial))
    else:
        time, channels = shape
        args = _b.klay_scan_args(_DTYPES[gates.dtype], semiring, gates.get_device(), channels, 1, time, offsets.shape[0] - 1,
                                 gates.data_ptr(), inputs.data_ptr(), 0, gs[0], 0, xs[0], offsets.data_ptr(), row_info.data_ptr(),
                                 _ptr(initial))
    return args, (gates, inputs, initial)


def _scan_forward(gates, inputs, initial, semiring, offsets):
    new = gates.new_empty
    row_info = None if offsets is None else new((gates.shape[0],), dtype=torch.int32)
    args, alive = _scan_args(gates, inputs, initial, semiring, offsets, row_info)
    states = new(gates.shape)
    final = new((args.sequences if offsets is not None else args.batch, args.channels), dtype=torch.float32)
    size = _b.klay_scan_workspace_bytes(args)
    work = new((size,), dtype=torch.uint8) if size else None
    _b.klay_scan_forward(args, states.data_ptr(), final.data_ptr(), _ptr(work), size, _stream(args.device))
    return states, final, row_info, args, alive


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gates, inputs, initial, semiring, offsets):
        states, final, row_info, ctx.args, (gates, inputs, initial) = _scan_forward(gates, inputs, initial, semiring, offsets)
        ctx.semiring = semiring
        if semiring != KLAY_LOG:
            inputs = None                                           # not read by the reverse sweep
        ctx.places = _places(gates, inputs, initial, offsets, row_info)
        ctx.save_for_backward(gates, inputs, initial, offsets, row_info, states)
        ctx.set_materialize_grads(False)
        return states, final

    @staticmethod
    @once_differentiable
    def backward(ctx, dstates, dfinal):
        gates, inputs, initial, offsets, row_info, states = ctx.saved_tensors
        if dstates is None and dfinal is None:
            return None, None, None, None, None
        args = ctx.args
        if ctx.places != _places(gates, inputs, initial, offsets, row_info):       # what was saved has been put elsewhere
            args, (gates, inputs, initial) = _scan_args(gates, gates if inputs is None else inputs, initial, ctx.semiring, offsets, row_info)
        dstates, dfinal = (None if t is None else t.contiguous() for t in (dstates, dfinal))
        dgates, dinputs = (gates.new_empty(gates.shape) if need else None for need in ctx.needs_input_grad[:2])
        dinitial = initial.new_empty(initial.shape) if ctx.needs_input_grad[2] else None
        size = _b.klay_scan_workspace_bytes(args)
        work = gates.new_empty((size,), dtype=torch.uint8) if size else None
        _b.klay_scan_backward(args, states.data_ptr(), _ptr(dstates), _ptr(dfinal), _ptr(dgates), _ptr(dinputs), _ptr(dinitial),
                              _ptr(work), size, _stream(args.device))
        return dgates, dinputs, dinitial, None, None


def _check_recurrence(gates, inputs, semiring):
    _check_tensor(gates, "gates", _DTYPES)
    _check_tensor(inputs, "inputs", _DTYPES)
    if inputs.shape != gates.shape or inputs.dtype != gates.dtype or inputs.device != gates.device:
        raise ValueError("gates and inputs must have the same shape, type and device")
    if semiring not in (KLAY_REAL, KLAY_LOG, KLAY_MAXLOG):
        raise ValueError("unknown semiring")
    if semiring != KLAY_REAL and gates.dtype != torch.float32:
        raise ValueError("the log-domain semirings take float32")
    if gates.dim() < 2 or not 1 <= gates.shape[-1] <= _MOST_CHANNELS:
        raise ValueError("gates must have 1 .. 2^25 channels")


def gated_scan(gates, inputs, initial=None, semiring=KLAY_REAL, offsets=None):
    """``(states, final)`` of the recurrence h_t = gates_t (x) h_{t-1} (+) inputs_t in a semiring: ``KLAY_REAL`` a h + x (the linear
    recurrence of a recurrent network), ``KLAY_LOG`` log(exp(a + h) + exp(x)) (a chain of AND and OR gates on log-probabilities),
    ``KLAY_MAXLOG`` max(a + h, x) (its heaviest proof tree).

    ``gates``, ``inputs``: ``[B, T, C]``, float32, or bfloat16 / float16 in the real semiring; states are kept in float32 and
    rounded once into ``states`` (of the inputs' type).  ``initial``, ``final``: float32 ``[B, C]``, the states before the first and
    behind the last step (default: 0, in the log domain -inf).  With ``offsets`` (int64 ``[S + 1]``, ascending) the sequences lie
    one after the other: ``gates``, ``inputs`` are ``[N, C]``, sequence s is the rows ``offsets[s]`` to ``offsets[s + 1] - 1``, the
    states are ``[S, C]``; a sequence may be empty, and rows of none get states and gradients of 0.

    With 16-bit types the gradient of a gate is made with the state before it as it was returned, rounded to those bits (its relative
    error about half as much again: 2.3e-3 for 1.7e-3 in bfloat16); pass float32 where that matters.

    Differentiable (``KLAY_REAL``, ``KLAY_LOG``; backward only: tensors with tangents are refused) with respect to gates, inputs and
    initial, through both results.  The channels should be next to each other; other layouts are copied first.
    """
    _check_recurrence(gates, inputs, semiring)
    if gates.dim() != (3 if offsets is None else 2):
        raise ValueError("gates and inputs must be [B, T, C], or [N, C] with offsets")
    if offsets is not None:
        _check_tensor(offsets, "offsets", (torch.int64,))
        if offsets.dim() != 1 or offsets.shape[0] < 1 or not offsets.is_contiguous() or offsets.device != gates.device:
            raise ValueError("offsets must be a contiguous [S + 1] tensor on the device of gates")
    if initial is not None:
        _check_tensor(initial, "initial", (torch.float32,))
        sequences = gates.shape[0] if offsets is None else offsets.shape[0] - 1
        if initial.shape != (sequences, gates.shape[-1]) or initial.device != gates.device:
            raise ValueError("initial must be [%d, %d] on the device of gates" % (sequences, gates.shape[-1]))
    semiring = int(semiring)
    _refuse_tangents("gated_scan", gates, inputs, initial)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (gates, inputs, initial)):
        if semiring == KLAY_MAXLOG:
            raise RuntimeError("the (max, +) semiring is not differentiated; evaluate it under torch.no_grad()")
        return _GatedScan.apply(gates, inputs, initial, semiring, offsets)
    return _scan_forward(gates, inputs, initial, semiring, offsets)[:2]


def gated_step(gates, inputs, state, semiring=KLAY_REAL, out=None):
    """One step of :func:`gated_scan` for B running sequences: ``state`` (float32 ``[B, C]``) becomes gates (x) state (+) inputs in
    place, and a copy of it in the type of ``gates``, ``inputs`` (``[B, C]``) is returned (in ``out``, where given).  Not
    differentiated: the tensors must not require a gradient while gradients are enabled."""
    _check_recurrence(gates, inputs, semiring)
    _check_tensor(state, "state", (torch.float32,))
    if gates.dim() != 2 or state.shape != gates.shape or state.device != gates.device:
        raise ValueError("gates, inputs and state must be [B, C] on one device")
    if out is None:
        out = gates.new_empty(gates.shape)
    elif not isinstance(out, torch.Tensor) or out.shape != gates.shape or out.dtype != gates.dtype or out.device != gates.device:
        raise ValueError("out must have the shape, type and device of gates")
    batch, channels = gates.shape
    ss, os = state.stride(), out.stride()
    if (channels > 1 and (ss[1] != 1 or os[1] != 1)) or (batch > 1 and (ss[0] < channels or os[0] < channels)):
        raise ValueError("state and out must have their channels next to each other and rows that do not overlap")
    _refuse_tangents("gated_step", gates, inputs, state, out)
    if torch.is_grad_enabled() and (gates.requires_grad or inputs.requires_grad or state.requires_grad or out.requires_grad):
        raise RuntimeError("gated_step is not differentiated; call it under torch.no_grad(), or gated_scan")
    (gates, gs), (inputs, xs) = _channels_last(gates), _channels_last(inputs)
    device = gates.get_device()
    _b.klay_scan_step(_DTYPES[gates.dtype], semiring, device, batch, channels, gates.data_ptr(), gs[0], inputs.data_ptr(), xs[0],
                      state.data_ptr(), ss[0], out.data_ptr(), os[0], _stream(device))
    torch.autograd.graph.increment_version((state, out))          # written in place: a graph that has saved them is to notice
    return out
