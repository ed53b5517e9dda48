"""The operators beside the decoder: the output layer that makes its log-likelihoods out of an encoder's hidden
states, and the probabilities of what was decoded.

Argument marshalling only, like `binding`: every function enqueues HIP kernels on `stream` (default: torch's current
stream of the tensors' device) and returns without waiting.  All tensors of a call are on one GPU, which need not be the
current one.  Results are new tensors (allocated on `stream`) unless `out` gives them.  Nothing is recorded by
autograd: `token_logprobs` has its gradient as a function of its own.  Shapes, types and layouts that a kernel does not
take raise ValueError here, what else is wrong with a call raises WfstError.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import NamedTuple, Optional

from .binding import WFST_OK, WfstError, _on, load_library, wfst_linear_args, wfst_loglikes_args, \
    wfst_token_logprobs_args, wfst_token_logprobs_backward_args

ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}
_types = None


def _type_codes():
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
    return _types


def _code(t, what):
    c = _type_codes().get(t.dtype)
    if c is None:
        raise ValueError(f"{what} must be float32, float16 or bfloat16, not {t.dtype}")
    return c


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, not on {dev}")


def _inner(t, what):
    """The last dimension's elements lie one after the other."""
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")


def _row_stride(t, what):
    """(rows, stride of a row) of a tensor [..., n] whose leading dimensions are one: a matrix, or a view that is like one."""
    _inner(t, what)
    if t.dim() == 2:
        return t.shape[0], t.stride(0)
    if t.dim() == 1:
        return 1, t.shape[0]
    rows, stride = 1, 0
    for size, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if rows == 1:
            stride = st
        elif st != rows * stride:
            raise ValueError(f"the leading dimensions of {what} do not merge into one (strides {tuple(t.stride())})")
        rows *= size
    return rows, stride if rows > 1 else t.shape[-1]


def _grid(t, what):
    """(sequences, frames, stride of a sequence, stride of a frame) of a tensor [n] / [frames, n] / [sequences, frames, n]."""
    _inner(t, what)
    if t.dim() == 3:
        return t.shape[0], t.shape[1], t.stride(0), t.stride(1)
    if t.dim() == 2:
        return 1, t.shape[0], 0, t.stride(0)
    raise ValueError(f"{what} must have 2 or 3 dimensions, not {t.dim()}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _lengths(lengths, seqs, dev):
    import torch
    if lengths is None:
        return
    if lengths.dtype != torch.int32 or lengths.shape != (seqs,) or not lengths.is_contiguous():
        raise ValueError(f"lengths must be a contiguous int32 tensor of {seqs} entries")
    _same_device(dev, lengths=lengths)


def _dense(t, shape, dtype, what, dev):
    if t is None:
        return
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    _same_device(dev, **{what: t})


def _cuda(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")


def _run(entry, args, dev, stream):
    import torch
    s = torch.cuda.current_stream(dev) if stream is None else stream
    if s.device != dev:
        raise ValueError(f"the stream is on {s.device}, the tensors on {dev}")
    with contextlib.nullcontext() if torch.cuda.current_device() == dev.index else torch.cuda.device(dev):
        rc = entry(C.byref(args), s.cuda_stream)
    if rc != WFST_OK:
        raise WfstError(rc, load_library().wfst_last_error(None).decode())


def linear(x, weight, bias=None, activation=None, residual=None, scale=1.0, out=None, out_dtype=None, stream=None):
    """residual + scale * activation(x @ weight.T + bias), in one kernel (wfst_linear).

    x: [..., k] and weight: [n, k], of one type (float32, float16 or bfloat16); their rows may have any stride.
    bias: [n], any of the types.  activation: None, "relu", "silu" or "gelu" (with erf).  residual: [..., n] of the
    result's type.  out: where the result goes, [..., n]; it may be `residual` itself.  out_dtype: the
    result's type without `out` (default x's)."""
    import torch
    _cuda(x, "x")
    dev = x.device
    if x.dim() < 1 or weight.dim() != 2 or x.shape[-1] != weight.shape[1]:
        raise ValueError(f"x {tuple(x.shape)} and weight {tuple(weight.shape)} do not fit")
    if weight.dtype != x.dtype:
        raise ValueError(f"weight is {weight.dtype}, x is {x.dtype}")
    if activation not in ACTIVATIONS:
        raise ValueError(f"unknown activation {activation!r}")
    n = weight.shape[0]
    shape = (*x.shape[:-1], n)
    _same_device(dev, weight=weight, bias=bias, residual=residual, out=out)
    _inner(weight, "weight")
    if bias is not None and (tuple(bias.shape) != (n,) or (n > 1 and bias.stride(0) != 1)):
        raise ValueError(f"bias must be a contiguous tensor of {n} entries")
    if out is None:
        with _on(stream):
            out = torch.empty(shape, dtype=x.dtype if out_dtype is None else out_dtype, device=dev)
    elif tuple(out.shape) != shape or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, the result {out_dtype or out.dtype} {shape}")
    rows, xs = _row_stride(x, "x")
    _, ys = _row_stride(out, "out")
    rs = 0
    if residual is not None:
        if tuple(residual.shape) != shape or residual.dtype != out.dtype:
            raise ValueError(f"residual is {residual.dtype} {tuple(residual.shape)}, the result {out.dtype} {shape}")
        rs = _row_stride(residual, "residual")[1]
    args = wfst_linear_args(x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(residual), out.data_ptr(), rows, xs, weight.stride(0), rs, ys,
                            x.shape[-1], n, _code(x, "x"), 0 if bias is None else _code(bias, "bias"), _code(out, "out"),
                            ACTIVATIONS[activation], float(scale))
    _run(load_library().wfst_linear, args, dev, stream)
    return out


def loglikes(hidden, weight, bias=None, log_prior=None, lengths=None, out=None, out_dtype=None, stream=None):
    """log_softmax(hidden @ weight.T + bias) - log_prior, in one kernel (wfst_loglikes): what `Decoder.decode_batch` and
    `Decoder.advance_chunk` take.

    hidden: [frames, k] or [sequences, frames, k], any strides of its first dimensions (time-major hidden states are
    given transposed); weight: [v, k] of hidden's type, v <= 2048; bias: [v]; log_prior: float32 [v].
    lengths: int32 CUDA tensor [sequences]: frames behind a sequence's length are not computed, and what `out` holds
    there stays (without `out` they are 0).  out_dtype: the result's type without `out` (default float32)."""
    import torch
    _cuda(hidden, "hidden")
    dev = hidden.device
    if weight.dim() != 2 or hidden.dim() not in (2, 3) or hidden.shape[-1] != weight.shape[1]:
        raise ValueError(f"hidden {tuple(hidden.shape)} and weight {tuple(weight.shape)} do not fit")
    if weight.dtype != hidden.dtype:
        raise ValueError(f"weight is {weight.dtype}, hidden is {hidden.dtype}")
    v = weight.shape[0]
    shape = (*hidden.shape[:-1], v)
    _same_device(dev, weight=weight, bias=bias, out=out)
    _inner(weight, "weight")
    if bias is not None and (tuple(bias.shape) != (v,) or (v > 1 and bias.stride(0) != 1)):
        raise ValueError(f"bias must be a contiguous tensor of {v} entries")
    _dense(log_prior, (v,), torch.float32, "log_prior", dev)
    seqs, frames, xss, xs = _grid(hidden, "hidden")
    _lengths(lengths, seqs, dev)
    if out is None:
        with _on(stream):
            out = (torch.empty if lengths is None else torch.zeros)(shape, dtype=out_dtype or torch.float32, device=dev)
    elif tuple(out.shape) != shape or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, the result {out_dtype or out.dtype} {shape}")
    _, _, oss, os_ = _grid(out, "out")
    args = wfst_loglikes_args(hidden.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(log_prior), _ptr(lengths), out.data_ptr(),
                              xss, xs, weight.stride(0), oss, os_, seqs, frames, hidden.shape[-1], v,
                              _code(hidden, "hidden"), 0 if bias is None else _code(bias, "bias"), _code(out, "out"))
    _run(load_library().wfst_loglikes, args, dev, stream)
    return out


class TokenLogprobs(NamedTuple):
    """What `token_logprobs` returns: float32 tensors, top_ids int32; None where nothing was asked for."""
    logprobs: Optional[object]       # [..., given]
    lse: object                      # [...]
    entropy: object                  # [...]
    stats: object                    # [..., 2]: the row's maximum, and the log of its sum of e^(score - maximum)
    top_ids: Optional[object]        # [..., top]
    top_logprobs: Optional[object]   # [..., top]


def token_logprobs(scores, tokens=None, top=0, lengths=None, stream=None):
    """Log-probabilities of given tokens, with the log of the sum, the entropy and the `top` best alternatives of every row of scores
    (wfst_token_logprobs).

    scores: [rows, v] or [sequences, frames, v] logits or log-likelihoods, float32, float16 or bfloat16, any strides of
    the first dimensions.  tokens: int32 [..., given] (or [...], one per row), -1 for none.  top: 0 to 64.
    lengths: int32 CUDA tensor [sequences]: rows behind a sequence's length are not read, their results are 0.
    A row that rules everything out (-inf) has lse -inf, log-probabilities -inf and entropy 0."""
    import torch
    _cuda(scores, "scores")
    dev = scores.device
    seqs, frames, ss, st = _grid(scores, "scores")
    lead, v = tuple(scores.shape[:-1]), scores.shape[-1]
    _lengths(lengths, seqs, dev)
    given = 0
    if tokens is not None:
        given = 1 if tokens.dim() == len(lead) else tokens.shape[-1]
        _dense(tokens, lead if tokens.dim() == len(lead) else (*lead, given), torch.int32, "tokens", dev)
    top = int(top)
    lib = load_library()
    with _on(stream):
        new = torch.empty if lengths is None else torch.zeros
        lp = new(tuple(tokens.shape), dtype=torch.float32, device=dev) if tokens is not None else None
        lse, ent = new(lead, dtype=torch.float32, device=dev), new(lead, dtype=torch.float32, device=dev)
        stats = new((*lead, 2), dtype=torch.float32, device=dev)
        ids = new((*lead, top), dtype=torch.int32, device=dev) if top > 0 else None
        tlp = new((*lead, top), dtype=torch.float32, device=dev) if top > 0 else None
        need = lib.wfst_token_logprobs_workspace(seqs * frames, v, top)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need > 0 else None
    args = wfst_token_logprobs_args(scores.data_ptr(), _ptr(tokens), _ptr(lengths), _ptr(lp), lse.data_ptr(), ent.data_ptr(), stats.data_ptr(),
                                    _ptr(ids), _ptr(tlp), _ptr(ws), max(need, 0), ss, st, seqs, frames, v, given, top, _code(scores, "scores"))
    _run(lib.wfst_token_logprobs, args, dev, stream)
    return TokenLogprobs(lp, lse, ent, stats, ids, tlp)


def token_logprobs_backward(scores, result, tokens=None, grad_logprobs=None, grad_lse=None, grad_entropy=None, grad_top=None,
                            lengths=None, out=None, stream=None):
    """The gradient of `token_logprobs` with respect to its scores (wfst_token_logprobs_backward).

    scores, tokens, lengths: as the forward call had them; result: what it returned.  grad_*: float32 gradients of
    result.logprobs, .lse, .entropy and .top_logprobs (None: 0).  Returns the gradient in the scores' type and shape; out
    may be the scores themselves.  Rows behind a sequence's length are not computed (0 without `out`)."""
    import torch
    _cuda(scores, "scores")
    dev = scores.device
    seqs, frames, ss, st = _grid(scores, "scores")
    lead, v = tuple(scores.shape[:-1]), scores.shape[-1]
    _lengths(lengths, seqs, dev)
    given, top = 0, 0
    if tokens is not None:
        given = 1 if tokens.dim() == len(lead) else tokens.shape[-1]
        _dense(tokens, lead if tokens.dim() == len(lead) else (*lead, given), torch.int32, "tokens", dev)
        _dense(grad_logprobs, tokens.shape, torch.float32, "grad_logprobs", dev)
    elif grad_logprobs is not None:
        raise ValueError("grad_logprobs without tokens")
    if grad_top is not None:
        if result.top_ids is None:
            raise ValueError("grad_top, but the result has no top alternatives")
        top = result.top_ids.shape[-1]
        _dense(result.top_ids, (*lead, top), torch.int32, "top_ids", dev)
        _dense(grad_top, (*lead, top), torch.float32, "grad_top", dev)
    _dense(result.stats, (*lead, 2), torch.float32, "stats", dev)
    _dense(result.entropy, lead, torch.float32, "entropy", dev)
    _dense(grad_lse, lead, torch.float32, "grad_lse", dev)
    _dense(grad_entropy, lead, torch.float32, "grad_entropy", dev)
    if out is None:
        with _on(stream):
            out = (torch.empty if lengths is None else torch.zeros)(tuple(scores.shape), dtype=scores.dtype, device=dev)
    elif out.shape != scores.shape or out.dtype != scores.dtype or out.device != dev:
        raise ValueError(f"out must be a {scores.dtype} tensor {tuple(scores.shape)} on {dev}")
    _, _, gs, gt = _grid(out, "out")
    args = wfst_token_logprobs_backward_args(
        scores.data_ptr(), _ptr(tokens), _ptr(lengths), result.stats.data_ptr(), result.entropy.data_ptr(),
        _ptr(result.top_ids) if top else None, _ptr(grad_logprobs), _ptr(grad_lse), _ptr(grad_entropy), _ptr(grad_top), out.data_ptr(),
        ss, st, gs, gt, seqs, frames, v, given, top, _code(scores, "scores"))
    _run(load_library().wfst_token_logprobs_backward, args, dev, stream)
    return out
