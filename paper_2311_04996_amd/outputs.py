"""The operators beside the decoder: the output layer that makes its log-likelihoods out of an encoder's hidden
states, and the probabilities of what was decoded.

Argument marshalling only, like `binding`: every function enqueues HIP kernels on `stream` (default: torch's current
stream of the tensors' device) and returns without waiting.  All tensors of a call are on one GPU, which need not be the
current one.  Results are new tensors (allocated on `stream`) unless `out` gives them.  `linear` and `loglikes` are
for serving: they have no gradient, and their results are detached.  `token_logprobs` is recorded by autograd where
its scores require a gradient, and has its gradient as a function of its own, too.  Shapes, types and layouts that a kernel
does not take raise ValueError here, what else is wrong with a call raises WfstError.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple, Optional

from .binding import WFST_OK, WfstError, load_library, wfst_linear_args, wfst_loglikes_args, \
    wfst_token_logprobs_args, wfst_token_logprobs_backward_args

ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _packer(args):
    """The argument struct as bytes, in one step (filling a ctypes struct costs a small call a tenth of its time).  "0P": all of
    it, up to the next multiple of a pointer, as the library may copy it whole."""
    letter = {C.c_void_p: "P", C.c_int64: "q", C.c_int32: "i", C.c_float: "f"}
    return struct.Struct("@" + "".join(letter[t] for _, t in args._fields_) + "0P")


_linear, _loglikes = _packer(wfst_linear_args), _packer(wfst_loglikes_args)
_logprobs, _backward = _packer(wfst_token_logprobs_args), _packer(wfst_token_logprobs_backward_args)
torch = lib = _codes = _raw_stream = _Recorded = None


def _recorded(torch):
    """The autograd function of `token_logprobs` (torch is not imported before the first call)."""
    from torch.autograd.function import once_differentiable

    class TokenLogprobsFunction(torch.autograd.Function):
        @staticmethod
        def forward(ctx, scores, tokens, top, lengths, stream):
            r = _token_logprobs(scores, tokens, top, lengths, stream)
            ctx.save_for_backward(scores, tokens, lengths, r.entropy, r.maximum, r.log_sum, r.top_ids)
            ctx.mark_non_differentiable(*(t for t in (r.maximum, r.log_sum, r.top_ids) if t is not None))
            ctx.set_materialize_grads(False)
            return tuple(r)

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_logprobs, grad_lse, grad_entropy, grad_maximum, grad_log_sum, grad_ids, grad_top):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("token_logprobs: autograd's backward pass is not recorded into a graph: call token_logprobs_backward there")
            scores, tokens, lengths, entropy, maximum, log_sum, top_ids = ctx.saved_tensors
            result = TokenLogprobs(None, None, entropy, maximum, log_sum, top_ids, None)
            g_lp, g_lse, g_h, g_top = (None if g is None else g.contiguous() for g in (grad_logprobs, grad_lse, grad_entropy, grad_top))
            return token_logprobs_backward(scores, result, tokens, g_lp, g_lse, g_h, g_top, lengths=lengths), None, None, None, None

    return TokenLogprobsFunction


def _start():
    """On the first call: the library, and torch with it.  `lib` comes last: another thread takes it as the sign that all is there."""
    global torch, lib, _codes, _raw_stream, _Recorded
    library = load_library()
    import torch as t
    _codes = {t.float32: 0, t.float16: 1, t.bfloat16: 2}
    _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda dev: t.cuda.current_stream(dev).cuda_stream)
    _Recorded = _recorded(t)
    torch = t
    lib = library


def _device(t, what):
    if lib is None:
        _start()
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    return t.get_device()


def _code(t, what):
    c = _codes.get(t.dtype)
    if c is None:
        raise ValueError(f"{what} must be float32, float16 or bfloat16, not {t.dtype}")
    return c


def _there(t, dev, what):
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on cuda:{dev}")


def _matrix(t, what):
    """(rows, stride of a row) of a tensor [..., n] whose leading dimensions are one: a matrix, or a view that is like one."""
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    if len(st) == 2:
        return t.shape[0], st[0]
    if t.numel() == 0:
        return 0, t.shape[-1]
    rows, stride = 1, t.shape[-1]
    for size, s in zip(reversed(t.shape[:-1]), reversed(st[:-1])):
        if size == 1:
            continue
        if rows == 1:
            stride = s
        elif s != rows * stride:
            raise ValueError(f"the leading dimensions of {what} do not merge into one (strides {tuple(st)})")
        rows *= size
    return rows, stride


def _grid(t, what):
    """(sequences, frames, stride of a sequence, stride of a frame) of a tensor [frames, n] or [sequences, frames, n]."""
    st, n = t.stride(), t.dim()
    if n != 2 and n != 3:
        raise ValueError(f"{what} must have 2 or 3 dimensions, not {n}")
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return (t.shape[0], t.shape[1], st[0], st[1]) if n == 3 else (1, t.shape[0], 0, st[0])


def _dense(t, shape, dtype, what, dev):
    """Address of a contiguous tensor of this shape and type, 0 if there is none."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    _there(t, dev, what)
    return t.data_ptr()


def _vector(t, n, what, dev):
    """(address, type) of a contiguous vector of n values of any type."""
    if t is None:
        return 0, 0
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor of {n} entries")
    _there(t, dev, what)
    return t.data_ptr(), _code(t, what)


def _new(make, shape, dtype, dev, stream):
    """A new tensor, allocated (and filled) on the stream that the kernel runs on."""
    if stream is None:
        return make(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=dev)


def _run(entry, packer, fields, dev, stream):
    try:
        args = packer.pack(*fields)
    except struct.error as e:
        raise ValueError(f"a size, a stride or a number is out of range: {e}") from None
    if stream is not None:
        if stream.device.index != dev:
            raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{dev}")
        raw = stream.cuda_stream
    else:
        raw = _raw_stream(dev)
    if torch.cuda.current_device() == dev:
        rc = entry(args, raw)
    else:
        with torch.cuda.device(dev):
            rc = entry(args, raw)
    if rc != WFST_OK:
        raise WfstError(rc, lib.wfst_last_error(None).decode())


def linear(x, weight, bias=None, activation=None, residual=None, scale=1.0, out=None, out_dtype=None, stream=None):
    """residual + scale * activation(x @ weight.T + bias), in one kernel (wfst_linear).  No gradient: the result is detached.

    x: [..., k] and weight: [n, k], of one type (float32, float16 or bfloat16); their rows may have any stride.
    bias: [n], any of the types.  activation: None, "relu", "silu" or "gelu" (with erf).  residual: [..., n] of the
    result's type.  out: where the result goes, [..., n]; it may be `residual` itself.  out_dtype: the
    result's type without `out` (default x's)."""
    dev = _device(x, "x")
    shape = x.shape
    if x.dim() < 1 or weight.dim() != 2 or shape[-1] != weight.shape[1]:
        raise ValueError(f"x {tuple(shape)} and weight {tuple(weight.shape)} do not fit")
    if weight.dtype != x.dtype:
        raise ValueError(f"weight is {weight.dtype}, x is {x.dtype}")
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"unknown activation {activation!r}")
    n, k = weight.shape
    shape = (*shape[:-1], n)
    code = _code(x, "x")
    _there(weight, dev, "weight")
    ws = _matrix(weight, "weight")[1]
    b, b_code = _vector(bias, n, "bias", dev)
    rows, xs = _matrix(x, "x")
    if out is None:
        out = _new(torch.empty, shape, x.dtype if out_dtype is None else out_dtype, x.device, stream)
        ys = n
    else:
        if out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, the result {out_dtype or out.dtype} {shape}")
        _there(out, dev, "out")
        ys = _matrix(out, "out")[1]
    r = rs = 0
    if residual is not None:
        if residual.shape != shape or residual.dtype != out.dtype:
            raise ValueError(f"residual is {residual.dtype} {tuple(residual.shape)}, the result {out.dtype} {shape}")
        _there(residual, dev, "residual")
        r, rs = residual.data_ptr(), _matrix(residual, "residual")[1]
    _run(lib.wfst_linear, _linear, (x.data_ptr(), weight.data_ptr(), b, r, out.data_ptr(), rows, xs, ws, rs, ys, k, n, code, b_code,
                                    _code(out, "out"), act, scale), dev, stream)
    return out


def loglikes(hidden, weight, bias=None, log_prior=None, lengths=None, out=None, out_dtype=None, stream=None):
    """log_softmax(hidden @ weight.T + bias) - log_prior, in one kernel (wfst_loglikes): what `Decoder.decode_batch` and
    `Decoder.advance_chunk` take.  No gradient: the result is detached.

    hidden: [frames, k] or [sequences, frames, k], any strides of its first dimensions (time-major hidden states are
    given transposed); weight: [v, k] of hidden's type, v <= 2048; bias: [v]; log_prior: float32 [v].
    lengths: int32 CUDA tensor [sequences]: frames behind a sequence's length are not computed, and what `out` holds
    there stays (without `out` they are 0).  out_dtype: the result's type without `out` (default float32)."""
    dev = _device(hidden, "hidden")
    if weight.dim() != 2 or hidden.dim() < 1 or hidden.shape[-1] != weight.shape[1]:
        raise ValueError(f"hidden {tuple(hidden.shape)} and weight {tuple(weight.shape)} do not fit")
    if weight.dtype != hidden.dtype:
        raise ValueError(f"weight is {weight.dtype}, hidden is {hidden.dtype}")
    v, k = weight.shape
    shape = (*hidden.shape[:-1], v)
    code = _code(hidden, "hidden")
    _there(weight, dev, "weight")
    ws = _matrix(weight, "weight")[1]
    b, b_code = _vector(bias, v, "bias", dev)
    prior = _dense(log_prior, (v,), torch.float32, "log_prior", dev)
    seqs, frames, xss, xs = _grid(hidden, "hidden")
    le = _dense(lengths, (seqs,), torch.int32, "lengths", dev)
    if out is None:
        out = _new(torch.empty if lengths is None else torch.zeros, shape, out_dtype or torch.float32, hidden.device, stream)
    elif out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, the result {out_dtype or out.dtype} {shape}")
    _there(out, dev, "out")
    _, _, oss, os_ = _grid(out, "out")
    _run(lib.wfst_loglikes, _loglikes, (hidden.data_ptr(), weight.data_ptr(), b, prior, le, out.data_ptr(), xss, xs, ws, oss, os_,
                                        seqs, frames, k, v, code, b_code, _code(out, "out")), dev, stream)
    return out


class TokenLogprobs(NamedTuple):
    """What `token_logprobs` returns: float32 tensors, top_ids int32; None where nothing was asked for."""
    logprobs: Optional[object]       # [..., given]
    lse: object                      # [...]
    entropy: object                  # [...]
    maximum: object                  # [...]: the row's maximum,
    log_sum: object                  # [...]: and the log of its sum of e^(score - maximum): what the gradient needs
    top_ids: Optional[object]        # [..., top]
    top_logprobs: Optional[object]   # [..., top]


def token_logprobs(scores, tokens=None, top=0, lengths=None, stream=None):
    """Log-probabilities of given tokens, with the log of the sum, the entropy and the `top` best alternatives of every row of scores
    (wfst_token_logprobs).

    scores: [rows, v] or [sequences, frames, v] logits or log-likelihoods, float32, float16 or bfloat16, any strides of
    the first dimensions.  tokens: int32 [..., given] (or [...], one per row), -1 for none; at most 256 per row.  top: 0 to 64.
    lengths: int32 CUDA tensor [sequences]: rows behind a sequence's length are not read, their results are 0.
    A row that rules everything out (-inf) has lse -inf, log-probabilities -inf and entropy 0.

    Where the scores require a gradient (and grad mode is on) autograd records the call: logprobs, lse, entropy and top_logprobs have
    the gradient that token_logprobs_backward computes, the others are constants.  Its backward pass is not for graphs under capture
    (RuntimeError): there, token_logprobs_backward is called itself."""
    _device(scores, "scores")
    if not (scores.requires_grad and torch.is_grad_enabled()):
        return _token_logprobs(scores, tokens, top, lengths, stream)
    if stream is None:
        return TokenLogprobs(*_Recorded.apply(scores, tokens, top, lengths, None))
    for t in (scores, tokens, lengths):                  # (autograd decides when it lets go of them)
        if t is not None and t.is_cuda:
            t.record_stream(stream)
    with torch.cuda.stream(stream):                      # (autograd runs the backward pass on the forward's current stream)
        return TokenLogprobs(*_Recorded.apply(scores, tokens, top, lengths, stream))


def _token_logprobs(scores, tokens, top, lengths, stream):
    dev = scores.get_device()
    code = _code(scores, "scores")
    seqs, frames, ss, st = _grid(scores, "scores")
    lead, v = scores.shape[:-1], scores.shape[-1]
    if not 0 <= top <= min(v, 64):                       # (before its results are allocated)
        raise WfstError(-1, "wfst_token_logprobs: top must be 0 to 64, and at most v")
    le = _dense(lengths, (seqs,), torch.int32, "lengths", dev)
    new = torch.empty if lengths is None else torch.zeros
    f32, i32, on = torch.float32, torch.int32, scores.device
    given = tok = lp_at = ids_at = tlp_at = ws_at = 0
    lp = ids = tlp = ws = None
    if tokens is not None:
        if tokens.dim() == len(lead):
            given, shape = 1, lead
        else:
            given = tokens.shape[-1]
            shape = (*lead, given)
        tok = _dense(tokens, shape, i32, "tokens", dev)
        lp = _new(new, shape, f32, on, stream)
        lp_at = lp.data_ptr()
    if scores.requires_grad:                             # (autograd wants results that are no views)
        lse, entropy, maximum, log_sum = (_new(new, lead, f32, on, stream) for _ in range(4))
    else:
        lse, entropy, maximum, log_sum = _new(new, (4, *lead), f32, on, stream).unbind(0)
    if top > 0:
        ids, tlp = _new(new, (*lead, top), i32, on, stream), _new(new, (*lead, top), f32, on, stream)
        ids_at, tlp_at = ids.data_ptr(), tlp.data_ptr()
    need = lib.wfst_token_logprobs_workspace(seqs * frames, v, top)
    if need > 0:
        ws = _new(torch.empty, need, torch.uint8, on, stream)
        ws_at = ws.data_ptr()
    _run(lib.wfst_token_logprobs, _logprobs, (scores.data_ptr(), tok, le, lp_at, lse.data_ptr(), entropy.data_ptr(), maximum.data_ptr(),
                                              log_sum.data_ptr(), ids_at, tlp_at, ws_at, need, ss, st, seqs, frames, v, given, top, code), dev, stream)
    return TokenLogprobs(lp, lse, entropy, maximum, log_sum, ids, tlp)


def token_logprobs_backward(scores, result, tokens=None, grad_logprobs=None, grad_lse=None, grad_entropy=None, grad_top=None,
                            lengths=None, out=None, stream=None):
    """The gradient of `token_logprobs` with respect to its scores (wfst_token_logprobs_backward).

    scores, tokens, lengths: as the forward call had them; result: what it returned.  grad_*: float32 gradients of
    result.logprobs, .lse, .entropy and .top_logprobs (None: 0).  Returns the gradient in the scores' type and shape; out
    may be the scores themselves.  Rows behind a sequence's length are not computed (0 without `out`)."""
    dev = _device(scores, "scores")
    code = _code(scores, "scores")
    seqs, frames, ss, st = _grid(scores, "scores")
    lead, v = scores.shape[:-1], scores.shape[-1]
    f32 = torch.float32
    le = _dense(lengths, (seqs,), torch.int32, "lengths", dev)
    given = top = tok = gl = ids = gt = 0
    if grad_logprobs is not None:
        if tokens is None:
            raise ValueError("grad_logprobs without tokens")
        given = 1 if tokens.dim() == len(lead) else tokens.shape[-1]
        tok = _dense(tokens, lead if tokens.dim() == len(lead) else (*lead, given), torch.int32, "tokens", dev)
        gl = _dense(grad_logprobs, tokens.shape, f32, "grad_logprobs", dev)
    if grad_top is not None:
        if result.top_ids is None:
            raise ValueError("grad_top, but the result has no top alternatives")
        top = result.top_ids.shape[-1]
        ids = _dense(result.top_ids, (*lead, top), torch.int32, "top_ids", dev)
        gt = _dense(grad_top, (*lead, top), f32, "grad_top", dev)
    m, ls = _dense(result.maximum, lead, f32, "maximum", dev), _dense(result.log_sum, lead, f32, "log_sum", dev)
    gs, gh = _dense(grad_lse, lead, f32, "grad_lse", dev), _dense(grad_entropy, lead, f32, "grad_entropy", dev)
    h = _dense(result.entropy, lead, f32, "entropy", dev) if gh else 0
    if out is None:
        out = _new(torch.empty if lengths is None else torch.zeros, scores.shape, scores.dtype, scores.device, stream)
    elif out.shape != scores.shape or out.dtype != scores.dtype:
        raise ValueError(f"out must be a {scores.dtype} tensor {tuple(scores.shape)}")
    _there(out, dev, "out")
    _, _, oss, ost = _grid(out, "out")
    _run(lib.wfst_token_logprobs_backward, _backward, (scores.data_ptr(), tok, le, m, ls, h, ids, gl, gs, gh, gt, out.data_ptr(), ss, st, oss, ost,
                                                       seqs, frames, v, given, top, code), dev, stream)
    return out
