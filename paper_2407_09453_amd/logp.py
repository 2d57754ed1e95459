"""Log probabilities of given tokens, their entropy and the likeliest tokens from logits, and the logits' gradient, on torch tensors.
Calls as those of the 8-bit layers: asynchronous on the tensors' current stream, or on ``stream``, recording nothing for autograd."""
from __future__ import annotations

import struct

from .binding import BSP_F32, _current_stream
from .f8 import _bytes_of, _call, _on, _on_stream, _rows, _type, _unrecorded

_LOG_PROBS, _LOG_PROBS_GRAD = 18, 19
_pack_logp, _pack_grad = struct.Struct("=7qd9q").pack, struct.Struct("=7qd7q").pack


def _tokens(tokens, X):
    import torch
    assert tokens.dtype in (torch.int32, torch.int64), "tokens as int32 or int64"
    assert tokens.shape == (X.shape[0],) and (X.shape[0] < 2 or tokens.stride() == (1,)), "a token a row"
    _on(X, tokens)
    return tokens.data_ptr(), tokens.element_size()


def _each(t, X):
    if t is None:
        return 0
    assert _type(t) == BSP_F32 and t.shape == (X.shape[0],) and (X.shape[0] < 2 or t.stride() == (1,)), "a float a row"
    _on(X, t)
    return t.data_ptr()


def log_probs(logits, tokens, top: int = 0, scale: float = 1.0, stream=None):
    """(logp, lse, entropy, top_logp, top_tokens) of softmax(scale logits) for logits [T][V] (fp32 or bf16; V <= 2^21, 0 < scale <= 2^100): the
    log probability of each row's token [T] (int32 or int64; below 0 there is none, and it is 0; V and above: NaN), the log of the sum, the
    entropy, and the ``top`` (at most 64) largest log probabilities with their tokens (int32), of equal logits the lower token first; None with top = 0."""
    import torch
    if stream is not None:
        return _on_stream(stream, logits, log_probs, logits, tokens, top, scale)
    if logits.requires_grad:
        _unrecorded(3)
    T, V, ld = _rows(logits)
    token, size = _tokens(tokens, logits)
    n = _bytes_of("bsp_log_probs_workspace", T, V, top)
    top_logp = top_tokens = None
    if top:  # (one block of memory: each that is asked for takes its 1.4 us)
        logp, lse, entropy, top_logp, top_tokens = logits.new_empty(T * (3 + 2 * top), dtype=torch.float32).split_with_sizes((T, T, T, T * top, T * top))
        top_logp, top_tokens = top_logp.view(T, top), top_tokens.view(torch.int32).view(T, top)
    else:
        logp, lse, entropy = logits.new_empty((3, T), dtype=torch.float32).unbind(0)
    ws = logits.new_empty(n, dtype=torch.uint8) if n else None
    _call(_LOG_PROBS, _pack_logp(logits.data_ptr(), ld, _type(logits), T, V, token, size, scale, top, logp.data_ptr(), lse.data_ptr(), entropy.data_ptr(),
                                 top_logp.data_ptr() if top else 0, top_tokens.data_ptr() if top else 0, ws.data_ptr() if n else 0, n,
                                 _current_stream(logits)), "bsp_log_probs")
    return logp, lse, entropy, top_logp, top_tokens


def log_probs_grad(logits, tokens, lse, entropy, dlogp=None, dentropy=None, scale: float = 1.0, out=None, stream=None):
    """The gradient of the logits, in their type, from those of logp and of the entropy (float [T], or None: zeros) and from what
    ``log_probs`` returned.  ``out`` may be the logits themselves, which it then replaces."""
    if stream is not None:
        return _on_stream(stream, logits, log_probs_grad, logits, tokens, lse, entropy, dlogp, dentropy, scale, out)
    if logits.requires_grad or (dlogp is not None and dlogp.requires_grad) or (dentropy is not None and dentropy.requires_grad):
        _unrecorded(3)
    T, V, ld = _rows(logits)
    token, size = _tokens(tokens, logits)
    if out is None:
        out = logits.new_empty((T, V))
        ld_out = V
    else:
        T2, V2, ld_out = _rows(out)
        assert (T2, V2) == (T, V) and out.dtype == logits.dtype
        _on(logits, out)
    _call(_LOG_PROBS_GRAD, _pack_grad(logits.data_ptr(), ld, _type(logits), T, V, token, size, scale, _each(lse, logits), _each(entropy, logits),
                                      _each(dlogp, logits), _each(dentropy, logits), out.data_ptr(), ld_out, _current_stream(logits)), "bsp_log_probs_grad")
    return out
