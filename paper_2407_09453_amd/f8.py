"""FC layers in 8-bit floating point, the 8-bit checkpoints of their inputs, their gradients, and layer norm, on torch
tensors.  Marshalling only: every call launches on the current stream of its tensors' device and returns before it is done;
tensors that it makes come from torch's allocator on that stream.

With ``stream`` (a handle as an integer) a call does as under ``torch.cuda.stream`` of that stream: what it reads has to be
ready there and is kept until it is done there (unless a call in that stream made it), and whoever uses its results elsewhere
waits for it.  Results may be dropped at any time, also behind uses in the stream that was current at the call.

Gradients are calls of their own: none of these records a graph for autograd, and a call whose results would be part of one
(an input requires a gradient, outside ``torch.no_grad``) says so with a warning.

A call's arguments go to the library as one string of words: of a small layer's 9 us on the host ctypes' conversion of 16 arguments
one by one took 2, and a tensor of torch's takes 1.5 us to make, so a checkpoint is one allocation."""
from __future__ import annotations

import ctypes
import struct
import warnings
from typing import Optional

import numpy as np

from .binding import (BSP_BF16, BSP_E4M3, BSP_E5M2, BSP_F32, BspError, _check, _current_stream, _np_ptr, bsp_codes,
                      bsp_weights_f8, load_library)

CODES = {"e4m3": BSP_E4M3, "e5m2": BSP_E5M2}
_SAVE, _LOAD, _FC, _VALUES, _GRAD, _NORM, _NORM_GRAD = range(7)
_pack9, _pack13, _pack17, _pack18, _pack20 = (struct.Struct("=%dq" % n).pack for n in (9, 13, 17, 18, 20))
_pack_norm = struct.Struct("=7qd10q").pack
_NO_CODES = (0, 0, 0, 0, 0)
_types = _torch = None


def _type(t) -> int:
    global _types
    if _types is None:
        import torch
        _types = {torch.bfloat16: BSP_BF16, torch.float32: BSP_F32}
    code = _types.get(t.dtype)
    assert code is not None, t.dtype
    return code


def _rows(t):
    """(T, K, elements from row to row) of a matrix whose rows are contiguous; rows may lie any distance apart."""
    T, K = t.shape
    ld, one = t.stride()
    assert t.is_cuda and (one == 1 or K == 1 or T == 0), "a matrix on a GPU with contiguous rows"
    return T, K, ld if T > 1 else K


def _blocks(n: int) -> int:
    return (n + 127) >> 7


def _on(t, *others):
    at = t.get_device()
    for o in others:
        assert o is None or o.get_device() == at, "tensors on different devices"


def _call(call, words, name):
    rc = load_library().bsp_f8_call_packed(call, words)
    if rc:
        raise BspError(rc, name)


def _unrecorded(depth: int):
    import torch
    if torch.is_grad_enabled():
        warnings.warn("an input requires a gradient, but this call records nothing for autograd: see grad_input, grad_weight and "
                      "layer_norm_grad (torch.no_grad() says that this is meant)", UserWarning, stacklevel=depth)


def _memory(v):
    """The tensors that a result is held in."""
    if isinstance(v, (tuple, list)):
        for x in v:
            yield from _memory(x)
    elif isinstance(v, BspCodes):
        yield v.buffer
    elif v is not None:
        yield v


def _on_stream(stream, at, call, *args):
    """call(*args) in the stream of this handle, on the device of tensor ``at``.  Workspaces and results come from the allocator's pool of
    that stream: a block of the current stream's pool may be one that was dropped there with work on it still to come, which
    the call, elsewhere, would not wait for.  Nothing is recorded for that stream, which is its owner's: what is recorded
    for a stream can be freed only while the stream is there."""
    import torch
    if int(stream) == _current_stream(at):
        return call(*args)
    here = torch.cuda.current_stream(at.device)
    # (an ExternalStream of no handle is not the default stream, but any of torch's)
    there = torch.cuda.ExternalStream(int(stream), device=at.device) if int(stream) else torch.cuda.default_stream(at.device)
    device = torch.cuda.current_device()
    torch.cuda.set_stream(there)  # (and its device; torch.cuda.stream's context takes twice as long)
    try:
        result = call(*args)
    finally:
        torch.cuda.set_stream(here)
        if device != there.device.index:
            torch.cuda.set_device(device)
    for t in _memory(result):
        t.record_stream(here)
    return result


class BspCodes:
    """A matrix [T][K] held as 8-bit floating-point codes with a power-of-two scale for each row's 128 columns: the form in
    which a layer's input is kept for the backward pass.  ``codes`` [T][128 ceil(K/128)] and ``scale``
    [ceil(K/128)][16 ceil(T/16)] (exponent + 127) are uint8 views of one buffer; ``kind`` is "e4m3" or "e5m2"."""

    __slots__ = ("T", "K", "kind", "buffer", "words")

    def __init__(self, T: int, K: int, kind: str = "e4m3", device="cuda:0"):
        import torch
        self.T, self.K, self.kind = T, K, kind
        nb = _blocks(K)
        self.buffer = torch.empty(nb * (128 * T + (T + 15 & ~15)), dtype=torch.uint8, device=device)
        p = self.buffer.data_ptr()
        self.words = (T, K, CODES[kind], p, p + nb * 128 * T)

    @property
    def codes(self):
        n = _blocks(self.K) * 128
        return self.buffer[:self.T * n].view(self.T, n)

    @property
    def scale(self):
        nb = _blocks(self.K)
        return self.buffer[self.T * nb * 128:].view(nb, self.T + 15 & ~15)

    @property
    def struct(self):
        return bsp_codes(*self.words[:3], self.words[3] or None, self.words[4] or None)

    def load(self, dtype=None, out=None, stream=None):
        """The values, as bf16 (or torch.float32)."""
        if stream is not None:
            return _on_stream(stream, self.buffer, self.load, dtype, out)
        if out is None:
            import torch
            out = torch.empty((self.T, self.K), dtype=dtype or torch.bfloat16, device=self.buffer.device)
            ld = self.K
        else:
            T, K, ld = _rows(out)
            assert (T, K) == (self.T, self.K)
            _on(self.buffer, out)
        _call(_LOAD, _pack9(*self.words, out.data_ptr(), _type(out), ld, _current_stream(out)), "bsp_f8_load")
        return out


def save8(X, kind: Optional[str] = None, out: Optional[BspCodes] = None, stream=None) -> BspCodes:
    """The 8-bit checkpoint of X (torch tensor [T][K], fp32 or bf16, rows contiguous), in codes of type ``kind``: e4m3 where none
    is asked for, or the type of ``out``."""
    if stream is not None:
        return _on_stream(stream, X, save8, X, kind, out)
    if X.requires_grad:
        _unrecorded(3)
    T, K, ld = _rows(X)
    if out is None:
        out = BspCodes(T, K, kind or "e4m3", X.device)
    else:
        assert (out.T, out.K) == (T, K)
        assert kind is None or kind == out.kind, "codes of %s asked for in a checkpoint of %s" % (kind, out.kind)
        _on(X, out.buffer)
    _call(_SAVE, _pack9(X.data_ptr(), _type(X), ld, *out.words, _current_stream(X)), "bsp_f8_save")
    return out


class BspLayerF8:
    """An FC layer Y = X W^t + b in 8-bit floating point, resident on a GPU: W [O][I] (numpy, or a torch tensor in fp32 or
    bf16) under a mask ``gamma`` [ceil(O/128)][ceil(I/128)] (1 = kept; None keeps all), bias float or None.  Each kept block
    of 128 x 128 weights is held as e4m3 codes with one power-of-two scale, in both directions: by rows for the layer,
    by columns for the gradient of its input."""

    def __init__(self, W, gamma=None, bias=None, device="cuda:0"):
        import torch
        global _torch
        _torch = torch
        lib = load_library()
        self.device = torch.device(device)
        O, I = W.shape
        self.O, self.I = O, I
        nbo, nbi = _blocks(O), _blocks(I)
        if gamma is None:
            gamma = np.ones((nbo, nbi), np.uint8)
        if isinstance(gamma, torch.Tensor):
            gamma = gamma.cpu().numpy()
        gamma = np.ascontiguousarray(gamma, dtype=np.uint8)
        assert gamma.shape == (nbo, nbi), (gamma.shape, (nbo, nbi))
        n = ctypes.c_int64(0)
        _check(lib.bsp_f8_count(_np_ptr(gamma), O, I, ctypes.byref(n)), "bsp_f8_count")
        self.gamma, self.nnzb = gamma, n.value
        self.row_ptr, self.col_idx = np.zeros(nbo + 1, np.int32), np.zeros(max(self.nnzb, 1), np.int32)
        self.col_ptr, self.row_idx = np.zeros(nbi + 1, np.int32), np.zeros(max(self.nnzb, 1), np.int32)
        _check(lib.bsp_f8_index(_np_ptr(gamma), O, I, self.col_idx.size, _np_ptr(self.row_ptr), _np_ptr(self.col_idx),
                                _np_ptr(self.col_ptr), _np_ptr(self.row_idx)), "bsp_f8_index")
        self.d_index = [torch.from_numpy(a).to(self.device) for a in (self.row_ptr, self.col_idx, self.col_ptr, self.row_idx)]
        # (a block where none is kept, so that an empty layer has addresses)
        self.payload, self.payload_t = (torch.empty((max(self.nnzb, 1), 128, 128), dtype=torch.uint8, device=self.device) for _ in range(2))
        self.scale, self.scale_t = (torch.empty(max(self.nnzb, 1), dtype=torch.uint8, device=self.device) for _ in range(2))
        self.struct = bsp_weights_f8(O, I, self.nnzb, *(t.data_ptr() for t in self.d_index), self.payload.data_ptr(),
                                     self.scale.data_ptr(), self.payload_t.data_ptr(), self.scale_t.data_ptr())
        self._address = ctypes.addressof(self.struct)
        self.device, self._index = self.payload.device, self.payload.get_device()
        self._workspace = {}  # bytes that a call takes, by its kind and rows
        self.d_bias = None
        if bias is not None:  # (a copy, as the weights' codes are: the caller's tensor stays the caller's)
            b = torch.as_tensor(bias).detach().to(self.device, torch.float32, copy=True, memory_format=torch.contiguous_format)
            assert b.shape == (O,), "a bias [%d]" % O
            self.d_bias = b
        self.update(W)

    def update(self, W, bias=None, stream=None) -> None:
        """Take new weights (same shape, same mask), and a new bias where one is given (to a layer that was made with one), as
        after a step of an optimiser."""
        import torch
        if stream is not None:
            return _on_stream(stream, self.payload, self.update, W, bias)
        if not isinstance(W, torch.Tensor):
            W = torch.from_numpy(np.ascontiguousarray(W, dtype=np.float32))
        W = W.to(self.device)
        O, I, ld = _rows(W)
        assert (O, I) == (self.O, self.I)
        kind = _type(W)
        if bias is not None:
            b = torch.as_tensor(bias).detach()
            assert self.d_bias is not None and b.shape == (O,), "a bias [%d] for a layer made with one" % O
            self.d_bias.copy_(b)
        _check(load_library().bsp_f8_pack(self.struct, W.data_ptr(), kind, ld, _current_stream(W)), "bsp_f8_pack")

    def _bytes(self, kind, T):
        n = self._workspace.get((kind, T))
        if n is None:
            lib, n = load_library(), ctypes.c_int64(0)
            if kind == "grad":
                _check(lib.bsp_f8_fc_grad_workspace(self.struct, T, n), "bsp_f8_fc_grad_workspace")
            else:
                _check(lib.bsp_f8_fc_workspace(self.struct, kind >> 1, T, kind & 1, n), "bsp_f8_fc_workspace")
            if len(self._workspace) > 4096:
                self._workspace.clear()
            n = self._workspace[(kind, T)] = n.value
        return n

    def _multiply(self, transposed, X, code, bias, residual, relu, gate, dtype, out):
        codes = type(X) is BspCodes
        if codes:
            T, K, at = X.T, X.K, X.buffer
        else:
            if X.requires_grad:
                _unrecorded(4)
            T, K, ld = _rows(X)
            at = X
        width, inner = (self.I, self.O) if transposed else (self.O, self.I)
        assert K == inner, (K, inner)
        assert at.get_device() == self._index, "tensors on different devices"
        if out is None:
            if dtype is None:
                dtype = _torch.bfloat16 if codes else X.dtype
            out = _torch.empty((T, width), dtype=dtype, device=self.device)
        else:
            assert out.shape == (T, width) and out.is_contiguous()
            _on(at, out)
        r, g = 0, _NO_CODES
        if residual is not None:
            if residual.requires_grad:
                _unrecorded(4)
            assert residual.shape == out.shape and residual.dtype == out.dtype and residual.is_contiguous()
            _on(at, residual)
            r = residual.data_ptr()
        if gate is not None:
            _on(at, gate.buffer)
            g = gate.words
        st = _current_stream(out)
        if codes:
            n = self._bytes(transposed * 2 + 1, T)
        else:  # (few whole rows become codes inside the product's kernel)
            x, size = X.data_ptr(), X.element_size()
            inside = T <= 16 and not (x | ld * size | K * size) & 15 and T * (_blocks(K) * 129 + 16) <= 73728
            n = self._bytes(transposed * 2 + inside, T)
        ws = _torch.empty(n, dtype=_torch.uint8, device=self.device) if n else None
        rest = (0 if bias is None else bias.data_ptr(), r, 1 if relu else 0, *g, out.data_ptr(), _type(out), 0 if ws is None else ws.data_ptr(), n, st)
        if codes:
            _call(_FC, _pack20(self._address, transposed, *X.words, *rest), "bsp_f8_fc")
        else:
            _call(_VALUES, _pack20(self._address, transposed, x, _type(X), ld, T, CODES[code], *rest), "bsp_f8_fc_values")
        return out

    def fc(self, X, relu=False, residual=None, dtype=None, out=None, stream=None):
        """Y [T][O] = act(X W^t + b + residual) for X [T][I]: a torch tensor (fp32 or bf16, brought to e4m3 codes within the
        call; Y has its type unless ``dtype`` says otherwise) or a BspCodes (Y is bf16 unless ``dtype`` says otherwise)."""
        if stream is not None:
            return _on_stream(stream, self.payload, self.fc, X, relu, residual, dtype, out)
        return self._multiply(0, X, "e4m3", self.d_bias, residual, relu, None, dtype, out)

    def grad_input(self, dY, relu_of: Optional[BspCodes] = None, code: str = "e5m2", dtype=None, out=None, stream=None):
        """dX [T][I] = dY W for dY [T][O] (brought to codes of type ``code`` within the call, or a BspCodes).  ``relu_of``: the
        checkpoint of this layer's input, where that is a ReLU's output; the result is then the gradient of what went
        into the ReLU."""
        if stream is not None:
            return _on_stream(stream, self.payload, self.grad_input, dY, relu_of, code, dtype, out)
        return self._multiply(1, dY, code, None, None, False, relu_of, dtype, out)

    def grad_weight(self, dY, X: BspCodes, bias: bool = True, out=None, stream=None):
        """(dW, db) from dY (bf16 [T][O]) and the checkpoint of the layer's input: dW float [O][I], zero where the mask is; db
        float [O], or None."""
        import torch
        if stream is not None:
            return _on_stream(stream, self.payload, self.grad_weight, dY, X, bias, out)
        if dY.requires_grad:
            _unrecorded(3)
        T, O, ld = _rows(dY)
        assert dY.dtype == torch.bfloat16 and (T, O) == (X.T, self.O)
        _on(self.payload, dY, X.buffer, out)
        if out is None:
            out = torch.empty((self.O, self.I), dtype=torch.float32, device=dY.device)
        else:
            assert out.shape == (self.O, self.I) and out.dtype == torch.float32 and out.is_contiguous()
        db = torch.empty(self.O, dtype=torch.float32, device=dY.device) if bias else None
        n = self._bytes("grad", T)
        ws = torch.empty(n, dtype=torch.uint8, device=dY.device) if n else None
        _call(_GRAD, _pack13(self._address, dY.data_ptr(), ld, *X.words, out.data_ptr(), 0 if db is None else db.data_ptr(),
                             0 if ws is None else ws.data_ptr(), n, _current_stream(dY)), "bsp_f8_fc_grad")
        return out, db


def _vector(t, D):
    if t is None:
        return 0
    assert t.is_cuda and _type(t) == BSP_F32 and t.shape == (D,) and t.is_contiguous()
    return t.data_ptr()


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5, code: Optional[str] = None, stream=None):
    """(Y, mean, rstd) of X [T][D] (fp32 or bf16) over its last axis; ``weight`` and ``bias`` are float [D] or None.  With ``code``
    ("e4m3", "e5m2") Y is a BspCodes, the form in which a BspLayerF8 reads it."""
    import torch
    if stream is not None:
        return _on_stream(stream, X, layer_norm, X, weight, bias, eps, code)
    if X.requires_grad or (weight is not None and weight.requires_grad) or (bias is not None and bias.requires_grad):
        _unrecorded(3)
    T, D, ld = _rows(X)
    _on(X, weight, bias)
    mean, rstd = torch.empty((2, T), dtype=torch.float32, device=X.device).unbind(0)
    if code is None:
        Y = torch.empty((T, D), dtype=X.dtype, device=X.device)
        y, words = Y.data_ptr(), _NO_CODES
    else:
        Y = BspCodes(T, D, code, X.device)
        y, words = 0, Y.words
    _call(_NORM, _pack_norm(X.data_ptr(), _type(X), ld, T, D, _vector(weight, D), _vector(bias, D), eps, y, D, *words, mean.data_ptr(),
                            rstd.data_ptr(), _current_stream(X)), "bsp_layer_norm")
    return Y, mean, rstd


def layer_norm_grad(dY, X, mean, rstd, weight=None, stream=None):
    """(dX, dweight, dbias) from the gradient of Y, the input and what ``layer_norm`` returned with it."""
    import torch
    if stream is not None:
        return _on_stream(stream, X, layer_norm_grad, dY, X, mean, rstd, weight)
    if dY.requires_grad or X.requires_grad or (weight is not None and weight.requires_grad):
        _unrecorded(3)
    T, D, ld = _rows(X)
    T2, D2, ld_dy = _rows(dY)
    assert (T2, D2) == (T, D) and dY.dtype == X.dtype and mean.shape == rstd.shape == (T,)
    assert _type(mean) == _type(rstd) == BSP_F32 and (T < 2 or mean.stride() == rstd.stride() == (1,))
    _on(X, dY, mean, rstd, weight)
    dX = torch.empty((T, D), dtype=X.dtype, device=X.device)
    dw, db = torch.empty((2, D), dtype=torch.float32, device=X.device).unbind(0)
    n = _norm_bytes(T, D)
    ws = torch.empty(n, dtype=torch.uint8, device=X.device) if n else None
    _call(_NORM_GRAD, _pack17(dY.data_ptr(), ld_dy, X.data_ptr(), ld, _type(X), T, D, mean.data_ptr(), rstd.data_ptr(), _vector(weight, D),
                              dX.data_ptr(), D, dw.data_ptr(), db.data_ptr(), 0 if ws is None else ws.data_ptr(), n, _current_stream(X)), "bsp_layer_norm_grad")
    return dX, dw, db


_norm_sizes = {}


def _norm_bytes(T, D):
    n = _norm_sizes.get((T, D))
    if n is None:
        n = ctypes.c_int64(0)
        _check(load_library().bsp_layer_norm_grad_workspace(T, D, n), "bsp_layer_norm_grad_workspace")
        if len(_norm_sizes) > 4096:
            _norm_sizes.clear()
        n = _norm_sizes[(T, D)] = n.value
    return n
