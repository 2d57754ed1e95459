"""FC layers in 8-bit floating point, the 8-bit checkpoints of their inputs, their gradients, and layer norm, on torch
tensors.  Marshalling only: every call launches on the current stream (or ``stream``) of its tensors' device and returns
before it is done; tensors that it makes come from torch's allocator on that stream."""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np

from .binding import (BSP_BF16, BSP_E4M3, BSP_E5M2, BSP_F32, _check, _current_stream, _np_ptr, bsp_codes, bsp_weights_f8,
                      load_library)

CODES = {"e4m3": BSP_E4M3, "e5m2": BSP_E5M2}


def _type(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BSP_BF16
    assert t.dtype == torch.float32, t.dtype
    return BSP_F32


def _rows(t):
    """(T, K, elements from row to row) of a matrix whose rows are contiguous; rows may lie any distance apart."""
    T, K = t.shape
    assert t.is_cuda and (t.stride(1) == 1 or K == 1 or T == 0)
    return T, K, t.stride(0) if T > 1 else K


def _blocks(n: int) -> int:
    return -(-n // 128)


def _on(t, *others):
    assert all(o is None or o.device == t.device for o in others)


class BspCodes:
    """A matrix [T][K] held as 8-bit floating-point codes with a power-of-two scale for each row's 128 columns: the form in
    which a layer's input is kept for the backward pass.  ``codes`` [T][128 ceil(K/128)] and ``scale``
    [ceil(K/128)][16 ceil(T/16)] (exponent + 127) are uint8 tensors; ``kind`` is "e4m3" or "e5m2"."""

    def __init__(self, T: int, K: int, kind: str = "e4m3", device="cuda:0"):
        import torch
        self.T, self.K, self.kind = T, K, kind
        nb = _blocks(K)
        self.codes = torch.empty((T, nb * 128), dtype=torch.uint8, device=device)
        self.scale = torch.empty((nb, (T + 15) // 16 * 16), dtype=torch.uint8, device=device)
        self.struct = bsp_codes(T, K, CODES[kind], self.codes.data_ptr() or None, self.scale.data_ptr() or None)

    def load(self, dtype=None, out=None, stream=None):
        """The values, as bf16 (or torch.float32)."""
        import torch
        if out is None:
            out = torch.empty((self.T, self.K), dtype=dtype or torch.bfloat16, device=self.codes.device)
        T, K, ld = _rows(out)
        assert (T, K) == (self.T, self.K)
        _on(self.codes, out)
        st = _current_stream(out) if stream is None else stream
        _check(load_library().bsp_f8_load(self.struct, out.data_ptr(), _type(out), ld, st), "bsp_f8_load")
        return out


def save8(X, kind: str = "e4m3", out: Optional[BspCodes] = None, stream=None) -> BspCodes:
    """The 8-bit checkpoint of X (torch tensor [T][K], fp32 or bf16, rows contiguous)."""
    T, K, ld = _rows(X)
    if out is None:
        out = BspCodes(T, K, kind, X.device)
    assert (out.T, out.K) == (T, K)
    _on(X, out.codes)
    st = _current_stream(X) if stream is None else stream
    _check(load_library().bsp_f8_save(X.data_ptr(), _type(X), ld, out.struct, st), "bsp_f8_save")
    return out


class BspLayerF8:
    """An FC layer Y = X W^t + b in 8-bit floating point, resident on a GPU: W [O][I] (numpy, or a torch tensor in fp32 or
    bf16) under a mask ``gamma`` [ceil(O/128)][ceil(I/128)] (1 = kept; None keeps all), bias float or None.  Each kept block
    of 128 x 128 weights is held as e4m3 codes with one power-of-two scale, in both directions: by rows for the layer,
    by columns for the gradient of its input."""

    def __init__(self, W, gamma=None, bias=None, device="cuda:0"):
        import torch
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
        # (one block more than is kept, so that an empty layer has addresses)
        self.payload, self.payload_t = (torch.empty((max(self.nnzb, 1), 128, 128), dtype=torch.uint8, device=self.device) for _ in range(2))
        self.scale, self.scale_t = (torch.empty(max(self.nnzb, 1), dtype=torch.uint8, device=self.device) for _ in range(2))
        self.struct = bsp_weights_f8(O, I, self.nnzb, *(t.data_ptr() for t in self.d_index), self.payload.data_ptr(),
                                     self.scale.data_ptr(), self.payload_t.data_ptr(), self.scale_t.data_ptr())
        self.d_bias = None
        if bias is not None:
            b = torch.as_tensor(bias, dtype=torch.float32).to(self.device).contiguous()
            assert b.shape == (O,)
            self.d_bias = b
        self.update(W)

    def update(self, W, stream=None) -> None:
        """Take new weights (same shape, same mask), as after a step of an optimiser."""
        import torch
        if not isinstance(W, torch.Tensor):
            W = torch.from_numpy(np.ascontiguousarray(W, dtype=np.float32))
        W = W.to(self.device)
        O, I, ld = _rows(W)
        assert (O, I) == (self.O, self.I)
        st = _current_stream(W) if stream is None else stream
        _check(load_library().bsp_f8_pack(self.struct, W.data_ptr(), _type(W), ld, st), "bsp_f8_pack")

    def _multiply(self, transposed, X, code, bias, residual, relu, gate, dtype, out, stream):
        import torch
        lib = load_library()
        codes = isinstance(X, BspCodes)
        if codes:
            T, K, at = X.T, X.K, X.codes
        else:
            T, K, ld = _rows(X)
            at = X
        width = self.I if transposed else self.O
        assert K == (self.O if transposed else self.I)
        if out is None:
            out = torch.empty((T, width), dtype=dtype or (torch.bfloat16 if codes else X.dtype), device=at.device)
        assert out.shape == (T, width) and out.is_contiguous()
        _on(self.payload, at, out, residual, None if gate is None else gate.codes)
        if residual is not None:
            assert residual.shape == out.shape and residual.dtype == out.dtype and residual.is_contiguous()
        st = _current_stream(out) if stream is None else stream
        rest = (None if bias is None else bias.data_ptr(), None if residual is None else residual.data_ptr(),
                1 if relu else 0, None if gate is None else gate.struct, out.data_ptr() or None, _type(out))
        if codes:
            _check(lib.bsp_f8_fc(self.struct, transposed, X.struct, *rest, st), "bsp_f8_fc")
            return out
        n = ctypes.c_int64(0)
        if not (T <= 16 and T * (_blocks(K) * 129 + 16) <= 73728 and (X.data_ptr() | ld * X.element_size() | K * X.element_size()) % 16 == 0):
            _check(lib.bsp_f8_fc_workspace(self.struct, transposed, T, n), "bsp_f8_fc_workspace")
        ws = torch.empty(n.value, dtype=torch.uint8, device=out.device) if n.value else None
        _check(lib.bsp_f8_fc_values(self.struct, transposed, X.data_ptr() or None, _type(X), ld, T, CODES[code], *rest,
                                    None if ws is None else ws.data_ptr(), n.value, st), "bsp_f8_fc_values")
        if ws is not None and stream is not None:
            ws.record_stream(torch.cuda.ExternalStream(st, device=ws.device))
        return out

    def fc(self, X, relu=False, residual=None, dtype=None, out=None, stream=None):
        """Y [T][O] = act(X W^t + b + residual) for X [T][I]: a torch tensor (fp32 or bf16, brought to e4m3 codes within the
        call; Y has its type unless ``dtype`` says otherwise) or a BspCodes (Y is bf16 unless ``dtype`` says otherwise)."""
        return self._multiply(0, X, "e4m3", self.d_bias, residual, relu, None, dtype, out, stream)

    def grad_input(self, dY, relu_of: Optional[BspCodes] = None, code: str = "e5m2", dtype=None, out=None, stream=None):
        """dX [T][I] = dY W for dY [T][O] (brought to codes of type ``code`` within the call, or a BspCodes).  ``relu_of``: the
        checkpoint of this layer's input, where that is a ReLU's output; the result is then the gradient of what went
        into the ReLU."""
        return self._multiply(1, dY, code, None, None, False, relu_of, dtype, out, stream)

    def grad_weight(self, dY, X: BspCodes, bias: bool = True, out=None, stream=None):
        """(dW, db) from dY (bf16 [T][O]) and the checkpoint of the layer's input: dW float [O][I], zero where the mask is; db
        float [O], or None."""
        import torch
        lib = load_library()
        T, O, ld = _rows(dY)
        assert dY.dtype == torch.bfloat16 and (T, O) == (X.T, self.O)
        _on(self.payload, dY, X.codes, out)
        if out is None:
            out = torch.empty((self.O, self.I), dtype=torch.float32, device=dY.device)
        assert out.shape == (self.O, self.I) and out.dtype == torch.float32 and out.is_contiguous()
        db = torch.empty(self.O, dtype=torch.float32, device=dY.device) if bias else None
        n = ctypes.c_int64(0)
        _check(lib.bsp_f8_fc_grad_workspace(self.struct, T, n), "bsp_f8_fc_grad_workspace")
        ws = torch.empty(n.value, dtype=torch.uint8, device=dY.device)
        st = _current_stream(dY) if stream is None else stream
        _check(lib.bsp_f8_fc_grad(self.struct, dY.data_ptr() or None, ld, X.struct, out.data_ptr(),
                                  None if db is None else db.data_ptr(), ws.data_ptr(), n.value, st), "bsp_f8_fc_grad")
        if stream is not None:
            ws.record_stream(torch.cuda.ExternalStream(st, device=ws.device))
        return out, db


def _vector(t, D):
    import torch
    if t is not None:
        assert t.is_cuda and t.dtype == torch.float32 and t.shape == (D,) and t.is_contiguous()
    return None if t is None else t.data_ptr()


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5, code: Optional[str] = None, stream=None):
    """(Y, mean, rstd) of X [T][D] (fp32 or bf16) over its last axis; ``weight`` and ``bias`` are float [D] or None.  With ``code``
    ("e4m3", "e5m2") Y is a BspCodes, the form in which a BspLayerF8 reads it."""
    import torch
    T, D, ld = _rows(X)
    _on(X, weight, bias)
    mean = torch.empty((2, T), dtype=torch.float32, device=X.device)
    rstd, mean = mean[1], mean[0]
    Y = torch.empty((T, D), dtype=X.dtype, device=X.device) if code is None else BspCodes(T, D, code, X.device)
    st = _current_stream(X) if stream is None else stream
    _check(load_library().bsp_layer_norm(X.data_ptr() or None, _type(X), ld, T, D, _vector(weight, D), _vector(bias, D), eps,
                                         (Y.data_ptr() or None) if code is None else None, D, None if code is None else Y.struct,
                                         mean.data_ptr() or None, rstd.data_ptr() or None, st), "bsp_layer_norm")
    return Y, mean, rstd


def layer_norm_grad(dY, X, mean, rstd, weight=None, stream=None):
    """(dX, dweight, dbias) from the gradient of Y, the input and what ``layer_norm`` returned with it."""
    import torch
    lib = load_library()
    T, D, ld = _rows(X)
    T2, D2, ld_dy = _rows(dY)
    assert (T2, D2) == (T, D) and dY.dtype == X.dtype and mean.shape == rstd.shape == (T,)
    assert mean.dtype == rstd.dtype == torch.float32 and (T < 2 or mean.stride(0) == rstd.stride(0) == 1)
    _on(X, dY, mean, rstd, weight)
    dX = torch.empty((T, D), dtype=X.dtype, device=X.device)
    dw, db = torch.empty((2, D), dtype=torch.float32, device=X.device).unbind(0)
    n = ctypes.c_int64(0)
    _check(lib.bsp_layer_norm_grad_workspace(T, D, n), "bsp_layer_norm_grad_workspace")
    ws = torch.empty(n.value, dtype=torch.uint8, device=X.device)
    st = _current_stream(X) if stream is None else stream
    _check(lib.bsp_layer_norm_grad(dY.data_ptr() or None, ld_dy, X.data_ptr() or None, ld, _type(X), T, D, mean.data_ptr() or None,
                                   rstd.data_ptr() or None, _vector(weight, D), dX.data_ptr() or None, D, dw.data_ptr(), db.data_ptr(),
                                   ws.data_ptr(), n.value, st), "bsp_layer_norm_grad")
    if stream is not None:
        ws.record_stream(torch.cuda.ExternalStream(st, device=ws.device))
    return dX, dw, db
