"""Low-rank adapters of many requests beside an 8-bit layer, on torch tensors: what a layer's ``fc`` and ``grad_input`` take as ``adapters`` and
``requests``, and the adapters' own gradients.  Calls as those of the layers: asynchronous on the tensors' current stream, or on
``stream``, recording nothing for autograd."""
from __future__ import annotations

import ctypes
import struct

from .binding import BSP_BF16, _check, _current_stream, bsp_f8_adapters, bsp_f8_requests, load_library
from .f8 import _NO_CODES, BspCodes, _call, _on, _on_stream, _rows, _type, _unrecorded

_ADAPTERS_GRAD = 21
_pack17 = struct.Struct("=17q").pack


class BspRequests:
    """The rows of a batch by their adapters: ``which`` [T] (a tensor of int32 or int64, or anything that makes one) holds each row's slot in a
    set of ``slots`` adapters; any other number is a row without one.  Made once for a batch, for all of its layers; ``update`` takes another
    batch of as many rows into the same memory, as a captured graph needs it."""

    def __init__(self, which, slots: int, device=None):
        import torch
        which = torch.as_tensor(which)
        self.device = torch.device(device) if device is not None else which.device if which.is_cuda else torch.device("cuda:0")
        assert which.dim() == 1, "a slot a row"
        self.T, self.N = which.shape[0], slots
        n = ctypes.c_int64(0)
        _check(load_library().bsp_f8_requests_size(self.T, self.N, n), "bsp_f8_requests_size")
        self.plan = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        self.device, self._index = self.plan.device, self.plan.get_device()
        self.struct = bsp_f8_requests(self.T, self.N, self.plan.data_ptr())
        self._address = ctypes.addressof(self.struct)
        self.update(which)

    def update(self, which, stream=None) -> None:
        import torch
        if stream is not None:
            return _on_stream(stream, self.plan, self.update, which)
        which = torch.as_tensor(which)
        assert which.shape == (self.T,), "a slot a row, %d of them" % self.T
        assert which.dtype in (torch.int32, torch.int64), "slots as int32 or int64"
        which = which.to(self.device).contiguous()
        _check(load_library().bsp_f8_requests_plan(self.struct, which.data_ptr() or None, which.element_size(), _current_stream(self.plan)), "bsp_f8_requests_plan")


class BspAdapters:
    """``slots`` low-rank adapters (at most 1024) of up to ``rank`` (at most 128) for layers of ``I`` inputs and ``O`` outputs: a row x of slot n gets
    scale[n] B[n] (A[n] x) beside the layer's own result.  Held as bf16, in both directions; slots that were not set add nothing."""

    def __init__(self, slots: int, rank: int, I: int, O: int, device="cuda:0"):
        import torch
        lib = load_library()
        na, nb = ctypes.c_int64(0), ctypes.c_int64(0)
        assert 1 <= slots <= 1024, "1 to 1024 slots"
        _check(lib.bsp_f8_adapters_size(rank, I, O, na, nb), "bsp_f8_adapters_size")
        self.N, self.R, self.I, self.O = slots, rank, I, O
        self.device = torch.device(device)
        self._held = [torch.zeros(slots * n.value, dtype=torch.bfloat16, device=self.device) for n in (na, na, nb, nb)]
        self.scale = torch.zeros(slots, dtype=torch.float32, device=self.device)
        self.device, self._index = self.scale.device, self.scale.get_device()
        self.struct = bsp_f8_adapters(slots, rank, I, O, *(t.data_ptr() for t in self._held), self.scale.data_ptr())
        self._address = ctypes.addressof(self.struct)
        self._workspace = {}

    def set(self, slot: int, A, B, scale: float = 1.0, stream=None) -> None:
        """Slot ``slot`` from A [r][I] and B [O][r], r <= rank (tensors on this device in fp32 or bf16, rows contiguous), rounded to bf16: a new
        adapter, or the weights that a step of an optimiser has left."""
        if stream is not None:
            return _on_stream(stream, self.scale, self.set, slot, A, B, scale)
        A, B = A.detach(), B.detach()
        _on(self.scale, A, B)
        r, I, lda = _rows(A)
        O, r2, ldb = _rows(B)
        assert (I, O) == (self.I, self.O) and r == r2 and A.dtype == B.dtype, "A [r][%d] and B [%d][r] of one type" % (self.I, self.O)
        assert 0 <= slot < self.N and 1 <= r <= self.R, "a slot of %d and a rank of at most %d" % (self.N, self.R)
        _check(load_library().bsp_f8_adapters_set(self.struct, slot, r, A.data_ptr(), lda, B.data_ptr(), ldb, _type(A), scale, _current_stream(A)), "bsp_f8_adapters_set")

    def clear(self, slot: int, stream=None) -> None:
        """Slot ``slot`` adds nothing from here on."""
        if stream is not None:
            return _on_stream(stream, self.scale, self.clear, slot)
        assert 0 <= slot < self.N, "a slot of %d" % self.N
        _check(load_library().bsp_f8_adapters_set(self.struct, slot, 0, None, 0, None, 0, BSP_BF16, 0.0, _current_stream(self.scale)), "bsp_f8_adapters_set")

    def grad(self, dY, X, requests: BspRequests, stream=None):
        """(dA [slots][rank][I], dB [slots][O][rank]) in float from the gradient of the layer's result (bf16 [T][O]) and the layer's input: its
        checkpoint, or bf16 values [T][I].  Zeros for adapters without rows."""
        import torch
        if stream is not None:
            return _on_stream(stream, self.scale, self.grad, dY, X, requests)
        codes = type(X) is BspCodes
        if dY.requires_grad or (not codes and X.requires_grad):
            _unrecorded(3)
        T, O, ldy = _rows(dY)
        assert dY.dtype == torch.bfloat16 and O == self.O
        if codes:
            assert (X.T, X.K) == (T, self.I)
            _on(self.scale, X.buffer)
            words, x, ldx = X.words, 0, 0
        else:
            T2, I, ldx = _rows(X)
            assert (T2, I) == (T, self.I) and X.dtype == torch.bfloat16
            _on(self.scale, X)
            words, x = _NO_CODES, X.data_ptr()
        assert (requests.T, requests.N) == (T, self.N), "requests of %d rows and %d slots" % (T, self.N)
        _on(self.scale, dY, requests.plan)
        dA = self.scale.new_empty((self.N, self.R, self.I))
        dB = self.scale.new_empty((self.N, self.O, self.R))
        n = self._workspace.get(T)
        if n is None:
            n = ctypes.c_int64(0)
            _check(load_library().bsp_f8_adapters_grad_workspace(self.struct, T, n), "bsp_f8_adapters_grad_workspace")
            if len(self._workspace) > 4096:
                self._workspace.clear()
            n = self._workspace[T] = n.value
        ws = self.scale.new_empty(n, dtype=torch.uint8) if n else None
        _call(_ADAPTERS_GRAD, _pack17(self._address, dY.data_ptr(), ldy, *words, x, ldx, T, requests._address, dA.data_ptr(), dB.data_ptr(),
                                      0 if ws is None else ws.data_ptr(), n, _current_stream(dY)), "bsp_f8_adapters_grad")
        return dA, dB
