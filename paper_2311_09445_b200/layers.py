"""ctypes binding of a layer's operators (include/pearl_layers.h): argument checks and marshalling only.

On the handle of the row operators: the norm before a layer and the dropout behind it, with their gradients, and a whole
expert layer for the few rows of a policy's step.  Every step runs in the library's CUDA kernels; there is no CPU path.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import routing as _routing
from .binding import PearlError
from .routing import _F32, _I32, _TYPES, _i, _room, _u32, _u64, _vp, RowRouter

MAX_WIDTH, MAX_FEW, MAX_INNER = 65536, 64, 65536
_f64 = C.c_double
# name -> (restype, argtypes); every symbol include/pearl_layers.h declares
SIGNATURES = {
    "pearl_layer_norm": (_i, [_vp, _u32, _u32, _u32, _vp, _u64, _u32, _vp, _vp, _f64, _vp, _u64, _vp, _vp]),
    "pearl_layer_norm_grad": (_i, [_vp, _u32, _u32, _u32, _vp, _u64, _vp, _u64, _vp, _vp, _u32, _vp, _vp, _u64, _vp, _vp, _vp, _u64]),
    "pearl_layer_norm_grad_work_bytes": (_u64, [_u32, _u32]),
    "pearl_layer_dropout": (_i, [_vp, _u32, _u32, _u32, _vp, _u64, _vp, _u64, _f64, _u64, _u64, _vp, _vp, _u64]),
    "pearl_layer_experts": (_i, [_vp, _u32, _u32, _u32, _u32, _u32, _u32, _u32, _vp, _u64, _vp, _i, _vp, _vp, _vp, _vp, _vp, _u64, _vp, _u64]),
    "pearl_layer_experts_work_bytes": (_u64, [_u32, _u32, _u32, _u32, _u32]),
}

_lib = None


def load_library():
    """The library of the row operators, with the signatures of a layer's declared."""
    global _lib
    if _lib is None:
        lib = _routing.load_library()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _word(value: int, what: str) -> int:
    if not 0 <= value < 1 << 64:
        raise ValueError("%s must be a number of 64 bits" % what)
    return value


class RowLayers(RowRouter):
    """The row operators and those of a layer on one GPU: calls enqueue on `stream` (default: the current torch stream at
    construction).

    All arrays are CUDA tensors of the handle's device that the caller owns, outputs and workspaces included.  Matrices of rows
    may be views whose rows lie apart; the elements of a row, and everything else, are contiguous.  A workspace serves one call
    at a time: streams and captured graphs that may run side by side have one each."""

    def __init__(self, device=None, stream=None):
        super().__init__(device, stream)
        load_library()

    def _rows_like(self, t: torch.Tensor, what: str, T: int, D: int, like: torch.Tensor, name: str):
        """(address, distance of the rows) of a matrix of another one's shape and type."""
        p, rows, cols, ld = self._matrix(t, what)
        if rows != T or cols != D or t.dtype is not like.dtype:
            raise ValueError("%s must have the shape and type of %s" % (what, name))
        return p, ld

    def _params(self, like: torch.Tensor, D: int, **arrays):
        """(type, addresses) of a norm's parameters, which are binary32 or of the rows' type."""
        dtype = None
        for what, t in arrays.items():
            if t is None:
                continue
            if t.dtype is not _F32 and t.dtype is not like.dtype:
                raise ValueError("%s must be float32 or of the rows' type" % what)
            if dtype is not None and t.dtype is not dtype:
                raise ValueError("the norm's parameters must have one type")
            dtype = t.dtype
        return _TYPES[dtype] if dtype is not None else 0, [None if t is None else self._dense(t, what, dtype, D) for what, t in arrays.items()]

    def _scratch(self, work: torch.Tensor):
        if work.dtype is not torch.uint8 or work.get_device() != self._ordinal or not work.is_contiguous():
            raise ValueError("work must be a contiguous uint8 tensor on %s" % self.device)
        return work.data_ptr(), work.numel()

    def _room_for(self, size: int) -> torch.Tensor:
        """A zeroed workspace, made on the handle's stream."""
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            return torch.zeros(size, dtype=torch.uint8, device=self.device)

    # ---- layer norm ------------------------------------------------------------------------------
    def layer_norm(self, x, y, gamma=None, beta=None, eps: float = 1e-5, mean=None, rstd=None) -> None:
        """y = (x - mean) * rstd * gamma + beta for each row of x [T, D]; gamma, beta [D] (float32 or of x's type), mean, rstd [T]
        (float32, outputs) may each be None."""
        p, T, D, ld = self._matrix(x, "x")
        q, ld_y = self._rows_like(y, "y", T, D, x, "x")
        ptype, (g, b) = self._params(x, D, gamma=gamma, beta=beta)
        rc = self._lib.pearl_layer_norm(self._h, T, D, self._type(x, "x"), p, ld, ptype, g, b, eps, q, ld_y,
                                        None if mean is None else self._dense(mean, "mean", _F32, T),
                                        None if rstd is None else self._dense(rstd, "rstd", _F32, T))
        if rc != 0:
            raise PearlError(rc, "pearl_layer_norm")

    def layer_norm_grad_work(self, rows: int, width: int) -> torch.Tensor:
        """A workspace for layer_norm_grad of up to `rows` rows of `width` elements."""
        return self._room_for(self._work_bytes("pearl_layer_norm_grad_work_bytes", rows, width))

    def _work_bytes(self, call: str, *sizes: int) -> int:
        for n in sizes:
            _room(n)
        size = int(getattr(self._lib, call)(*sizes))
        if size == 0:
            raise ValueError("a size is out of range")
        return size

    def layer_norm_grad(self, dy, x, mean, rstd, gamma=None, dx=None, dgamma=None, dbeta=None, work=None) -> None:
        """dy, x [T, D], what layer_norm returned -> dx [T, D], dgamma, dbeta [D] (float32; they need `work`); each may be None."""
        p, T, D, ld = self._matrix(dy, "dy")
        q, ld_x = self._rows_like(x, "x", T, D, dy, "dy")
        r, ld_dx = (None, 0) if dx is None else self._rows_like(dx, "dx", T, D, dy, "dy")
        ptype, (g,) = self._params(x, D, gamma=gamma)
        if (dgamma is not None or dbeta is not None) and work is None:
            raise ValueError("dgamma and dbeta need work")
        scratch, size = (None, 0) if work is None else self._scratch(work)
        rc = self._lib.pearl_layer_norm_grad(self._h, T, D, self._type(dy, "dy"), p, ld, q, ld_x, self._dense(mean, "mean", _F32, T),
                                             self._dense(rstd, "rstd", _F32, T), ptype, g, r, ld_dx,
                                             None if dgamma is None else self._dense(dgamma, "dgamma", _F32, D),
                                             None if dbeta is None else self._dense(dbeta, "dbeta", _F32, D), scratch, size)
        if rc != 0:
            raise PearlError(rc, "pearl_layer_norm_grad")

    # ---- dropout ---------------------------------------------------------------------------------
    def dropout(self, x, y, p: float, seed: int, call: int = 0, residual=None, calls=None) -> None:
        """y = (keep ? x / (1 - p) : 0) + residual; the mask is a function of seed, call, row and column alone.  calls: an int64 tensor of
        one element that is added to `call` when the kernel runs.  y may be x or residual."""
        a, T, D, ld = self._matrix(x, "x")
        b, ld_y = self._rows_like(y, "y", T, D, x, "x")
        r, ld_r = (None, 0) if residual is None else self._rows_like(residual, "residual", T, D, x, "x")
        rc = self._lib.pearl_layer_dropout(self._h, T, D, self._type(x, "x"), a, ld, r, ld_r, p, _word(seed, "seed"), _word(call, "call"),
                                           None if calls is None else self._dense(calls, "calls", torch.int64, 1), b, ld_y)
        if rc != 0:
            raise PearlError(rc, "pearl_layer_dropout")

    def dropout_grad(self, dy, dx, p: float, seed: int, call: int = 0, calls=None) -> None:
        """dx = keep ? dy / (1 - p) : 0, with the mask of dropout's call (the residual's gradient is dy itself)."""
        self.dropout(dy, dx, p, seed, call, None, calls)

    # ---- a whole expert layer for a few rows -----------------------------------------------------
    def expert_layer_work(self, rows: int, width: int, hidden: int, experts: int, k: int) -> torch.Tensor:
        """A workspace for expert_layer of up to these sizes."""
        return self._room_for(self._work_bytes("pearl_layer_experts_work_bytes", rows, width, hidden, experts, k))

    def _weights(self, t: torch.Tensor, what: str, shape, like: torch.Tensor) -> int:
        if tuple(t.shape) != shape or t.dtype is not like.dtype or t.get_device() != self._ordinal or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor on %s of the type of x" % (what, list(shape), self.device))
        return t.data_ptr()

    def expert_layer(self, x, router, up, down, y, w, ids, work, gated: bool = True, over_chosen: bool = True) -> None:
        """y[t] = sum over j of w[t, j] * down[e] act(up[e] x[t]), e = ids[t, j], for up to 64 rows x [T, D].  router [E, D] chooses them and
        their weights (outputs w [T, k], ids [T, k]); None: w and ids are given.  up [E, 2H, D] (H gates, then H values: silu(gate) *
        value), not gated [E, H, D] (relu); down [E, D, H]."""
        p, T, D, ld = self._matrix(x, "x")
        q, ld_y = self._rows_like(y, "y", T, D, x, "x")
        if down.dim() != 3 or ids.dim() != 2 or ids.shape[0] != T:
            raise ValueError("down must be [E, %d, H] and ids [%d, k]" % (D, T))
        E, H, k = down.shape[0], down.shape[2], ids.shape[1]
        _room(E | H | k)
        scratch, size = self._scratch(work)
        rc = self._lib.pearl_layer_experts(self._h, T, D, H, E, k, self._type(x, "x"), 0 if gated else 1, p, ld,
                                           None if router is None else self._weights(router, "router", (E, D), x), 1 if over_chosen else 0,
                                           self._weights(up, "up", (E, 2 * H if gated else H, D), x),
                                           self._weights(down, "down", (E, D, H), x), self._dense(w, "w", _F32, T * k),
                                           self._dense(ids, "ids", _I32, T * k), q, ld_y, scratch, size)
        if rc != 0:
            raise PearlError(rc, "pearl_layer_experts")
