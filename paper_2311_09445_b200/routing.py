"""ctypes binding of the row operators (include/pearl_rows.h): argument checks and marshalling only.

Beside the replay buffer's "draw, weigh, gather" these choose, weigh and move rows of a batch: a router with the sort
of rows by expert and the way back, with their gradients, and a beam search's selection with the move of the beams'
states.  Every step runs in the library's CUDA kernels; there is no CPU path.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from . import binding as _binding
from .binding import PearlError

ST_BAD_INDEX, ST_INTERNAL, ST_BAD_SCORE = 1, 16, 64
MAX_EXPERTS, MAX_ROW_BYTES, MAX_CHOICES, MAX_BEAMS, MAX_BEST, MAX_VOCAB = 1024, 1 << 23, 32, 32, 64, 1 << 24


class _States(C.Structure):
    _fields_ = [("block_pitch", C.c_uint64), ("state_pitch", C.c_uint64), ("piece_pitch", C.c_uint64)]


_vp, _u32, _u64, _i = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int
# name -> (restype, argtypes); every symbol include/pearl_rows.h declares
SIGNATURES = {
    "pearl_rows_slab_bytes": (_u64, []),
    "pearl_rows_create": (_i, [C.POINTER(_vp), _i, _vp, _vp, _u64]),
    "pearl_rows_destroy": (_i, [_vp]),
    "pearl_rows_route": (_i, [_vp, _u32, _u32, _u32, _u32, _vp, _u64, _i, _vp, _vp]),
    "pearl_rows_route_grad": (_i, [_vp, _u32, _u32, _u32, _u32, _vp, _u64, _i, _vp, _vp, _vp, _vp, _u64]),
    "pearl_rows_sort": (_i, [_vp, _u32, _u32, _vp, _vp, _vp, _vp]),
    "pearl_rows_dispatch": (_i, [_vp, _u32, _u32, _u32, _vp, _u64, _vp, _u32, _vp]),
    "pearl_rows_combine": (_i, [_vp, _u32, _u32, _u32, _u32, _vp, _u32, _vp, _vp, _vp, _u64]),
    "pearl_rows_combine_grad": (_i, [_vp, _u32, _u32, _u32, _u32, _vp, _u64, _vp, _u32, _vp, _vp, _vp, _vp]),
    "pearl_rows_beam_select": (_i, [_vp, _u32, _u32, _u32, _u32, _u32, _vp, _u64, _vp, _vp, C.c_int32, _vp, _vp, _vp]),
    "pearl_rows_beam_reorder": (_i, [_vp, _u32, _u32, _u32, _u32, _u64, _vp, _vp, C.POINTER(_States), _vp, C.POINTER(_States)]),
    "pearl_rows_sync": (_i, [_vp, C.POINTER(_u32)]),
    "pearl_rows_kernel_launches": (_u64, [_vp]),
}
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_I32, _F32 = torch.int32, torch.float32

_lib = None


def load_library():
    """The library of the replay buffer, with the signatures of its row operators declared."""
    global _lib
    if _lib is None:
        lib = _binding.load_library()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _room(counts: int) -> None:
    """counts: sizes that go to the library as 32-bit numbers, OR'ed together.  ctypes would hand on the low bits of a larger one."""
    if counts >> 32:
        raise ValueError("a size is negative or above 2^32 - 1")


def _pieces(shape, stride):
    """A state's axes (those from the fourth on) as (pieces, elements of a piece, distance of pieces)."""
    width, i = 1, len(shape)
    while i > 3 and (shape[i - 1] == 1 or stride[i - 1] == width):
        i -= 1
        width *= shape[i]
    pieces, pitch = 1, width
    while i > 3:
        i -= 1
        if shape[i] == 1:
            continue
        if pieces == 1:
            pitch = stride[i]
        elif stride[i] != pitch * pieces:
            raise ValueError("a state must be equally distant pieces of contiguous elements")
        pieces *= shape[i]
    return pieces, width, pitch


def _distances(shape, stride):
    """The distance of a block from the next one, and of a state."""
    blocks, G, W = shape[:3]
    if G > 1 and W > 1 and stride[1] != W * stride[2]:
        raise ValueError("states must lie equally far apart")
    return stride[0] if blocks > 1 else 0, stride[2] if W > 1 else (stride[1] if G > 1 else 0)


@functools.lru_cache(maxsize=256)
def _move(shape, stride, stride_out, size):
    """pearl_rows_beam_reorder's arguments that follow from shapes and strides alone (a growing cache's for each of its lengths)."""
    pieces, width, pitch = _pieces(shape, stride)
    pieces_out, width_out, pitch_out = _pieces(shape, stride_out)
    if pieces != pieces_out:
        # one of the two is more contiguous than the other: cut it into the other's pieces
        if pieces == 1:
            pieces, width, pitch = pieces_out, width_out, width_out
        elif pieces_out == 1:
            pitch_out = width
        else:
            raise ValueError("states and out must be cut into the same pieces")
    _room(shape[0] | shape[1] | shape[2] | pieces)
    src, dst = (_States(block * size, state * size, p * size) for (block, state), p in
                ((_distances(shape, stride), pitch), (_distances(shape, stride_out), pitch_out)))
    return pieces, width * size, C.byref(src), C.byref(dst)


class RowRouter:
    """The row operators on one GPU: calls enqueue on `stream` (default: the current torch stream at construction).

    All arrays are CUDA tensors of the handle's device that the caller owns, outputs included.  `logits` and matrices of rows may
    be views whose rows lie apart; the elements of a row, and everything else, are contiguous."""

    def __init__(self, device: Optional[torch.device] = None, stream: Optional[torch.cuda.Stream] = None):
        self._h = None
        lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("RowRouter needs a CUDA device; there is no CPU path")
        if device is None:
            device = stream.device if stream is not None else "cuda:%d" % torch.cuda.current_device()
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("RowRouter runs on a CUDA device")
        self.device = torch.device("cuda", device.index if device.index is not None else torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        if self.stream.device_index != self.device.index:
            raise ValueError("the stream belongs to another device")
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            self._slab = torch.empty(int(lib.pearl_rows_slab_bytes()), dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        rc = lib.pearl_rows_create(C.byref(h), self.device.index, C.c_void_p(self.stream.cuda_stream),
                                   C.c_void_p(self._slab.data_ptr()), self._slab.numel())
        if rc != 0:
            raise PearlError(rc, "pearl_rows_create")
        self._h = h
        self._lib = lib
        self._ordinal = self.device.index

    # ---- argument checks -------------------------------------------------------------------------
    # (a device is compared by its number, -1 for a tensor that is not on a GPU: half the time of comparing torch.device objects,
    # and these checks are a good part of what a small call costs)
    def _dense(self, t: torch.Tensor, what: str, dtype, count: int) -> int:
        if t.dtype is not dtype or t.numel() != count or t.get_device() != self._ordinal or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor of %d elements on %s" % (what, dtype, count, self.device))
        return t.data_ptr()

    def _matrix(self, t: torch.Tensor, what: str):
        """(address, rows, row length, distance of the rows in elements) of a 2-D tensor."""
        if t.dim() != 2 or t.get_device() != self._ordinal:
            raise ValueError("%s must be a 2-D tensor on %s with contiguous rows" % (what, self.device))
        rows, cols = t.shape
        _room(rows | cols)
        if t.is_contiguous():
            return t.data_ptr(), rows, cols, cols
        ld, step = t.stride()
        if cols > 1 and step != 1:
            raise ValueError("%s must be a 2-D tensor on %s with contiguous rows" % (what, self.device))
        ld = ld if rows > 1 else cols
        if ld < cols:
            raise ValueError("the rows of %s overlap" % what)
        return t.data_ptr(), rows, cols, ld

    @staticmethod
    def _type(t: torch.Tensor, what: str) -> int:
        code = _TYPES.get(t.dtype)
        if code is None:
            raise ValueError("%s must be float32, float16 or bfloat16" % what)
        return code

    # ---- expert layers ---------------------------------------------------------------------------
    def route(self, logits, w, ids, over_chosen: bool = False) -> None:
        """logits [T, E] -> w [T, k] (float32), ids [T, k] (int32): the k best experts of a row and their softmax weights."""
        p, T, E, ld = self._matrix(logits, "logits")
        if ids.dim() != 2 or ids.shape[0] != T:
            raise ValueError("ids must be [%d, k]" % T)
        k = ids.shape[1]
        _room(k)
        rc = self._lib.pearl_rows_route(self._h, T, E, k, self._type(logits, "logits"), p, ld, 1 if over_chosen else 0,
                                        self._dense(w, "w", _F32, T * k), self._dense(ids, "ids", _I32, T * k))
        if rc != 0:
            raise PearlError(rc, "pearl_rows_route")

    def route_grad(self, logits, w, ids, dw, dlogits, over_chosen: bool = False) -> None:
        """dw [T, k] -> dlogits [T, E]; logits may be None if over_chosen."""
        d, T, E, ld_d = self._matrix(dlogits, "dlogits")
        p, ld = None, E
        if logits is not None:
            p, rows, cols, ld = self._matrix(logits, "logits")
            if (rows, cols) != (T, E) or logits.dtype is not dlogits.dtype:
                raise ValueError("logits and dlogits must have one shape and type")
        if ids.dim() != 2 or ids.shape[0] != T:
            raise ValueError("ids must be [%d, k]" % T)
        _room(ids.shape[1])
        n = T * ids.shape[1]
        rc = self._lib.pearl_rows_route_grad(self._h, T, E, ids.shape[1], self._type(dlogits, "dlogits"), p, ld,
                                             1 if over_chosen else 0, self._dense(w, "w", _F32, n),
                                             self._dense(ids, "ids", _I32, n), self._dense(dw, "dw", _F32, n), d, ld_d)
        if rc != 0:
            raise PearlError(rc, "pearl_rows_route_grad")

    def sort(self, ids, experts: int, offsets, order, place) -> None:
        """ids (any shape, int32) -> offsets [experts + 1], order and place (as many as ids; order may be None)."""
        n = ids.numel()
        _room(n | experts)
        rc = self._lib.pearl_rows_sort(self._h, n, experts, self._dense(ids, "ids", _I32, n),
                                       self._dense(offsets, "offsets", _I32, experts + 1),
                                       None if order is None else self._dense(order, "order", _I32, n),
                                       self._dense(place, "place", _I32, n))
        if rc != 0:
            raise PearlError(rc, "pearl_rows_sort")

    def _sorted(self, t: torch.Tensor, what: str, width: int, like: torch.Tensor, name: str):
        """(address, rows) of a dense matrix of rows in sorted order."""
        if (t.dim() != 2 or t.shape[1] != width or t.dtype is not like.dtype or not t.is_contiguous() or
                t.get_device() != self._ordinal):
            raise ValueError("%s must be a contiguous [rows, %d] tensor on %s of the type of %s" % (what, width, self.device, name))
        _room(t.shape[0])
        return t.data_ptr(), t.shape[0]

    def _place(self, place: torch.Tensor, T: int):
        if place.dim() != 2 or place.shape[0] != T:
            raise ValueError("place must be [%d, k]" % T)
        _room(place.shape[1])
        return self._dense(place, "place", _I32, place.numel()), place.shape[1]

    def dispatch(self, x, place, xs) -> None:
        """xs[place[t, j]] = x[t] for rows of any type; place [T, k]."""
        p, T, width, ld = self._matrix(x, "x")
        at, k = self._place(place, T)
        to, rows = self._sorted(xs, "xs", width, x, "x")
        size = x.element_size()
        _room(width * size)
        rc = self._lib.pearl_rows_dispatch(self._h, T, k, width * size, p, ld * size, at, rows, to)
        if rc != 0:
            raise PearlError(rc, "pearl_rows_dispatch")

    def dispatch_grad(self, dxs, place, dx) -> None:
        """dx[t] = sum over j of dxs[place[t, j]]: the gradient of dispatch."""
        self.combine(dxs, place, None, dx)

    def combine(self, z, place, w, y) -> None:
        """y[t] = sum over j of w[t, j] * z[place[t, j]]; w None: weights of 1."""
        p, T, D, ld = self._matrix(y, "y")
        at, k = self._place(place, T)
        src, rows = self._sorted(z, "z", D, y, "y")
        rc = self._lib.pearl_rows_combine(self._h, T, k, D, self._type(y, "y"), src, rows, at,
                                          None if w is None else self._dense(w, "w", _F32, T * k), p, ld)
        if rc != 0:
            raise PearlError(rc, "pearl_rows_combine")

    def combine_grad(self, dy, z, place, w, dz=None, dw=None) -> None:
        """dz[place[t, j]] = w[t, j] * dy[t] and dw[t, j] = <dy[t], z[place[t, j]]>; dz or dw may be None (z with dw None, too)."""
        p, T, D, ld = self._matrix(dy, "dy")
        at, k = self._place(place, T)
        src, rows = (None, None) if z is None else self._sorted(z, "z", D, dy, "dy")
        to, rows_dz = (None, None) if dz is None else self._sorted(dz, "dz", D, dy, "dy")
        if dw is not None and z is None:
            raise ValueError("dw needs z")
        if rows is not None and rows_dz is not None and rows != rows_dz:
            raise ValueError("z and dz must have one shape")
        rc = self._lib.pearl_rows_combine_grad(self._h, T, k, D, self._type(dy, "dy"), p, ld, src,
                                               (rows if rows is not None else rows_dz) or 0, at,
                                               None if w is None else self._dense(w, "w", _F32, T * k), to,
                                               None if dw is None else self._dense(dw, "dw", _F32, T * k))
        if rc != 0:
            raise PearlError(rc, "pearl_rows_combine_grad")

    # ---- beam search -----------------------------------------------------------------------------
    def beam_select(self, logits, scores, best_score, best_beam, best_token, done=None, end_token: int = 0) -> None:
        """logits [G, W, V], scores [G, W] -> the C best offers of each group: best_score, best_beam, best_token [G, C].
        done [G, W] (uint8 or bool): finished beams, which offer end_token at their score."""
        if logits.dim() != 3 or logits.get_device() != self._ordinal or (logits.shape[2] > 1 and logits.stride(2) != 1):
            raise ValueError("logits must be a 3-D tensor on %s with contiguous rows" % self.device)
        G, W, V = logits.shape
        ld = logits.stride(1) if W > 1 else (logits.stride(0) if G > 1 else V)
        if (G > 1 and W > 1 and logits.stride(0) != W * ld) or ld < V:
            raise ValueError("the rows of logits must lie equally far apart")
        if best_token.dim() != 2 or best_token.shape[0] != G:
            raise ValueError("best_token must be [%d, C]" % G)
        best = best_token.shape[1]
        _room(G | W | V | best)
        if not -(1 << 31) <= end_token < 1 << 31:
            raise ValueError("end_token must be a 32-bit number")
        if done is not None and done.dtype is torch.bool:
            done = done.view(torch.uint8)
        rc = self._lib.pearl_rows_beam_select(self._h, G, W, V, best, self._type(logits, "logits"), logits.data_ptr(), ld,
                                              self._dense(scores, "scores", _F32, G * W),
                                              None if done is None else self._dense(done, "done", torch.uint8, G * W), end_token,
                                              self._dense(best_score, "best_score", _F32, G * best),
                                              self._dense(best_beam, "best_beam", _I32, G * best),
                                              self._dense(best_token, "best_token", _I32, G * best))
        if rc != 0:
            raise PearlError(rc, "pearl_rows_beam_select")

    def beam_reorder(self, states, parent, out=None) -> None:
        """out[o, g, i] = states[o, g, parent[g, i]]; states [blocks, G, W, ...], out None (or the same view): in place.
        The axes behind W may be a part of a larger cache, such as [heads, :length, dim]."""
        out = states if out is None else out
        shape = states.shape
        if len(shape) < 3 or states.get_device() != self._ordinal or out.get_device() != self._ordinal:
            raise ValueError("states and out must be [blocks, G, W, ...] on %s" % self.device)
        if out.shape != shape or out.dtype is not states.dtype:
            raise ValueError("out must have the shape and type of states")
        if states.numel() == 0:
            return
        pieces, piece_bytes, src, dst = _move(shape, states.stride(), out.stride(), states.element_size())
        rc = self._lib.pearl_rows_beam_reorder(self._h, shape[0], shape[1], shape[2], pieces, piece_bytes,
                                               self._dense(parent, "parent", _I32, shape[1] * shape[2]), states.data_ptr(), src,
                                               out.data_ptr(), dst)
        if rc != 0:
            raise PearlError(rc, "pearl_rows_beam_reorder")

    # ---- synchronisation -------------------------------------------------------------------------
    def sync(self) -> int:
        st = C.c_uint32(0)
        rc = self._lib.pearl_rows_sync(self._h, C.byref(st))
        if rc != 0:
            raise PearlError(rc, "pearl_rows_sync")
        return int(st.value)

    def kernel_launches(self) -> int:
        return int(self._lib.pearl_rows_kernel_launches(self._h))

    def close(self) -> None:
        if self._h is not None:
            self._lib.pearl_rows_destroy(self._h)
            self._h = None
            self._slab = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
