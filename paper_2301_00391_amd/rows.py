"""The operators on node rows that stand between two aggregations of a model: the norms around a block with its gate and
residual scale, the gated feed-forward block, and the gradients of both.  Argument marshalling only, as in binding.py; the
contract is in ``include/pipad.h``:
  pipad_residual_norm, pipad_residual_norm_backward -> :func:`residual_norm`, :func:`residual_norm_backward`
  pipad_gated_ff, pipad_gated_ff_backward           -> :func:`gated_ff`, :func:`gated_ff_backward`

Matrices are given as for :func:`frame_aggregate`: a list of k float32 [n, F] matrices that share a row stride, or one [n, k, F]
tensor.  Results that are not given are allocated in the form of the first operand, a list's k matrices as one piece of memory.
Calls only enqueue work on the stream.  Plain calls with memory for their results go through the binding's native half (see
binding.py), which leaves anything else to the code here.  The workspace comes from PyTorch's allocator where none is given.

What a call with ``stream=`` makes (results, gradients, the workspace) is memory of that stream and lives until the work that
is on the current stream when it is dropped has ended.  As always with PyTorch, the streams have to be ordered by the caller: the
given one behind what makes the operands, the current one behind the call before results are read; and an operand or a
workspace of another stream that is dropped early needs ``record_stream``.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding
from .binding import MAX_K, Features, _address, _check, _current_device, _current_raw_stream, _on_device, _operand, _pack_pointers, load_library

_NORMS = {None: 0, "rms": 1, "layer": 2}
_ACTIVATIONS = {"sigmoid": 0, "relu": 1, "gelu": 2, "silu": 3}
_MOST_ROWS, _TOO_LARGE = 2 ** 31 - 1, -4           # (ctypes would pass on the low 32 bits)
_size_t = ctypes.c_size_t
_pack_norm = struct.Struct("iiif5P").pack          # pipad_residual_norm_t
_pack_norm_grads = struct.Struct("5P").pack        # pipad_residual_norm_grads_t
_pack_ff = struct.Struct("4i3P3q3P").pack          # pipad_gated_ff_t
_pack_ff_grads = struct.Struct("3P3q3P").pack      # pipad_gated_ff_grads_t


class _Rows:
    """n, k, the device and the width of the first operand; everything else has to go with them."""

    def __init__(self, x: Features, name: str, stream=None):
        if isinstance(x, torch.Tensor):
            if x.dim() != 3:
                raise ValueError(f"{name}: a single tensor must have shape [n, k, F]")
            self.n, self.k, self.wide, first = x.shape[0], x.shape[1], True, x
        else:
            if not len(x) or x[0].dim() != 2:
                raise ValueError(f"{name}: need 1 to {MAX_K} matrices [n, F]")
            self.n, self.k, self.wide, first = x[0].shape[0], len(x), False, x[0]
        if not 1 <= self.k <= MAX_K:
            raise ValueError(f"{name}: need 1 to {MAX_K} matrices [n, F]")
        if self.n > _MOST_ROWS:
            _check(_TOO_LARGE)
        if not first.is_cuda:
            raise ValueError(f"{name}: every matrix must be float32 [n, F] on the GPU")
        self.device, self.index = first.device, first.get_device()
        self.raw, self.side = _current_raw_stream(self.index), None
        if stream is not None and int(stream.cuda_stream) != self.raw:
            self.raw = int(stream.cuda_stream)
            if isinstance(stream, torch.cuda.Stream):
                self.side = stream
            else:  # (the default stream has no pointer to be known by)
                self.side = torch.cuda.ExternalStream(self.raw, self.device) if self.raw else torch.cuda.default_stream(self.device)

    def empty(self, shape, dtype: torch.dtype = torch.float32, returned: bool = True) -> torch.Tensor:
        """Memory for a call on its stream.  The current stream's would not do for another one: the allocator gives again what has just been
        given back, which work that is queued on the current stream may still read."""
        if self.side is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.side):
            made = torch.empty(shape, dtype=dtype, device=self.device)
        if returned:
            made.record_stream(torch.cuda.current_stream(self.device))  # that is where it is read
        return made

    def operand(self, x: Optional[Features], name: str, F: Optional[int] = None):
        """(packed pointers, row stride) of an operand of F columns, or of none."""
        if x is None:
            return None, 0
        pointers, stride, width = _operand(x, self.n, self.k, name)
        if F is not None and width != F:
            raise ValueError(f"{name} must have {F} columns")
        for m in ((x,) if isinstance(x, torch.Tensor) else x):
            if m.get_device() != self.index:
                raise ValueError(f"{name} must be on the device of the other operands")
        return _pack_pointers(self.k)(*pointers), stride

    def width(self, x: Features) -> int:
        return (x if self.wide else x[0]).shape[-1]

    def room(self, F: int) -> Features:
        if self.wide:
            return self.empty((self.n, self.k, F))
        return list(self.empty((self.k, self.n, F)).unbind(0))

    def vector(self, v: Optional[torch.Tensor], F: int, name: str) -> int:
        if v is None:
            return 0
        if v.dtype != torch.float32 or v.dim() != 1 or v.shape[0] != F or (F > 1 and v.stride(0) != 1) or v.get_device() != self.index:
            raise ValueError(f"{name} must be a contiguous float32 vector of {F} entries on the operands' device")
        return v.data_ptr()

    def matrix(self, w: torch.Tensor, rows: int, columns: int, name: str) -> Tuple[int, int]:
        if w.dtype != torch.float32 or w.dim() != 2 or tuple(w.shape) != (rows, columns) or (columns > 1 and w.stride(1) != 1) or \
                w.get_device() != self.index:
            raise ValueError(f"{name} must be a float32 [{rows}, {columns}] matrix with unit column stride on the operands' device")
        return w.data_ptr(), w.stride(0) if rows > 1 else max(columns, w.stride(0))

    def call(self, fn, *args) -> None:
        _check(_on_device(self.index, fn, *args, self.raw))

    def workspace(self, given: Optional[torch.Tensor], nbytes: int) -> Tuple[Optional[torch.Tensor], int, int]:
        """(what to keep until the call is enqueued, its address, its bytes)"""
        if given is not None:
            if given.get_device() != self.index or not given.is_contiguous():
                raise ValueError("workspace must be contiguous memory on the operands' device")
            return given, given.data_ptr(), given.numel() * given.element_size()
        if not nbytes:
            return None, 0, 0
        made = self.empty(nbytes, torch.uint8, returned=False)
        return made, made.data_ptr(), nbytes


def _native(results):
    """(the native half, the current device, its stream) for a call on the current stream that brings the memory of its results."""
    if binding._host is None or any(r is None for r in results):
        return None
    device = _current_device()
    return binding._host, device, _current_raw_stream(device)


def _code(table, key):
    try:
        return table.get(key)
    except TypeError:  # nothing that a table could have
        return None


def _choice(table, key, name):
    code = _code(table, key)
    if code is None:
        raise ValueError(f"{name} must be one of {list(table)}")
    return code


# ---- norms ------------------------------------------------------------------------------------------------------------


class ResidualNormGrads(NamedTuple):
    """What :func:`residual_norm_backward` returns; None for what there is not or was not wanted."""
    dR: Optional[Features]
    dB: Optional[Features]
    dgate: Optional[Features]
    dscale: Optional[torch.Tensor]
    dw_post: Optional[torch.Tensor]
    db_post: Optional[torch.Tensor]
    dw_pre: Optional[torch.Tensor]
    db_pre: Optional[torch.Tensor]


def _norm_struct(rows, F, post, pre, eps, scale, w_post, b_post, w_pre, b_pre) -> bytes:
    vectors = [rows.vector(v, F, name) for v, name in ((scale, "scale"), (w_post, "w_post"), (b_post, "b_post"), (w_pre, "w_pre"), (b_pre, "b_pre"))]
    return _pack_norm(F, _choice(_NORMS, post, "post"), _choice(_NORMS, pre, "pre"), eps, *vectors)


def residual_norm(R: Features, B: Optional[Features] = None, gate: Optional[Features] = None, *, post: Optional[str] = None,
                  pre: Optional[str] = "rms", scale: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                  b_post: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, b_pre: Optional[torch.Tensor] = None,
                  eps: float = 1e-5, R_out: Optional[Features] = None, Z: Optional[Features] = None, stream=None):
    """pipad_residual_norm: R_out = R + scale * sigmoid(gate) * post(B) and Z = pre(R_out), in one pass over the rows of all snapshots;
    returns (R_out, Z).  ``post`` and ``pre`` are "rms", "layer" or None.  Without B, R_out is R and only Z is made; with
    ``pre=None`` there is no Z.  ``R_out`` may be ``R`` itself: the residual stream updated in place."""
    lib = load_library()
    native = _native((R_out,) * (B is not None) + (Z,) * (pre is not None)) if stream is None else None
    codes = _code(_NORMS, post), _code(_NORMS, pre)
    if native is not None and None not in codes:
        host, device, raw = native
        status = host.residual_norm(_address["pipad_residual_norm"], device, raw, R, B, gate, *codes, eps, scale, w_post, b_post, w_pre,
                                    b_pre, R_out, Z)
        if status is not None:
            if status:
                _check(status)
            return (R if B is None else R_out), Z
    rows = _Rows(R, "R", stream)
    F = rows.width(R)
    r = rows.operand(R, "R")
    norm = _norm_struct(rows, F, post, pre, eps, scale, w_post, b_post, w_pre, b_pre)
    if B is not None and R_out is None:
        R_out = rows.room(F)
    if pre is not None and Z is None:
        Z = rows.room(F)
    rows.call(lib.pipad_residual_norm, norm, rows.n, rows.k, *r, *rows.operand(B, "B", F), *rows.operand(gate, "gate", F),
              *rows.operand(R_out, "R_out", F), *rows.operand(Z, "Z", F))
    return (R if B is None else R_out), Z


def residual_norm_backward(R: Features, dR_out: Optional[Features] = None, dZ: Optional[Features] = None, B: Optional[Features] = None,
                           gate: Optional[Features] = None, *, post: Optional[str] = None, pre: Optional[str] = "rms",
                           scale: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                           b_post: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, eps: float = 1e-5,
                           vectors: bool = True, biases: bool = True, dR: Optional[Features] = None, dB: Optional[Features] = None,
                           dgate: Optional[Features] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> ResidualNormGrads:
    """pipad_residual_norm_backward: from R (the forward call's R_out; without B its R), B, gate and the gradients of R_out and Z (one of them
    may be None) those of R, B, gate and, unless ``vectors=False``, of the shared vectors: scale, the norms' weights and, unless
    ``biases=False``, their biases.  ``dR`` may be ``dR_out`` itself."""
    lib = load_library()
    wanted = (B is not None, post is not None, post is not None and biases, pre is not None, pre is not None and biases)
    wanted = tuple(bool(vectors and w) for w in wanted)
    native = _native((dR,) + (dB,) * (B is not None) + (dgate,) * (gate is not None)) if stream is None and workspace is None else None
    codes = _code(_NORMS, post), _code(_NORMS, pre)
    if native is not None and None not in codes:
        host, device, raw = native
        made = host.residual_norm_backward(_address["pipad_residual_norm_backward"], _address["pipad_residual_norm_workspace"], device, raw, R, dR_out, dZ,
                                           B, gate, *codes, eps, scale, w_post, b_post, w_pre, None, dR, dB, dgate, *wanted)
        if made is not None:
            if made[0]:
                _check(made[0])
            return ResidualNormGrads(dR, dB, dgate, *made[1:])
    rows = _Rows(R, "R", stream)
    F = rows.width(R)
    r = rows.operand(R, "R")
    norm = _norm_struct(rows, F, post, pre, eps, scale, w_post, b_post, w_pre, None)
    if dR is None:
        dR = rows.room(F)
    if B is not None and dB is None:
        dB = rows.room(F)
    if gate is not None and dgate is None:
        dgate = rows.room(F)
    grads = [rows.empty(F) if w else None for w in wanted]
    packed, kept, ws = None, None, (0, 0)
    if any(wanted):
        packed = _pack_norm_grads(*[0 if d is None else d.data_ptr() for d in grads])
        need = _size_t()
        _check(lib.pipad_residual_norm_workspace(F, rows.n, rows.k, ctypes.byref(need)))
        kept, *ws = rows.workspace(workspace, need.value)
    rows.call(lib.pipad_residual_norm_backward, norm, rows.n, rows.k, *r, *rows.operand(B, "B", F), *rows.operand(gate, "gate", F),
              *rows.operand(dR_out, "dR_out", F), *rows.operand(dZ, "dZ", F), *rows.operand(dR, "dR", F), *rows.operand(dB, "dB", F),
              *rows.operand(dgate, "dgate", F), packed, *ws)
    return ResidualNormGrads(dR, dB, dgate, *grads)


# ---- the gated feed-forward block -------------------------------------------------------------------------------------


class GatedFFGrads(NamedTuple):
    """What :func:`gated_ff_backward` returns; None for what was not wanted."""
    dX: Optional[Features]
    dWg: Optional[torch.Tensor]
    dWu: Optional[torch.Tensor]
    dWd: Optional[torch.Tensor]
    dbg: Optional[torch.Tensor]
    dbu: Optional[torch.Tensor]
    dbd: Optional[torch.Tensor]


def _ff_struct(rows, F, Wg, Wu, Wd, bg, bu, bd, activation) -> Tuple[bytes, int, int]:
    if Wg.dim() != 2 or Wd.dim() != 2:
        raise ValueError("Wg, Wu and Wd must be float32 matrices [F, hidden], [F, hidden] and [hidden, Fo]")
    hidden, Fo = Wg.shape[1], Wd.shape[1]
    (pg, lg), (pu, lu) = rows.matrix(Wg, F, hidden, "Wg"), rows.matrix(Wu, F, hidden, "Wu")
    pd, ld = rows.matrix(Wd, hidden, Fo, "Wd")
    return _pack_ff(F, hidden, Fo, _choice(_ACTIVATIONS, activation, "activation"), pg, pu, pd, lg, lu, ld, rows.vector(bg, hidden, "bg"),
                    rows.vector(bu, hidden, "bu"), rows.vector(bd, Fo, "bd")), hidden, Fo


def gated_ff(X: Features, Wg: torch.Tensor, Wu: torch.Tensor, Wd: torch.Tensor, bg: Optional[torch.Tensor] = None,
             bu: Optional[torch.Tensor] = None, bd: Optional[torch.Tensor] = None, *, activation: str = "silu", Y: Optional[Features] = None,
             workspace: Optional[torch.Tensor] = None, stream=None) -> Features:
    """pipad_gated_ff: Y = (act(X Wg + bg) * (X Wu + bu)) Wd + bd on the rows of all snapshots, whatever lies between staying on the
    chip.  Wg and Wu are float32 [F, hidden], Wd [hidden, Fo]; ``activation`` is "silu", "gelu" (the exact one), "relu" or "sigmoid"."""
    lib = load_library()
    native = _native((Y,)) if stream is None and workspace is None else None
    code = _code(_ACTIVATIONS, activation)
    if native is not None and code is not None:
        host, device, raw = native
        status = host.gated_ff(_address["pipad_gated_ff"], _address["pipad_gated_ff_workspace"], device, raw, X, Wg, Wu, Wd, bg, bu, bd,
                               code, Y)
        if status is not None:
            if status:
                _check(status)
            return Y
    rows = _Rows(X, "X", stream)
    F = rows.width(X)
    x = rows.operand(X, "X")
    block, _, Fo = _ff_struct(rows, F, Wg, Wu, Wd, bg, bu, bd, activation)
    if Y is None:
        Y = rows.room(Fo)
    need = _size_t()
    _check(lib.pipad_gated_ff_workspace(block, rows.n, rows.k, 0, ctypes.byref(need)))
    kept, *ws = rows.workspace(workspace, need.value)
    rows.call(lib.pipad_gated_ff, block, rows.n, rows.k, *x, *rows.operand(Y, "Y", Fo), *ws)
    return Y


def gated_ff_backward(X: Features, dY: Features, Wg: torch.Tensor, Wu: torch.Tensor, Wd: torch.Tensor, bg: Optional[torch.Tensor] = None,
                      bu: Optional[torch.Tensor] = None, *, activation: str = "silu", rows_grad: bool = True, weights: bool = True,
                      biases: bool = True, dX: Optional[Features] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> GatedFFGrads:
    """pipad_gated_ff_backward: from X and dY the gradient of X (unless ``rows_grad=False``), of the matrices (unless ``weights=False``) and
    of the biases (unless ``biases=False``); G, U and H are made again, so nothing has to be kept from the forward call.
    Made for rows of up to 256 columns: for many wider ones the matrices' gradients take longer than products one by one."""
    lib = load_library()
    native = _native((dX,) * bool(rows_grad)) if stream is None and workspace is None else None
    code = _code(_ACTIVATIONS, activation)
    if native is not None and code is not None:
        host, device, raw = native
        made = host.gated_ff_backward(_address["pipad_gated_ff_backward"], _address["pipad_gated_ff_workspace"], device, raw, X, Wg, Wu, Wd, bg, bu, None,
                                      code, dY, dX if rows_grad else None, bool(weights), bool(biases))
        if made is not None:
            if made[0]:
                _check(made[0])
            return GatedFFGrads(dX if rows_grad else None, *made[1:])
    rows = _Rows(X, "X", stream)
    F = rows.width(X)
    x = rows.operand(X, "X")
    block, hidden, Fo = _ff_struct(rows, F, Wg, Wu, Wd, bg, bu, None, activation)
    dy = rows.operand(dY, "dY", Fo)
    if not rows_grad:
        dX = None
    elif dX is None:
        dX = rows.room(F)
    shapes = [(F, hidden), (F, hidden), (hidden, Fo)] if weights else [None] * 3
    shapes += [(hidden,), (hidden,), (Fo,)] if biases else [None] * 3
    grads = [None if s is None else rows.empty(s) for s in shapes]
    packed = None
    if weights or biases:
        at = [0 if d is None else d.data_ptr() for d in grads]
        packed = _pack_ff_grads(*at[:3], hidden, hidden, Fo, *at[3:])
    need = _size_t()
    _check(lib.pipad_gated_ff_workspace(block, rows.n, rows.k, 1, ctypes.byref(need)))
    kept, *ws = rows.workspace(workspace, need.value)
    rows.call(lib.pipad_gated_ff_backward, block, rows.n, rows.k, *x, *dy, *rows.operand(dX, "dX", F), packed, *ws)
    return GatedFFGrads(dX, *grads)
