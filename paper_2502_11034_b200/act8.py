"""Activation checkpoints in 8 bits and their use in the backward pass (include/adagc_ops.h).

Forward of a SwiGLU MLP:              Backward:
    x8 = encode(x)                        grad_h = grad_y @ w_down
    h, gate8, up8 = swiglu(gate, up)      grad_gate, grad_up, h8 = swiglu_backward(grad_h, gate8, up8, recompute_h=True)
                                          linear_wgrad(grad_y, h8, out=grad_w_down)
                                          linear_wgrad(grad_gate, x8, out=grad_w_gate)   ...

x8, gate8 and up8 are all that is kept between the two: 3 + 3/32 bytes per element instead of 8 (bfloat16 x, gate, up, h).
Calls only enqueue work, on `stream` (default: the current stream); outputs belong to that stream.  Tensors made or freed on
another stream have to be ordered by the caller, as with every entry point of this package.  There is no autograd here: tensors
that require a gradient are read (and written) as they are, results never require one, and the backward pass is calls of its own.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import ADAGC_BF16, adagc_act8, check, lib, matrix_args, run_on

GROUP = 32         # consecutive elements of a row that share one power of two
PITCH_STEP = 128   # rows of codes are padded to a multiple of this


def pitch(cols: int) -> int:
    """Codes per row of a checkpoint of `cols` columns."""
    return -(-int(cols) // PITCH_STEP) * PITCH_STEP


class Act8:
    """A checkpoint of a [rows, cols] matrix: codes [rows, pitch(cols)] int8 and exps [rows, pitch(cols) / 32] uint8."""

    __slots__ = ("rows", "cols", "device", "_parts", "_both", "_at", "_ref")

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor, cols: int):
        p = pitch(cols)
        if codes.dtype != torch.int8 or exps.dtype != torch.uint8 or not codes.is_cuda or codes.device != exps.device:
            raise ValueError("a checkpoint has int8 codes and uint8 exponents on one CUDA device")
        if codes.dim() != 2 or codes.shape[1] != p or exps.shape != (codes.shape[0], p // GROUP):
            raise ValueError(f"a checkpoint of {cols} columns has codes [rows, {p}] and exponents [rows, {p // GROUP}], got "
                             f"{tuple(codes.shape)} and {tuple(exps.shape)}")
        if not codes.is_contiguous() or not exps.is_contiguous():
            raise ValueError("the parts of a checkpoint must be contiguous")
        self.rows, self.cols, self.device = codes.shape[0], int(cols), codes.device
        self._parts, self._both, self._at = (codes, exps), None, 0
        self._ref = C.byref(adagc_act8(codes.data_ptr(), exps.data_ptr()))

    def _views(self):
        """(codes, exps); of a checkpoint made by empty() they are views of its one buffer, made when first asked for."""
        if self._parts is None:
            p = pitch(self.cols)
            mid = self._at + self.rows * p
            self._parts = (self._both[self._at:mid].view(self.rows, p),
                           self._both[mid:mid + self.rows * (p // GROUP)].view(torch.uint8).view(self.rows, p // GROUP))
        return self._parts

    @property
    def codes(self) -> torch.Tensor:
        return self._views()[0]

    @property
    def exps(self) -> torch.Tensor:
        return self._views()[1]

    @property
    def nbytes(self) -> int:
        return self.rows * (pitch(self.cols) + pitch(self.cols) // GROUP)

    def __getitem__(self, rows: slice) -> "Act8":
        """The checkpoint of a range of rows (a view)."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            raise ValueError("a checkpoint is indexed by a range of rows")
        return Act8(self.codes[rows], self.exps[rows], self.cols)


def empty(rows: int, cols: int, device) -> Act8:
    """An uninitialised checkpoint, both parts in one buffer."""
    return _inside(torch.empty(rows * (pitch(cols) + pitch(cols) // GROUP), dtype=torch.int8, device=device), 0, rows, cols, pitch(cols))


def _new(like: torch.Tensor, rows: int, cols: int) -> Act8:
    p = -(-cols // PITCH_STEP) * PITCH_STEP
    return _inside(like.new_empty((rows * (p + p // GROUP),), dtype=torch.int8), 0, rows, cols, p)


def _new_pair(like: torch.Tensor, rows: int, cols: int) -> Tuple[Act8, Act8]:
    """Two checkpoints of one size in one buffer."""
    p = -(-cols // PITCH_STEP) * PITCH_STEP
    n = -(-rows * (p + p // GROUP) // 16) * 16
    both = like.new_empty((2 * n,), dtype=torch.int8)
    return _inside(both, 0, rows, cols, p), _inside(both, n, rows, cols, p)


def _inside(both: torch.Tensor, at: int, rows: int, cols: int, p: int) -> Act8:
    c = Act8.__new__(Act8)
    c.rows, c.cols, c.device, c._parts, c._both, c._at = rows, cols, both.device, None, both, at
    base = both.data_ptr() + at
    c._ref = C.byref(adagc_act8(base, base + rows * p))
    return c


def _like(t: torch.Tensor) -> torch.Tensor:
    """An uninitialised contiguous matrix of t's shape and dtype."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _same(name: str, t: torch.Tensor, like: torch.Tensor) -> None:
    if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: expected {tuple(like.shape)} {like.dtype} on {like.device}, got {tuple(t.shape)} {t.dtype} on {t.device}")


def _same8(name: str, c: Act8, rows: int, cols: int, device: torch.device) -> None:
    if c.rows != rows or c.cols != cols or c.device != device:
        raise ValueError(f"{name}: expected a checkpoint of [{rows}, {cols}] on {device}, got [{c.rows}, {c.cols}] on {c.device}")


def encode(x: torch.Tensor, out: Optional[Act8] = None, stream=None) -> Act8:
    """adagc_act8_encode: x [rows, cols] float32 or bfloat16 (any row stride)."""
    return run_on(x.device, stream, _encode, x, out)


def _encode(x, out, stream):
    p, dtype, rows, cols, ld = matrix_args(x, "x")
    if out is None:
        out = _new(x, rows, cols)
    else:
        _same8("out", out, rows, cols, x.device)
    check(lib().adagc_act8_encode(p, dtype, rows, cols, ld, out._ref, stream), "adagc_act8_encode")
    return out


def decode(c: Act8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """adagc_act8_decode: the values the checkpoint stands for (exact in either dtype)."""
    return run_on(c.device, stream, _decode, c, dtype, out)


def _decode(c, dtype, out, stream):
    if out is None:
        out = (c.codes if c._both is None else c._both).new_empty((c.rows, c.cols), dtype=dtype)
    p, code, rows, cols, ld = matrix_args(out, "out")
    _same8("out", c, rows, cols, out.device)
    check(lib().adagc_act8_decode(c._ref, rows, cols, p, code, ld, stream), "adagc_act8_decode")
    return out


def swiglu(gate: torch.Tensor, up: torch.Tensor, stream=None) -> Tuple[torch.Tensor, Act8, Act8]:
    """adagc_act8_swiglu: (h = silu(gate) * up, checkpoint of gate, checkpoint of up)."""
    return run_on(gate.device, stream, _swiglu, gate, up)


def _swiglu(gate, up, stream):
    _same("up", up, gate)
    pg, dtype, rows, cols, ldg = matrix_args(gate, "gate")
    pu, _, _, _, ldu = matrix_args(up, "up")
    h = _like(gate)
    gate8, up8 = _new_pair(gate, rows, cols)
    check(lib().adagc_act8_swiglu(pg, ldg, pu, ldu, dtype, rows, cols, h.data_ptr(), max(cols, 1), gate8._ref, up8._ref, stream),
          "adagc_act8_swiglu")
    return h, gate8, up8


def swiglu_backward(grad_h: torch.Tensor, gate8: Act8, up8: Act8, recompute_h: bool = False,
                    out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, Optional[Act8]]:
    """adagc_act8_swiglu_backward: (grad_gate, grad_up, checkpoint of h or None).  `out` = (grad_gate, grad_up) to write into,
    for instance the two halves of one [rows, 2 * cols] matrix where one weight holds both projections."""
    return run_on(grad_h.device, stream, _swiglu_backward, grad_h, gate8, up8, recompute_h, out)


def _swiglu_backward(grad_h, gate8, up8, recompute_h, out, stream):
    p, dtype, rows, cols, ld = matrix_args(grad_h, "grad_h")
    dev = grad_h.device
    _same8("gate8", gate8, rows, cols, dev)
    _same8("up8", up8, rows, cols, dev)
    if out is None:
        grad_gate, grad_up = _like(grad_h), _like(grad_h)
        pg, pu, ldg, ldu = grad_gate.data_ptr(), grad_up.data_ptr(), max(cols, 1), max(cols, 1)
    else:
        grad_gate, grad_up = out
        _same("out[0]", grad_gate, grad_h)
        _same("out[1]", grad_up, grad_h)
        pg, _, _, _, ldg = matrix_args(grad_gate, "out[0]")
        pu, _, _, _, ldu = matrix_args(grad_up, "out[1]")
    h8 = _new(grad_h, rows, cols) if recompute_h else None
    check(lib().adagc_act8_swiglu_backward(p, ld, dtype, rows, cols, gate8._ref, up8._ref, pg, ldg, pu, ldu, h8._ref if recompute_h else None,
                                           stream), "adagc_act8_swiglu_backward")
    return grad_gate, grad_up, h8


def linear_wgrad(grad_y: torch.Tensor, x8: Act8, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                 accumulate: bool = False, stream=None) -> torch.Tensor:
    """adagc_act8_linear_wgrad: grad_y^T x^ for grad_y [tokens, out_features] bfloat16 and the checkpoint of
    [tokens, in_features].  `out` (float32 or bfloat16, any row stride) may be a tensor of the gradient arena; with
    `accumulate` the result is added to it."""
    return run_on(grad_y.device, stream, _linear_wgrad, grad_y, x8, dtype, out, accumulate)


def _linear_wgrad(grad_y, x8, dtype, out, accumulate, stream):
    p, gy, tokens, n, ld = matrix_args(grad_y, "grad_y")
    if gy != ADAGC_BF16:
        raise ValueError(f"grad_y must be bfloat16, got {grad_y.dtype}")
    dev = grad_y.device
    _same8("x8", x8, tokens, x8.cols, dev)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = grad_y.new_empty((n, x8.cols), dtype=dtype)
    q, code, on, ok, old = matrix_args(out, "out")
    if on != n or ok != x8.cols or out.device != dev:
        raise ValueError(f"out: expected [{n}, {x8.cols}] on {dev}, got {tuple(out.shape)} on {out.device}")
    L = lib()
    nbytes = L.adagc_act8_linear_wgrad_workspace_bytes(tokens, n, ok, p, ld)
    if nbytes < 0:
        check(nbytes, "adagc_act8_linear_wgrad_workspace_bytes")
    ws = grad_y.new_empty((nbytes,), dtype=torch.uint8) if nbytes else None
    check(L.adagc_act8_linear_wgrad(p, gy, ld, x8._ref, tokens, n, ok, q, code, old, 1 if accumulate else 0,
                                    ws.data_ptr() if nbytes else None, nbytes, stream), "adagc_act8_linear_wgrad")
    return out
