"""The operators of a Dense Part made of experts (include/gear.h) on PyTorch tensors: argument checks, output and workspace
memory, marshalling.  Matrices are [rows x width] with neighbouring columns next to each other; rows may lie further apart.
Calls enqueue on the current stream and do not synchronise."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from .binding import (GEAR_BF16, GEAR_E4M3, GEAR_ERR_INVALID, GEAR_F32, GearError, _check, _ptr, _stream, gear_expert_args,
                      gear_expert_wgrad_args, gear_grad_tensor, gear_norm_args, gear_norm_backward_args, lib)

_CODE = {torch.float32: GEAR_F32, torch.bfloat16: GEAR_BF16}
_BYTE = (torch.uint8, torch.float8_e4m3fn)


def _need(ok: bool, where: str, what: str) -> None:
    if not ok:
        raise GearError(GEAR_ERR_INVALID, f"{where}: {what}")


def _matrix(t: torch.Tensor, where: str, name: str, dtype: Optional[torch.dtype] = None, shape=None) -> int:
    """Checks a matrix on the device and returns the distance between its rows."""
    _need(t.is_cuda and t.dim() == 2 and (t.dtype == dtype if dtype is not None else t.dtype in _CODE), where,
          f"{name} has to be a matrix on the GPU of {dtype or 'float32 or bfloat16'}")
    _need(shape is None or tuple(t.shape) == tuple(shape), where, f"{name} has to be {shape}, not {tuple(t.shape)}")
    _need(t.shape[1] <= 1 or t.stride(1) == 1, where, f"{name}'s columns have to lie next to each other")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t: torch.Tensor, where: str, name: str, dtype: torch.dtype, n: int) -> None:
    _need(t.is_cuda and t.dtype == dtype and t.is_contiguous() and t.numel() == n, where, f"{name} has to be {n} contiguous {dtype} on the GPU")


class Rows8(NamedTuple):
    """Rows in 8 bits: q [rows x gear_rows8_ld(dim)] (bytes of e4m3), scale [rows x gear_scales8_ld(dim)] (exponent + 127)."""
    q: torch.Tensor
    scale: torch.Tensor
    dim: int

    @staticmethod
    def empty(rows: int, dim: int, device) -> "Rows8":
        return Rows8(torch.empty((rows, (dim + 127) // 128 * 128), dtype=torch.float8_e4m3fn, device=device),
                     torch.empty((rows, (dim + 511) // 512 * 4), dtype=torch.uint8, device=device), dim)

    def check(self, where: str) -> None:
        rows = self.q.shape[0]
        _need(self.q.is_cuda and self.q.dtype in _BYTE and self.q.is_contiguous() and self.q.shape == (rows, lib.gear_rows8_ld(self.dim)),
              where, "q has to be [rows x gear_rows8_ld(dim)] contiguous bytes on the GPU")
        _need(self.scale.is_cuda and self.scale.dtype == torch.uint8 and self.scale.is_contiguous() and
              self.scale.shape == (rows, lib.gear_scales8_ld(self.dim)), where,
              "scale has to be [rows x gear_scales8_ld(dim)] contiguous bytes on the GPU")


class NormOutput(NamedTuple):
    sum: Optional[torch.Tensor]     # x + residual; None without a residual
    y: Optional[torch.Tensor]
    rows8: Optional[Rows8]


def gear_rmsnorm(x: torch.Tensor, gain: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None, y: bool = True,
                 q8: bool = False, out: Optional[NormOutput] = None) -> NormOutput:
    """Norm of h = x + residual: the sum (where there is a residual), the norm times gain (`y`), the same in 8 bits (`q8`).
    out: memory for the results (any of its fields may be None) instead of new tensors; sum may be residual or x itself."""
    where = "gear_rmsnorm"
    ld_x = _matrix(x, where, "x")
    rows, dim = x.shape
    _vector(gain, where, "gain", torch.float32, dim)
    ld_r = ld_s = ld_y = 0
    given = out or NormOutput(None, None, None)
    o_sum = o_y = r8 = None
    if residual is not None:
        ld_r = _matrix(residual, where, "residual", x.dtype, x.shape)
    if residual is not None or given.sum is not None:
        o_sum = given.sum if given.sum is not None else torch.empty((rows, dim), dtype=x.dtype, device=x.device)
        ld_s = _matrix(o_sum, where, "sum", x.dtype, x.shape)
    if y:
        o_y = given.y if given.y is not None else torch.empty((rows, dim), dtype=x.dtype, device=x.device)
        ld_y = _matrix(o_y, where, "y", x.dtype, x.shape)
    if q8:
        r8 = given.rows8 if given.rows8 is not None else Rows8.empty(rows, dim, x.device)
        if given.rows8 is not None:
            r8.check(where)
            _need(r8.dim == dim and r8.q.shape[0] == rows, where, "rows8 has another shape than x")
    a = gear_norm_args(rows, dim, _CODE[x.dtype], eps, _ptr(x), _ptr(residual), _ptr(gain), _ptr(o_sum), _ptr(o_y), ld_x, ld_r, ld_s,
                       ld_y, _ptr(r8.q) if r8 else None, _ptr(r8.scale) if r8 else None)
    _check(lib.gear_rmsnorm(C.byref(a), _stream()), where)
    return NormOutput(o_sum, o_y, r8)


def gear_rmsnorm_backward(h: torch.Tensor, gain: torch.Tensor, dy: torch.Tensor, eps: float, dsum: Optional[torch.Tensor] = None,
                          dx: Optional[torch.Tensor] = None, dgain: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dgain) of the norm at h, dsum (what flows into the sum itself) added to dx; dx may be dy or dsum."""
    where = "gear_rmsnorm_backward"
    ld_h, ld_dy = _matrix(h, where, "h"), _matrix(dy, where, "dy", h.dtype, h.shape)
    rows, dim = h.shape
    _vector(gain, where, "gain", torch.float32, dim)
    ld_ds = _matrix(dsum, where, "dsum", h.dtype, h.shape) if dsum is not None else 0
    if dx is None:
        dx = torch.empty((rows, dim), dtype=h.dtype, device=h.device)
    ld_dx = _matrix(dx, where, "dx", h.dtype, h.shape)
    if dgain is None:
        dgain = torch.empty(dim, dtype=torch.float32, device=h.device)
    _vector(dgain, where, "dgain", torch.float32, dim)
    ws = torch.empty(lib.gear_norm_backward_workspace_bytes(rows, dim), dtype=torch.uint8, device=h.device)
    a = gear_norm_backward_args(rows, dim, _CODE[h.dtype], eps, _ptr(h), _ptr(dy), _ptr(dsum), _ptr(gain), _ptr(dx), _ptr(dgain), ld_h,
                                ld_dy, ld_ds, ld_dx)
    _check(lib.gear_rmsnorm_backward(C.byref(a), _ptr(ws), ws.numel(), _stream()), where)
    return dx, dgain


def gear_rows8(x: torch.Tensor, out: Optional[Rows8] = None) -> Rows8:
    """x in 8 bits, a scale for every row and 128 columns."""
    where = "gear_rows8"
    ld = _matrix(x, where, "x")
    rows, dim = x.shape
    if out is None:
        out = Rows8.empty(rows, dim, x.device)
    out.check(where)
    _need(out.dim == dim and out.q.shape[0] == rows, where, "out has another shape than x")
    _check(lib.gear_rows8(_ptr(x), _CODE[x.dtype], ld, rows, dim, _ptr(out.q), _ptr(out.scale), _stream()), where)
    return out


def _weights(w: torch.Tensor, where: str) -> Tuple[int, int, int]:
    _need(w.is_cuda and w.dim() in (2, 3) and w.dtype in _CODE and w.is_contiguous(), where,
          "w has to be contiguous [experts x N x K] or [N x K] on the GPU, float32 or bfloat16")
    return (1, *w.shape) if w.dim() == 2 else tuple(w.shape)


def _packed_room(operand: int, experts: int, n: int, k: int, transposed: bool, device, where: str) -> torch.Tensor:
    size = lib.gear_packed_weights_bytes(operand, experts, n, k, int(transposed))
    _need(size > 0, where, f"weights of {experts} x {n} x {k} have no packed form")
    return torch.empty(size, dtype=torch.uint8, device=device)


class Weights8(NamedTuple):
    """Weights in 8 bits, laid out for gear_matmul8."""
    packed: torch.Tensor
    scale: torch.Tensor
    experts: int
    N: int
    K: int


def gear_weights8(w: torch.Tensor) -> Weights8:
    """w ([experts x N x K] or [N x K], float32 or bfloat16) in 8 bits, a scale for every 128 x 128 weights."""
    experts, n, k = _weights(w, "gear_weights8")
    size = lib.gear_weight_scales_bytes(experts, n, k)
    _need(size > 0, "gear_weights8", f"weights of {experts} x {n} x {k} have no packed form")
    scale = torch.empty(size, dtype=torch.uint8, device=w.device)
    packed = _packed_room(GEAR_E4M3, experts, n, k, False, w.device, "gear_weights8")
    _check(lib.gear_pack_weights(_ptr(w), _CODE[w.dtype], GEAR_E4M3, experts, n, k, _ptr(packed), None, _ptr(scale), _stream()), "gear_weights8")
    return Weights8(packed, scale, experts, n, k)


class ExpertWeights:
    """Weights of every expert laid out for the forward product and (transposed) for the gradient of its input, in float32
    or bfloat16 (`operand`, w's own type if not given).  A training program calls update() when the weights have changed."""

    def __init__(self, w: torch.Tensor, operand: Optional[torch.dtype] = None, backward: bool = True):
        self.experts, self.N, self.K = _weights(w, "ExpertWeights")
        self.dtype = operand or w.dtype
        _need(self.dtype in _CODE, "ExpertWeights", "operand has to be float32 or bfloat16")
        self.forward = _packed_room(_CODE[self.dtype], self.experts, self.N, self.K, False, w.device, "ExpertWeights")
        self.transposed = _packed_room(_CODE[self.dtype], self.experts, self.N, self.K, True, w.device, "ExpertWeights") if backward else None
        self.update(w)

    def update(self, w: torch.Tensor) -> None:
        e, n, k = _weights(w, "ExpertWeights.update")
        _need((e, n, k) == (self.experts, self.N, self.K), "ExpertWeights.update", "w has another shape than before")
        _check(lib.gear_pack_weights(_ptr(w), _CODE[w.dtype], _CODE[self.dtype], e, n, k, _ptr(self.forward), _ptr(self.transposed), None,
                                     _stream()), "ExpertWeights.update")


def _offsets(off: Optional[torch.Tensor], experts: int, status: Optional[torch.Tensor], device, where: str):
    if off is None:
        _need(experts == 1, where, "off may only be left out where there is one expert")
        return status
    _vector(off, where, "off", torch.int32, experts + 1)
    if status is None:
        status = torch.empty(1, dtype=torch.int32, device=device)
    return status


def _product(where, dtype, x, x_scale, ld_x, packed, w_scale, rows, n, k, experts, off, out, out_dtype, status) -> torch.Tensor:
    status = _offsets(off, experts, status, x.device, where)
    if out is None:
        out = torch.empty((rows, n), dtype=out_dtype, device=x.device)
    ld_out = _matrix(out, where, "out", None, (rows, n))
    a = gear_expert_args(dtype, _CODE[out.dtype], rows, k, n, experts, _ptr(x), _ptr(x_scale), _ptr(packed), _ptr(w_scale), _ptr(off),
                         _ptr(out), ld_x, ld_out, _ptr(status))
    _check(lib.gear_expert_product(C.byref(a), _stream()), where)
    return out


def gear_matmul8(rows8: Rows8, weights: Weights8, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 out_dtype: torch.dtype = torch.bfloat16, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rows8 times the transposed 8-bit weights.  off [experts + 1] (int32, on the GPU): where each expert's rows begin; rows
    from off[experts] on are not written.  status [1] (int32): GEAR_ERR_RANGE if off is no such list, and nothing is written."""
    where = "gear_matmul8"
    rows8.check(where)
    _need(rows8.dim == weights.K, where, f"rows of {rows8.dim} for weights of {weights.K}")
    return _product(where, GEAR_E4M3, rows8.q, rows8.scale, rows8.q.shape[1], weights.packed, weights.scale, rows8.q.shape[0], weights.N,
                    weights.K, weights.experts, off, out, out_dtype, status)


def gear_expert_matmul(x: torch.Tensor, weights: ExpertWeights, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows x K] times the transposed weights of each row's expert: [rows x N]; off and status as for gear_matmul8."""
    where = "gear_expert_matmul"
    ld = _matrix(x, where, "x", weights.dtype, (x.shape[0], weights.K))
    return _product(where, _CODE[x.dtype], x, None, ld, weights.forward, None, x.shape[0], weights.N, weights.K, weights.experts, off, out,
                    out_dtype or x.dtype, status)


def gear_expert_dgrad(dy: torch.Tensor, weights: ExpertWeights, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      out_dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dy [rows x N] times the weights of each row's expert: the gradient [rows x K] of gear_expert_matmul's x."""
    where = "gear_expert_dgrad"
    ld = _matrix(dy, where, "dy", weights.dtype, (dy.shape[0], weights.N))
    _need(weights.transposed is not None, where, "the weights were laid out without backward")
    return _product(where, _CODE[dy.dtype], dy, None, ld, weights.transposed, None, dy.shape[0], weights.K, weights.N, weights.experts, off,
                    out, out_dtype or dy.dtype, status)


def gear_expert_wgrad(dy: torch.Tensor, x: torch.Tensor, off: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                      status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dy_e^T x_e for every expert: [experts x N x K] float32, zeros for one without rows."""
    where = "gear_expert_wgrad"
    ld_x = _matrix(x, where, "x")
    rows, k = x.shape
    n = dy.shape[-1]
    ld_dy = _matrix(dy, where, "dy", x.dtype, (rows, n))
    experts = 1 if off is None else off.numel() - 1
    status = _offsets(off, experts, status, x.device, where)
    if dw is None:
        dw = torch.empty((experts, n, k), dtype=torch.float32, device=x.device)
    _vector(dw, where, "dw", torch.float32, experts * n * k)
    ws = torch.empty(lib.gear_expert_wgrad_workspace_bytes(_CODE[x.dtype], rows, experts, n, k), dtype=torch.uint8, device=x.device)
    a = gear_expert_wgrad_args(_CODE[x.dtype], rows, k, n, experts, _ptr(dy), _ptr(x), _ptr(off), _ptr(dw), ld_dy, ld_x, _ptr(status))
    _check(lib.gear_expert_wgrad(C.byref(a), _ptr(ws), ws.numel(), _stream()), where)
    return dw


class GradList:
    """A list of gradients for gear_grad_norm and gear_clip_grads; `out` (the tensors that receive the clipped gradients) is
    the gradients themselves unless given.  Holds for as long as the tensors keep their memory: build it once, or again when
    a gradient has been replaced."""

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        where = "GradList"
        _need(len(grads) > 0 and (out is None or len(out) == len(grads)), where, "a list of tensors, and as many to receive them")
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        entries = (gear_grad_tensor * len(self.grads))()
        for e, g, o in zip(entries, self.grads, self.out):
            _need(all(t.is_cuda and t.is_contiguous() and t.dtype in _CODE for t in (g, o)) and g.dtype == o.dtype and g.numel() == o.numel(),
                  where, "contiguous float32 or bfloat16 tensors on the GPU, each as large as the one that receives it")
            e.src, e.dst, e.n, e.dtype = g.data_ptr() or None, o.data_ptr() or None, g.numel(), _CODE[g.dtype]
        host = torch.empty(lib.gear_grad_list_bytes(len(self.grads)), dtype=torch.uint8)
        chunks = C.c_int64()
        _check(lib.gear_grad_list_pack(entries, len(self.grads), host.data_ptr(), C.byref(chunks)), where)
        self.chunks = chunks.value
        self.list = host.to(self.grads[0].device)
        self.workspace = torch.empty(lib.gear_grad_workspace_bytes(self.chunks), dtype=torch.uint8, device=self.list.device)


def gear_grad_norm(grads: GradList, norm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The norm [1] of all gradients of the list together."""
    norm = torch.empty((), dtype=torch.float32, device=grads.list.device) if norm is None else norm
    _vector(norm, "gear_grad_norm", "norm", torch.float32, 1)
    _check(lib.gear_grad_norm(_ptr(grads.list), len(grads.grads), grads.chunks, _ptr(grads.workspace), grads.workspace.numel(), _ptr(norm),
                              _stream()), "gear_grad_norm")
    return norm


def gear_clip_grads(grads: GradList, max_norm: float, norm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scales the gradients of the list so that their norm is at most max_norm; returns the norm [1] that they had."""
    norm = torch.empty((), dtype=torch.float32, device=grads.list.device) if norm is None else norm
    _vector(norm, "gear_clip_grads", "norm", torch.float32, 1)
    _check(lib.gear_clip_grads(_ptr(grads.list), len(grads.grads), grads.chunks, max_norm, _ptr(grads.workspace), grads.workspace.numel(),
                               _ptr(norm), _stream()), "gear_clip_grads")
    return norm
