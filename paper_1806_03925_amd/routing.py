"""Rows that choose their experts, and products in 8-bit integers (include/gear.h), on PyTorch tensors: argument checks, output
and workspace memory, marshalling, by the rules of experts.py.  All tensors of a call are on the current GPU, calls enqueue on its
current stream and do not synchronise, and results have no autograd history: gradients are calls of their own."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import (GEAR_BF16, GEAR_F32, GEAR_I8, GEAR_SCORE_SIGMOID, GEAR_SCORE_SOFTMAX, _check, gear_expert_combine_args,
                      gear_expert_combine_backward_args, gear_i8_args, gear_route_args, gear_route_backward_args, lib)
from .experts import _CODE, _Packed, _gpu, _matrix, _raw_stream, _refuse, _vector, _weights, _word

_SIZE = {GEAR_F32: 4, GEAR_BF16: 2}
_SCORE = {"softmax": GEAR_SCORE_SOFTMAX, "sigmoid": GEAR_SCORE_SIGMOID}


class Route:
    """Where rows go.  expert [rows x k] (int32, best first; -1: none), weight [rows x k] (float32), place [rows x k] (int32: the
    pair's row in the order of experts; -1: none), off [experts + 1] (int32: where each expert's rows begin).  gear_route makes one;
    a program may put one together from tensors of its own, whose places have to be distinct."""
    __slots__ = ("rows", "k", "experts", "gpu", "p_expert", "p_weight", "p_place", "p_off", "_room", "_expert", "_weight", "_place", "_off")

    def __init__(self, expert: torch.Tensor, weight: torch.Tensor, place: torch.Tensor, off: torch.Tensor):
        where = "Route"
        self.gpu = _gpu(expert.get_device(), where, "expert")
        if expert.dim() != 2 or expert.shape[1] < 1 or off.dim() != 1 or off.numel() < 2:
            _refuse(where, "expert has to be [rows x k] and off [experts + 1]")
        self.rows, self.k = expert.shape
        self.experts = off.numel() - 1
        for t, name, dtype in ((expert, "expert", torch.int32), (weight, "weight", torch.float32), (place, "place", torch.int32)):
            if t.shape != expert.shape:
                _refuse(where, f"{name} has to be {tuple(expert.shape)}, not {tuple(t.shape)}")
            _vector(t, self.gpu, where, name, dtype, self.rows * self.k)
        _vector(off, self.gpu, where, "off", torch.int32, self.experts + 1)
        self._room = None
        self._expert, self._weight, self._place, self._off = expert, weight, place, off
        self.p_expert, self.p_weight, self.p_place, self.p_off = (t.data_ptr() for t in (expert, weight, place, off))

    @staticmethod
    def _empty(rows: int, k: int, experts: int, gpu: int, more: int) -> "Route":
        """One allocation for all four, and `more` bytes behind them on 256 bytes; the tensors are made when somebody asks for them."""
        r = object.__new__(Route)
        r.rows, r.k, r.experts, r.gpu = rows, k, experts, gpu
        r._expert = r._weight = r._place = r._off = None
        r._room = room = torch.empty((3 * rows * k + experts + 64 & -64) + more // 4, dtype=torch.int32, device=gpu)
        r.p_expert = p = room.data_ptr()
        step = 4 * rows * k
        r.p_weight, r.p_place, r.p_off = p + step, p + 2 * step, p + 3 * step
        return r

    def _part(self, i: int) -> torch.Tensor:
        k = self.k
        return self._room.as_strided((self.rows, k), (k, 1), i * self.rows * k)

    @property
    def expert(self) -> torch.Tensor:
        if self._expert is None:
            self._expert = self._part(0)
        return self._expert

    @property
    def weight(self) -> torch.Tensor:
        if self._weight is None:
            self._weight = self._part(1).view(torch.float32)
        return self._weight

    @property
    def place(self) -> torch.Tensor:
        if self._place is None:
            self._place = self._part(2)
        return self._place

    @property
    def off(self) -> torch.Tensor:
        if self._off is None:
            self._off = self._room.as_strided((self.experts + 1,), (1,), 3 * self.rows * self.k)
        return self._off


def _logits(t: torch.Tensor, where: str, name: str, dtype=None, shape=None) -> int:
    """Checks a matrix of logits, of any width, and returns the distance between its rows."""
    return _matrix(t, _gpu(t.get_device(), where, name), where, name, dtype, shape)


class _Lines(NamedTuple):
    """Where a matrix lies, in bytes: `rows` lines of `width`, `apart` from one to the next."""
    at: int
    rows: int
    apart: int
    width: int


def _lines(t: torch.Tensor, ld: int) -> _Lines:
    size = t.element_size()
    return _Lines(t.data_ptr(), t.shape[0], ld * size, t.shape[1] * size)


def _apart(out: _Lines, other: _Lines, where: str, what: str, itself: bool = False) -> None:
    """Refuses memory for a result that holds what the call reads: workgroups come in any order.  Columns of one matrix beside each other
    are apart; itself: out may be the other one."""
    if not out.rows or not other.rows or (itself and out == other):
        return
    if out.at + (out.rows - 1) * out.apart + out.width <= other.at or other.at + (other.rows - 1) * other.apart + other.width <= out.at:
        return
    between = (other.at - out.at) % out.apart if out.apart else 0
    if out.apart != other.apart or between < out.width or between + other.width > out.apart:
        _refuse(where, what)


def _clear_of(out: _Lines, where: str, what: str, *words: Tuple[Optional[int], int]) -> None:
    """Refuses memory for a result that holds any of `words`, (address, bytes) each; an address of None or 0 is nothing."""
    end = out.at + out.rows * out.apart
    for at, size in words:
        if at and at < end and out.at < at + size:     # else they are far apart: these calls are short
            _apart(out, _Lines(at, 1, size, size), where, what)


def gear_route(logits: torch.Tensor, k: int, score: str = "softmax", bias: Optional[torch.Tensor] = None, groups: int = 1, groups_kept: int = 1,
               group_best: int = 1, renormalise: bool = True, scale: float = 1.0, n: Optional[torch.Tensor] = None) -> Route:
    """The k experts of every row of logits [rows x experts] (float32 or bfloat16), their weights, and the order of all pairs by
    expert.  score: "softmax" or "sigmoid" of the logits.  bias [experts] (float32) is added to the scores for the choice, not for
    the weights.  groups > 1: experts come in groups, of which the groups_kept best may be chosen from, by the sum of their
    group_best (1 or 2) best.  renormalise: weights are divided by their sum.  n [1] (int32): rows from n on are padding and go
    nowhere.  Experts with a logit or bias of -inf are not chosen (include/gear.h has all of the definition)."""
    where = "gear_route"
    ld = _logits(logits, where, "logits")
    rows, experts = logits.shape
    gpu = logits.get_device()
    code = _SCORE.get(score)
    if code is None:
        _refuse(where, f"score has to be softmax or sigmoid, not {score}")
    if bias is not None:
        _vector(bias, gpu, where, "bias", torch.float32, experts)
        bias = bias.data_ptr()
    if n is not None:
        _vector(n, gpu, where, "n", torch.int32, 1)
        n = n.data_ptr()
    size = lib.gear_route_workspace_bytes(rows, experts, k, groups)
    if size == 0:
        _refuse(where, f"{k} of {experts} experts in {groups} groups for {rows} rows")
    r = Route._empty(rows, k, experts, gpu, size)
    a = gear_route_args(rows, experts, k, _CODE[logits.dtype], code, groups, groups_kept, group_best, 1 if renormalise else 0, scale,
                        logits.data_ptr(), ld, bias, n, r.p_expert, r.p_weight, r.p_off, r.p_place)
    status = lib.gear_route(C.byref(a), r.p_off + 4 * experts + 259 & -256, size, _raw_stream(gpu))
    if status:
        _check(status, where)
    return r


def gear_route_backward(logits: torch.Tensor, route: Route, dweight: torch.Tensor, score: str = "softmax", renormalise: bool = True,
                        scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient [rows x experts] of the logits from that of the route's weights; score, renormalise and scale as gear_route had
    them.  `out` shares no memory with what is read."""
    where = "gear_route_backward"
    ld = _logits(logits, where, "logits")
    gpu, dtype, shape = logits.get_device(), logits.dtype, logits.shape
    rows, experts = shape
    if route.rows != rows or route.experts != experts or route.gpu != gpu:
        _refuse(where, "the route is of other logits")
    code = _SCORE.get(score)
    if code is None:
        _refuse(where, f"score has to be softmax or sigmoid, not {score}")
    _vector(dweight, gpu, where, "dweight", torch.float32, rows * route.k)
    if out is None:
        out, ld_out = torch.empty(shape, dtype=dtype, device=gpu), experts
    else:
        ld_out = _matrix(out, gpu, where, "out", dtype, shape)
        lines = _lines(out, ld_out)
        _apart(lines, _lines(logits, ld), where, "out may not share memory with the logits")
        words = 4 * rows * route.k
        for p in (dweight.data_ptr(), route.p_weight, route.p_expert):
            _apart(lines, _Lines(p, 1, words, words), where, "out may not share memory with dweight or the route")
    a = gear_route_backward_args(rows, experts, route.k, _CODE[dtype], code, 1 if renormalise else 0, scale, logits.data_ptr(), ld, route.p_expert,
                                 route.p_weight, dweight.data_ptr(), out.data_ptr(), ld_out)
    status = lib.gear_route_backward(C.byref(a), _raw_stream(gpu))
    if status:
        _check(status, where)
    return out


def _of_route(t: torch.Tensor, route: Route, rows: int, where: str, name: str, dtype=None, dim: Optional[int] = None) -> int:
    """Checks a matrix of `rows` rows on the route's GPU, and returns the distance between its rows."""
    size = t.shape
    if len(size) == 2 and (size[0] != rows or (dim is not None and size[1] != dim)):
        _refuse(where, f"{name} has to be {(rows, dim if dim is not None else size[1])}, not {tuple(size)}")
    return _matrix(t, route.gpu, where, name, dtype)


def gear_expert_gather(x: torch.Tensor, route: Route, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows x dim] copied to every place that the route gives its rows: [rows * k x dim] for gear_expert_matmul with route.off.  Rows
    from route.off[experts] on are not written.  Its gradient is gear_expert_combine(dxs, route, weighted=False)."""
    where = "gear_expert_gather"
    _gpu(route.gpu, where, "the route")
    ld = _of_route(x, route, route.rows, where, "x")
    dim, places, p_x, code = x.shape[1], route.rows * route.k, x.data_ptr(), _CODE[x.dtype]
    if out is None:
        out, ld_out = torch.empty(places, dim, dtype=x.dtype, device=route.gpu), dim
    else:
        ld_out = _of_route(out, route, places, where, "out", x.dtype, dim)
        p_out, size = out.data_ptr(), _SIZE[code]
        if p_out < p_x + route.rows * ld * size and p_x < p_out + places * ld_out * size:     # else they are far apart: these calls are short
            _apart(_lines(out, ld_out), _lines(x, ld), where, "out may not share memory with x")
        if p_out < route.p_place + 4 * places and route.p_place < p_out + places * ld_out * size:
            _clear_of(_lines(out, ld_out), where, "out may not share memory with the route", (route.p_place, 4 * places))
    status = lib.gear_expert_gather(p_x, code, ld, route.rows, dim, route.p_place, route.k, out.data_ptr(), ld_out, _raw_stream(route.gpu))
    if status:
        _check(status, where)
    return out


def gear_expert_combine(y: torch.Tensor, route: Route, weighted: bool = True, residual: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The way back: residual + the sum of the rows' places in y [rows * k x dim], each times its weight (weighted=False: 1).  out
    may be residual itself.  Both are of y's type, or bfloat16 for y in float32 where out_dtype says so: products in float32 are then rounded
    once, in the sum, and not each before it."""
    where = "gear_expert_combine"
    _gpu(route.gpu, where, "the route")
    rows, places = route.rows, route.rows * route.k
    ld_y = _of_route(y, route, places, where, "y")
    dim = y.shape[1]
    dtype = out_dtype or y.dtype
    y_f32 = dtype is not y.dtype
    if y_f32 and (dtype is not torch.bfloat16 or y.dtype is not torch.float32):
        _refuse(where, f"out_dtype has to be y's type, or bfloat16 for y in float32, not {dtype} for {y.dtype}")
    ld_r, p_r = 0, None
    if residual is not None:
        ld_r, p_r = _of_route(residual, route, rows, where, "residual", dtype, dim), residual.data_ptr()
    if out is None:
        out, ld_out = torch.empty(rows, dim, dtype=dtype, device=route.gpu), dim
    else:
        ld_out = _of_route(out, route, rows, where, "out", dtype, dim)
        lines = _lines(out, ld_out)
        _apart(lines, _lines(y, ld_y), where, "out may not share memory with y")
        if residual is not None:
            _apart(lines, _lines(residual, ld_r), where, "out may be residual itself, but not share a part of its memory", True)
        _clear_of(lines, where, "out may not share memory with the route", (route.p_place, 4 * places), (route.p_weight if weighted else None, 4 * places))
    a = gear_expert_combine_args(rows, dim, route.k, _CODE[dtype], y_f32, y.data_ptr(), p_r, route.p_place, route.p_weight if weighted else None,
                                 out.data_ptr(), ld_y, ld_r, ld_out)
    status = lib.gear_expert_combine(C.byref(a), _raw_stream(route.gpu))
    if status:
        _check(status, where)
    return out


def gear_expert_combine_backward(dout: torch.Tensor, y: torch.Tensor, route: Route, dy: Optional[torch.Tensor] = None,
                                 dweight: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dy, dweight) of gear_expert_combine with weights: dy [rows * k x dim], of which rows from route.off[experts] on are not
    written (dy may be y itself), and dweight [rows x k] (float32).  y is of dout's type, also where the sum took it in float32.  The residual's
    gradient is dout."""
    where = "gear_expert_combine_backward"
    _gpu(route.gpu, where, "the route")
    rows, places = route.rows, route.rows * route.k
    ld_dout = _of_route(dout, route, rows, where, "dout")
    dtype, dim = dout.dtype, dout.shape[1]
    code = _CODE[dtype]
    ld_y = _of_route(y, route, places, where, "y", dtype, dim)
    if dy is None:
        dy, ld_dy = torch.empty(places, dim, dtype=dtype, device=route.gpu), dim
    else:
        ld_dy = _of_route(dy, route, places, where, "dy", dtype, dim)
        size = _SIZE[code]
        p_dy, p_dout, p_y, n = dy.data_ptr(), dout.data_ptr(), y.data_ptr(), places * ld_dy * size
        if p_dy < p_dout + rows * ld_dout * size and p_dout < p_dy + n:
            _apart(_lines(dy, ld_dy), _lines(dout, ld_dout), where, "dy may not share memory with dout")
        if p_dy < p_y + places * ld_y * size and p_y < p_dy + n:
            _apart(_lines(dy, ld_dy), _lines(y, ld_y), where, "dy may be y itself, but not share a part of its memory", True)
        for p in (route.p_place, route.p_weight):
            if p_dy < p + 4 * places and p < p_dy + n:
                _clear_of(_lines(dy, ld_dy), where, "dy may not share memory with the route", (p, 4 * places))
    if dweight is None:
        dweight = torch.empty(rows, route.k, dtype=torch.float32, device=route.gpu)
    else:
        _vector(dweight, route.gpu, where, "dweight", torch.float32, places)
        lines = _Lines(dweight.data_ptr(), 1 if places else 0, 4 * places, 4 * places)
        for other in (_lines(dout, ld_dout), _lines(y, ld_y), _lines(dy, ld_dy), lines._replace(at=route.p_weight), lines._replace(at=route.p_place)):
            _apart(lines, other, where, "dweight may not share memory with another matrix or the route")
    a = gear_expert_combine_backward_args(rows, dim, route.k, code, dout.data_ptr(), y.data_ptr(), route.p_place, route.p_weight, dy.data_ptr(),
                                          dweight.data_ptr(), ld_dout, ld_y, ld_dy)
    status = lib.gear_expert_combine_backward(C.byref(a), _raw_stream(route.gpu))
    if status:
        _check(status, where)
    return dy, dweight


# ---- 8-bit integers ---------------------------------------------------------------------------------------------------
class RowsI8:
    """Rows in 8-bit integers: q [rows x gear_rows8_ld(dim)] (int8, zeros behind a row's end), scale [rows] (float32)."""
    __slots__ = ("rows", "dim", "ld", "gpu", "_q", "_scale", "_room", "p_q", "p_scale")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, dim: int):
        where = "RowsI8"
        self.gpu = _gpu(q.get_device(), where, "q")
        rows = q.shape[0] if q.dim() else 0
        if q.dtype is not torch.int8 or dim < 1 or q.shape != (rows, (dim + 127) // 128 * 128) or not q.is_contiguous():
            _refuse(where, "q has to be [rows x gear_rows8_ld(dim)] contiguous int8")
        _vector(scale, self.gpu, where, "scale", torch.float32, rows)
        _apart(_Lines(q.data_ptr(), 1, q.numel(), q.numel()), _Lines(scale.data_ptr(), 1, 4 * rows, 4 * rows), where, "scale may not share memory with q")
        self.rows, self.dim, self.ld = rows, dim, q.shape[1]
        self._q, self._scale, self._room, self.p_q, self.p_scale = q, scale, None, q.data_ptr(), scale.data_ptr()

    @staticmethod
    def empty(rows: int, dim: int, gpu: int) -> "RowsI8":
        """One allocation for both; the tensors are made when somebody asks for them."""
        r = object.__new__(RowsI8)
        r.rows, r.dim, r.ld, r.gpu = rows, dim, (dim + 127) // 128 * 128, gpu
        r._q = r._scale = None
        r._room = torch.empty(rows * (r.ld + 4), dtype=torch.int8, device=gpu)
        r.p_q = r._room.data_ptr()
        r.p_scale = r.p_q + rows * r.ld
        return r

    @property
    def q(self) -> torch.Tensor:
        if self._q is None:
            self._q = self._room[:self.rows * self.ld].view(self.rows, self.ld)
        return self._q

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            self._scale = self._room[self.rows * self.ld:].view(torch.float32)
        return self._scale


def _rows_i8(x: torch.Tensor, ld: int, rows: int, place: Optional[int], k: int, out: Optional[RowsI8], gpu: int, where: str) -> RowsI8:
    dim = x.shape[1]
    if out is None:
        out = RowsI8.empty(rows * k, dim, gpu)
    elif out.dim != dim or out.rows != rows * k or out.gpu != gpu:
        _refuse(where, "out has another shape than the rows or is on another GPU")
    else:
        lines = _lines(x, ld)
        for mine in (_Lines(out.p_q, out.rows, out.ld, out.ld), _Lines(out.p_scale, 1, 4 * out.rows, 4 * out.rows)):
            _apart(mine, lines, where, "out may not share memory with x")
            _clear_of(mine, where, "out may not share memory with the route", (place, 4 * rows * k))
    status = lib.gear_rows_i8(x.data_ptr(), _CODE[x.dtype], ld, rows, dim, place, k, out.p_q, out.p_scale, _raw_stream(gpu))
    if status:
        _check(status, where)
    return out


def gear_rows_i8(x: torch.Tensor, out: Optional[RowsI8] = None) -> RowsI8:
    """x [rows x dim] in 8-bit integers, a scale for every row."""
    where = "gear_rows_i8"
    gpu = _gpu(x.get_device(), where, "x")
    return _rows_i8(x, _matrix(x, gpu, where, "x"), x.shape[0], None, 1, out, gpu, where)


def gear_expert_gather_i8(x: torch.Tensor, route: Route, out: Optional[RowsI8] = None) -> RowsI8:
    """gear_expert_gather and gear_rows_i8 in one: rows from route.off[experts] on are not written."""
    where = "gear_expert_gather_i8"
    _gpu(route.gpu, where, "the route")
    ld = _of_route(x, route, route.rows, where, "x")
    return _rows_i8(x, ld, route.rows, route.p_place, route.k, out, route.gpu, where)


class WeightsI8(_Packed):
    """Weights in 8-bit integers with a scale [experts x N] for every output, laid out for gear_matmul_i8 (gear_weights_i8 makes them)."""

    def __init__(self, w: torch.Tensor, scale: Optional[torch.Tensor] = None):
        where = "gear_weights_i8"
        if scale is None:
            self.experts, self.N, self.K = shape = _weights(w, where)
            code = _CODE[w.dtype]
        else:
            _gpu(w.get_device(), where, "w")
            if w.dim() not in (2, 3) or w.dtype is not torch.int8 or not w.is_contiguous():
                _refuse(where, "w with a scale has to be contiguous int8 [experts x N x K] or [N x K]")
            self.experts, self.N, self.K = shape = (1, *w.shape) if w.dim() == 2 else tuple(w.shape)
            _vector(scale, w.get_device(), where, "scale", torch.float32, shape[0] * shape[1])
            code = GEAR_I8
        size = lib.gear_packed_i8_bytes(*shape)
        if size == 0:
            _refuse(where, f"weights of {shape} have no packed form")
        self._allocate(size, w.device)
        self.scale = torch.empty(shape[:2], dtype=torch.float32, device=w.device) if scale is None else scale.reshape(shape[:2]).clone()
        self.p_scale = self.scale.data_ptr()
        _check(lib.gear_pack_weights_i8(w.data_ptr(), code, *shape, self.address, self.p_scale, _raw_stream(self.gpu)), where)


def gear_weights_i8(w: torch.Tensor, scale: Optional[torch.Tensor] = None) -> WeightsI8:
    """w ([experts x N x K] or [N x K], float32 or bfloat16) in 8-bit integers, a scale for every output; or w in int8 already, with its
    scale [experts x N]."""
    return WeightsI8(w, scale)


def gear_matmul_i8(rows: RowsI8, weights: WeightsI8, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   out_dtype: torch.dtype = torch.bfloat16, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rows times the transposed weights of each row's expert, [rows x N]: integers added up exactly, then scaled, then rounded to out_dtype;
    float32 is for what gear_expert_combine adds up.  off, status and rows from off[experts] on as for gear_matmul8.  `out` shares no memory
    with what is read."""
    where = "gear_matmul_i8"
    gpu, n, experts = _gpu(rows.gpu, where, "rows"), weights.N, weights.experts
    if rows.dim != weights.K:
        _refuse(where, f"rows of {rows.dim} for weights of {weights.K}")
    if weights.gpu != gpu:
        _refuse(where, "rows and weights are on different GPUs")
    if off is not None:
        _vector(off, gpu, where, "off", torch.int32, experts + 1)
        off = off.data_ptr()
    elif experts != 1:
        _refuse(where, "off may only be left out where there is one expert")
    keep = 0
    if status is not None:
        _vector(status, gpu, where, "status", torch.int32, 1)
        status = status.data_ptr()
    elif off is not None:
        status, keep = _word(gpu, where)[1], 1
    if out is None:
        if out_dtype not in _CODE:
            _refuse(where, f"out_dtype has to be float32 or bfloat16, not {out_dtype}")
        out, ld_out = torch.empty(rows.rows, n, dtype=out_dtype, device=gpu), n
    else:
        ld_out = _matrix(out, gpu, where, "out", None, (rows.rows, n))
        _clear_of(_lines(out, ld_out), where, "out may not share memory with what is read", (rows.p_q, rows.rows * rows.ld), (rows.p_scale, 4 * rows.rows),
                  (weights.address, weights.packed.numel()), (weights.p_scale, 4 * experts * n), (off, 4 * (experts + 1)), (status, 4))
    a = gear_i8_args(_CODE[out.dtype], rows.rows, weights.K, n, experts, rows.p_q, rows.p_scale, weights.address, weights.p_scale, off,
                     out.data_ptr(), rows.ld, ld_out, status, keep)
    code = lib.gear_product_i8(C.byref(a), _raw_stream(gpu))
    if code:
        _check(code, where)
    return out
