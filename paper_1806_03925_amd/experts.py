"""The operators of a Dense Part made of experts (include/gear.h) on PyTorch tensors: argument checks, output and workspace
memory, marshalling.  Matrices are [rows x width] with neighbouring columns next to each other; rows may lie further apart.
All tensors of a call are on the current GPU.  Calls enqueue on its current stream and do not synchronise.

These calls are no part of PyTorch's autograd: results have no history, also where an input requires a gradient.  Gradients
are calls of their own (gear_rmsnorm_backward, gear_expert_dgrad, gear_expert_wgrad) that the program puts together."""
from __future__ import annotations

import bisect
import ctypes as C
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from .binding import (GEAR_BF16, GEAR_E4M3, GEAR_ERR_INVALID, GEAR_F32, GearError, _check, _ptr, gear_expert_args,
                      gear_expert_wgrad_args, gear_grad_tensor, gear_norm_args, gear_norm_backward_args, lib)

_CODE = {torch.float32: GEAR_F32, torch.bfloat16: GEAR_BF16}
_BYTE = (torch.uint8, torch.float8_e4m3fn)
_raw_stream = torch._C._cuda_getCurrentRawStream   # of current_stream(), without the object around it: these calls are short
_current_gpu = torch._C._cuda_getDevice            # asked for once there is a tensor on a GPU


def _refuse(where: str, what: str) -> None:
    raise GearError(GEAR_ERR_INVALID, f"{where}: {what}")


def _need(ok: bool, where: str, what: str) -> None:
    if not ok:
        _refuse(where, what)


def _gpu(index: int, where: str, name: str) -> int:
    """The GPU of a call, whose tensors all have to be on it: the current one, as kernels run there."""
    if index < 0 or index != _current_gpu():
        _refuse(where, f"{name} has to be on the current GPU")
    return index


def _matrix(t: torch.Tensor, gpu: int, where: str, name: str, dtype: Optional[torch.dtype] = None, shape=None) -> int:
    """Checks a matrix and returns the distance between its rows."""
    size = t.shape
    if t.get_device() != gpu or len(size) != 2 or (t.dtype is not dtype if dtype is not None else t.dtype not in _CODE):
        _refuse(where, f"{name} has to be a matrix on GPU {gpu} of {dtype or 'float32 or bfloat16'}")
    if shape is not None and size != shape:
        _refuse(where, f"{name} has to be {tuple(shape)}, not {tuple(size)}")
    apart = t.stride()
    if apart[1] != 1 and size[1] > 1:
        _refuse(where, f"{name}'s columns have to lie next to each other")
    return apart[0] if size[0] > 1 else size[1]


def _vector(t: torch.Tensor, gpu: int, where: str, name: str, dtype: torch.dtype, n: int) -> None:
    if t.get_device() != gpu or t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _refuse(where, f"{name} has to be {n} contiguous {dtype} on GPU {gpu}")


_words = {}      # GPU -> the word that calls without a status of their own report into, and its address


def _word(index: int, where: str) -> Tuple[torch.Tensor, int]:
    found = _words.get(index)
    if found is None:
        if torch.cuda.is_current_stream_capturing():
            _refuse(where, "the first report of this GPU cannot be made while a graph is captured: give it a status, or call gear_expert_status before")
        with torch.inference_mode(False):
            word = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", index))
        torch.cuda.current_stream(index).synchronize()      # any stream may report from now on
        found = _words.setdefault(index, (word, word.data_ptr()))
    return found


def gear_expert_status(device=None) -> torch.Tensor:
    """The word [1] (int32) of a GPU that products and weight gradients report into when they are given no status: GEAR_ERR_RANGE
    once offsets were no list of rows, until the caller clears it (zero_()); 0 before.  Calls that work leave it alone, so any
    streams share it."""
    device = torch.device("cuda" if device is None else device)
    return _word(torch.cuda.current_device() if device.index is None else device.index, "gear_expert_status")[0]


class Rows8:
    """Rows in 8 bits: q [rows x gear_rows8_ld(dim)] (bytes of e4m3), scale [rows x gear_scales8_ld(dim)] (exponent + 127)."""
    __slots__ = ("rows", "dim", "ld", "device", "gpu", "_q", "_scale", "_room", "p_q", "p_scale")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, dim: int):
        rows = q.shape[0] if q.dim() else 0
        if not q.is_cuda or q.dtype not in _BYTE or q.shape != (rows, (dim + 127) // 128 * 128) or not q.is_contiguous():
            _refuse("Rows8", "q has to be [rows x gear_rows8_ld(dim)] contiguous bytes on the GPU")
        if scale.device != q.device or scale.dtype is not torch.uint8 or scale.shape != (rows, (dim + 511) // 512 * 4) or not scale.is_contiguous():
            _refuse("Rows8", "scale has to be [rows x gear_scales8_ld(dim)] contiguous bytes on q's GPU")
        self.rows, self.dim, self.ld, self.device, self.gpu = rows, dim, q.shape[1], q.device, q.get_device()
        self._q, self._scale, self._room, self.p_q, self.p_scale = q, scale, None, q.data_ptr(), scale.data_ptr()

    @staticmethod
    def empty(rows: int, dim: int, device) -> "Rows8":
        """One allocation for both; the tensors are made when somebody asks for them."""
        r = object.__new__(Rows8)
        r.rows, r.dim, r.ld, r.device, r.gpu = rows, dim, (dim + 127) // 128 * 128, device, device.index
        r._q = r._scale = None
        r._room = torch.empty(rows * (r.ld + (dim + 511) // 512 * 4), dtype=torch.uint8, device=device)
        r.p_q = r._room.data_ptr()
        r.p_scale = r.p_q + rows * r.ld
        return r

    @property
    def q(self) -> torch.Tensor:
        if self._q is None:
            self._q = self._room[:self.rows * self.ld].view(torch.float8_e4m3fn).view(self.rows, self.ld)
        return self._q

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            self._scale = self._room[self.rows * self.ld:].view(self.rows, (self.dim + 511) // 512 * 4)
        return self._scale


class NormOutput(NamedTuple):
    sum: Optional[torch.Tensor]     # x + residual; None without a residual
    y: Optional[torch.Tensor]
    rows8: Optional[Rows8]


def gear_rmsnorm(x: torch.Tensor, gain: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None, y: bool = True,
                 q8: bool = False, out: Optional[NormOutput] = None) -> NormOutput:
    """Norm of h = x + residual: the sum (where there is a residual), the norm times gain (`y`), the same in 8 bits (`q8`).
    out: memory for the results (any of its fields may be None) instead of new tensors; sum may be residual or x itself."""
    where = "gear_rmsnorm"
    gpu = _gpu(x.get_device(), where, "x")
    ld_x = _matrix(x, gpu, where, "x")
    dtype, device, shape = x.dtype, x.device, x.shape
    rows, dim = shape
    _vector(gain, gpu, where, "gain", torch.float32, dim)
    o_sum, o_y, r8 = out if out is not None else (None, None, None)
    p_res = p_sum = p_y = p_q = p_scale = None
    ld_r = ld_s = ld_y = 0
    if residual is not None:
        ld_r, p_res = _matrix(residual, gpu, where, "residual", dtype, shape), residual.data_ptr()
    if o_sum is not None:
        ld_s, p_sum = _matrix(o_sum, gpu, where, "sum", dtype, shape), o_sum.data_ptr()
    elif residual is not None:
        o_sum = torch.empty_like(x) if x.is_contiguous() else x.new_empty(shape)
        ld_s, p_sum = dim, o_sum.data_ptr()
    if not y:
        o_y = None
    elif o_y is not None:
        ld_y, p_y = _matrix(o_y, gpu, where, "y", dtype, shape), o_y.data_ptr()
    else:
        o_y = torch.empty_like(x) if x.is_contiguous() else x.new_empty(shape)
        ld_y, p_y = dim, o_y.data_ptr()
    if not q8:
        r8 = None
    else:
        if r8 is None:
            r8 = Rows8.empty(rows, dim, device)
        elif r8.dim != dim or r8.rows != rows or r8.gpu != gpu:
            _refuse(where, "rows8 has another shape than x or is on another GPU")
        p_q, p_scale = r8.p_q, r8.p_scale
    a = gear_norm_args(rows, dim, _CODE[dtype], eps, x.data_ptr(), p_res, gain.data_ptr(), p_sum, p_y, ld_x, ld_r, ld_s, ld_y, p_q, p_scale)
    code = lib.gear_rmsnorm(C.byref(a), _raw_stream(gpu))
    if code:
        _check(code, where)
    return NormOutput(o_sum, o_y, r8)


def gear_rmsnorm_backward(h: torch.Tensor, gain: torch.Tensor, dy: torch.Tensor, eps: float, dsum: Optional[torch.Tensor] = None,
                          dx: Optional[torch.Tensor] = None, dgain: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dgain) of the norm at h, dsum (what flows into the sum itself) added to dx; dx may be dy or dsum."""
    where = "gear_rmsnorm_backward"
    gpu = _gpu(h.get_device(), where, "h")
    dtype, device, shape = h.dtype, h.device, h.shape
    ld_h, ld_dy = _matrix(h, gpu, where, "h"), _matrix(dy, gpu, where, "dy", dtype, shape)
    rows, dim = shape
    _vector(gain, gpu, where, "gain", torch.float32, dim)
    ld_ds = _matrix(dsum, gpu, where, "dsum", dtype, shape) if dsum is not None else 0
    if dx is None:
        dx, ld_dx = torch.empty_like(h) if h.is_contiguous() else h.new_empty(shape), dim
    else:
        ld_dx = _matrix(dx, gpu, where, "dx", dtype, shape)
    if dgain is None:
        dgain = torch.empty_like(gain)
    else:
        _vector(dgain, gpu, where, "dgain", torch.float32, dim)
    size = lib.gear_norm_backward_workspace_bytes(rows, dim)
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    a = gear_norm_backward_args(rows, dim, _CODE[dtype], eps, h.data_ptr(), dy.data_ptr(), _ptr(dsum), gain.data_ptr(), dx.data_ptr(),
                                dgain.data_ptr(), ld_h, ld_dy, ld_ds, ld_dx)
    code = lib.gear_rmsnorm_backward(C.byref(a), ws.data_ptr(), size, _raw_stream(gpu))
    if code:
        _check(code, where)
    return dx, dgain


def gear_rows8(x: torch.Tensor, out: Optional[Rows8] = None) -> Rows8:
    """x in 8 bits, a scale for every row and 128 columns."""
    where = "gear_rows8"
    gpu = _gpu(x.get_device(), where, "x")
    ld = _matrix(x, gpu, where, "x")
    rows, dim = x.shape
    if out is None:
        out = Rows8.empty(rows, dim, x.device)
    elif out.dim != dim or out.rows != rows or out.gpu != gpu:
        _refuse(where, "out has another shape than x or is on another GPU")
    _check(lib.gear_rows8(x.data_ptr(), _CODE[x.dtype], ld, rows, dim, out.p_q, out.p_scale, _raw_stream(gpu)), where)
    return out


def _weights(w: torch.Tensor, where: str) -> Tuple[int, int, int]:
    _gpu(w.get_device(), where, "w")
    if w.dim() not in (2, 3) or w.dtype not in _CODE or not w.is_contiguous():
        _refuse(where, "w has to be contiguous [experts x N x K] or [N x K], float32 or bfloat16")
    return (1, *w.shape) if len(w.shape) == 2 else tuple(w.shape)


class _Packed:
    """Memory of weights laid out for the products."""

    def _allocate(self, size: int, device) -> None:
        self.gpu = device.index
        self.packed = torch.empty(size, dtype=torch.uint8, device=device)
        self.address = self.packed.data_ptr()
        if self.gpu not in _words and not torch.cuda.is_current_stream_capturing():
            _word(self.gpu, "weights")                  # there when products are captured

    @property
    def status(self) -> torch.Tensor:
        """gear_expert_status of the weights' GPU."""
        return gear_expert_status(self.packed.device)


class Weights8(_Packed):
    """Weights in 8 bits, laid out for gear_matmul8 (gear_weights8 makes them)."""

    def __init__(self, w: torch.Tensor):
        where = "gear_weights8"
        self.experts, self.N, self.K = shape = _weights(w, where)
        size, scales = lib.gear_packed_weights_bytes(GEAR_E4M3, *shape, 0), lib.gear_weight_scales_bytes(*shape)
        if size == 0:
            _refuse(where, f"weights of {shape} have no packed form")
        self._allocate(size + scales, w.device)
        self.p_scale = self.address + size
        _check(lib.gear_pack_weights(w.data_ptr(), _CODE[w.dtype], GEAR_E4M3, *shape, self.address, None, self.p_scale,
                                     _raw_stream(self.gpu)), where)


def gear_weights8(w: torch.Tensor) -> Weights8:
    """w ([experts x N x K] or [N x K], float32 or bfloat16) in 8 bits, a scale for every 128 x 128 weights."""
    return Weights8(w)


class ExpertWeights(_Packed):
    """Weights of every expert laid out for the forward product and (transposed) for the gradient of its input, in float32
    or bfloat16 (`operand`, w's own type if not given).  A training program calls update() when the weights have changed."""

    def __init__(self, w: torch.Tensor, operand: Optional[torch.dtype] = None, backward: bool = True):
        where = "ExpertWeights"
        self.experts, self.N, self.K = shape = _weights(w, where)
        self.dtype = operand or w.dtype
        if self.dtype not in _CODE:
            _refuse(where, "operand has to be float32 or bfloat16")
        self.code = _CODE[self.dtype]
        forward = lib.gear_packed_weights_bytes(self.code, *shape, 0)
        size = forward + (lib.gear_packed_weights_bytes(self.code, *shape, 1) if backward else 0)
        if forward == 0:
            _refuse(where, f"weights of {shape} have no packed form")
        self._allocate(size, w.device)
        self.forward = self.address
        self.transposed = self.forward + forward if backward else None
        self._lay_out(w)

    def _lay_out(self, w: torch.Tensor) -> None:
        code = lib.gear_pack_weights(w.data_ptr(), _CODE[w.dtype], self.code, self.experts, self.N, self.K, self.forward, self.transposed, None,
                                     _raw_stream(self.gpu))
        if code:
            _check(code, "ExpertWeights")

    def update(self, w: torch.Tensor) -> None:
        if _weights(w, "ExpertWeights.update") != (self.experts, self.N, self.K) or w.get_device() != self.gpu:
            _refuse("ExpertWeights.update", "w has another shape than before or is on another GPU")
        self._lay_out(w)


def _product(where, dtype, p_x, p_x_scale, ld_x, weights, packed, p_w_scale, rows, n, k, off, out, out_dtype, status, gpu) -> torch.Tensor:
    experts = weights.experts
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
        out, ld_out = torch.empty(rows, n, dtype=out_dtype, device=gpu), n
    else:
        ld_out = _matrix(out, gpu, where, "out", None, (rows, n))
    a = gear_expert_args(dtype, _CODE[out.dtype], rows, k, n, experts, p_x, p_x_scale, packed, p_w_scale, off, out.data_ptr(), ld_x, ld_out,
                         status, keep)
    code = lib.gear_expert_product(C.byref(a), _raw_stream(gpu))
    if code:
        _check(code, where)
    return out


def gear_matmul8(rows8: Rows8, weights: Weights8, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 out_dtype: torch.dtype = torch.bfloat16, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rows8 times the transposed 8-bit weights.  off [experts + 1] (int32, on the GPU): where each expert's rows begin; rows
    from off[experts] on are not written.  status [1] (int32): GEAR_ERR_RANGE if off is no such list, and nothing is written,
    otherwise 0; without it the error is left in gear_expert_status.  Sums of eight neighbouring columns keep fewer bits than
    fp32 (include/gear.h): 1.5e-5 of the result, which out_dtype=float32 shows."""
    gpu = _gpu(rows8.gpu, "gear_matmul8", "rows8")
    if rows8.dim != weights.K:
        _refuse("gear_matmul8", f"rows of {rows8.dim} for weights of {weights.K}")
    return _product("gear_matmul8", GEAR_E4M3, rows8.p_q, rows8.p_scale, rows8.ld, weights, weights.address, weights.p_scale, rows8.rows,
                    weights.N, weights.K, off, out, out_dtype, status, gpu)


def gear_expert_matmul(x: torch.Tensor, weights: ExpertWeights, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows x K] times the transposed weights of each row's expert: [rows x N]; off and status as for gear_matmul8."""
    where = "gear_expert_matmul"
    gpu = _gpu(x.get_device(), where, "x")
    ld = _matrix(x, gpu, where, "x", weights.dtype)
    rows, k = x.shape
    if k != weights.K:
        _refuse(where, f"rows of {k} for weights of {weights.K}")
    return _product(where, weights.code, x.data_ptr(), None, ld, weights, weights.forward, None, rows, weights.N, k, off, out,
                    out_dtype or weights.dtype, status, gpu)


def gear_expert_dgrad(dy: torch.Tensor, weights: ExpertWeights, off: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      out_dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dy [rows x N] times the weights of each row's expert: the gradient [rows x K] of gear_expert_matmul's x."""
    where = "gear_expert_dgrad"
    gpu = _gpu(dy.get_device(), where, "dy")
    ld = _matrix(dy, gpu, where, "dy", weights.dtype)
    rows, n = dy.shape
    if n != weights.N:
        _refuse(where, f"rows of {n} for weights of {weights.N} outputs")
    if weights.transposed is None:
        _refuse(where, "the weights were laid out without backward")
    return _product(where, weights.code, dy.data_ptr(), None, ld, weights, weights.transposed, None, rows, weights.K, n, off, out,
                    out_dtype or weights.dtype, status, gpu)


def gear_expert_wgrad(dy: torch.Tensor, x: torch.Tensor, off: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                      status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dy_e^T x_e for every expert: [experts x N x K] float32, zeros for one without rows.  off as for gear_matmul8; status [1]
    (int32): GEAR_ERR_RANGE if it is no such list, and nothing is written, otherwise 0; without it the error is left in
    gear_expert_status."""
    where = "gear_expert_wgrad"
    gpu = _gpu(x.get_device(), where, "x")
    ld_x = _matrix(x, gpu, where, "x")
    ld_dy = _matrix(dy, gpu, where, "dy", x.dtype)
    rows, k = x.shape
    rows_dy, n = dy.shape
    if rows_dy != rows:
        _refuse(where, f"dy has {rows_dy} rows and x {rows}")
    experts = 1
    if off is not None:
        experts = off.numel() - 1
        if experts < 1:
            _refuse(where, "off has to hold a begin and an end at least")
        _vector(off, gpu, where, "off", torch.int32, experts + 1)
    keep, p_status = 0, None
    if status is not None:
        _vector(status, gpu, where, "status", torch.int32, 1)
        p_status = status.data_ptr()
    elif off is not None:
        p_status, keep = _word(gpu, where)[1], 1
    if dw is None:
        dw = torch.empty(experts, n, k, dtype=torch.float32, device=gpu)
    else:
        _vector(dw, gpu, where, "dw", torch.float32, experts * n * k)
    dtype = _CODE[x.dtype]
    size = lib.gear_expert_wgrad_workspace_bytes(dtype, rows, experts, n, k)
    ws = torch.empty(size, dtype=torch.uint8, device=gpu)
    a = gear_expert_wgrad_args(dtype, rows, k, n, experts, dy.data_ptr(), x.data_ptr(), _ptr(off), dw.data_ptr(), ld_dy, ld_x,
                               p_status, keep)
    code = lib.gear_expert_wgrad(C.byref(a), ws.data_ptr(), size, _raw_stream(gpu))
    if code:
        _check(code, where)
    return dw


def _share_memory(src: Sequence[Tuple[int, int]], dst: Sequence[Tuple[int, int]]) -> bool:
    """Whether a range (address, bytes) of dst meets another one of dst, or one of src other than all of its own."""
    at = sorted((a, a + n, i) for i, (a, n) in enumerate(dst) if n > 0)
    if any(a[1] > b[0] for a, b in zip(at, at[1:])):
        return True
    ends = [a[1] for a in at]
    for i, (a, n) in enumerate(src):
        k = bisect.bisect_right(ends, a)
        while n > 0 and k < len(at) and at[k][0] < a + n:
            if at[k] != (a, a + n, i):
                return True
            k += 1
    return False


class GradList:
    """A list of gradients for gear_grad_norm and gear_clip_grads; `out` (the tensors that receive the clipped gradients) is
    the gradients themselves unless given.  Holds for as long as the tensors keep their memory: build it once, or again when
    a gradient has been replaced.  Elements that two workgroups would scale, or one reads while another writes them, are
    refused: list a tensor that is used twice once.  (Without `out` such a list has its norm, but cannot be clipped.)  Calls
    on one list share its workspace: they come one after another."""

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        where = "GradList"
        _need(len(grads) > 0 and (out is None or len(out) == len(grads)), where, "a list of tensors, and as many to receive them")
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        self.gpu = _gpu(self.grads[0].get_device(), where, "the first gradient")
        entries = (gear_grad_tensor * len(self.grads))()
        for e, g, o in zip(entries, self.grads, self.out):
            _need(all(t.get_device() == self.gpu and t.is_contiguous() and t.dtype in _CODE for t in (g, o)) and g.dtype == o.dtype and g.numel() == o.numel(),
                  where, "contiguous float32 or bfloat16 tensors on one GPU, each as large as the one that receives it")
            e.src, e.dst, e.n, e.dtype = g.data_ptr() or None, o.data_ptr() or None, g.numel(), _CODE[g.dtype]
        where_of = lambda tensors: [(t.data_ptr(), t.numel() * t.element_size()) for t in tensors]
        self.clips = not _share_memory(where_of(self.grads), where_of(self.out))
        if not self.clips:
            _need(out is None, where, "a tensor that receives clipped gradients shares memory with another one of the list")
            for e in entries:
                e.dst = None
        host = torch.empty(lib.gear_grad_list_bytes(len(self.grads)), dtype=torch.uint8)
        chunks = C.c_int64()
        _check(lib.gear_grad_list_pack(entries, len(self.grads), host.data_ptr(), C.byref(chunks)), where)
        self.chunks = chunks.value
        self.list = host.to(self.grads[0].device)
        self.workspace = torch.empty(lib.gear_grad_workspace_bytes(self.chunks), dtype=torch.uint8, device=self.list.device)
        self.plan = (self.list.data_ptr(), len(self.grads), self.chunks), (self.workspace.data_ptr(), self.workspace.numel())


def _norm_word(norm: Optional[torch.Tensor], grads: GradList, where: str) -> torch.Tensor:
    _gpu(grads.gpu, where, "grads")
    if norm is None:
        return torch.empty((), dtype=torch.float32, device=grads.list.device)
    _vector(norm, grads.gpu, where, "norm", torch.float32, 1)
    return norm


def gear_grad_norm(grads: GradList, norm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The norm [1] of all gradients of the list together."""
    norm = _norm_word(norm, grads, "gear_grad_norm")
    what, room = grads.plan
    _check(lib.gear_grad_norm(*what, *room, norm.data_ptr(), _raw_stream(grads.gpu)), "gear_grad_norm")
    return norm


def gear_clip_grads(grads: GradList, max_norm: float, norm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scales the gradients of the list so that their norm is at most max_norm; returns the norm [1] that they had."""
    _need(grads.clips, "gear_clip_grads", "tensors of the list share memory")
    norm = _norm_word(norm, grads, "gear_clip_grads")
    what, room = grads.plan
    _check(lib.gear_clip_grads(*what, max_norm, *room, norm.data_ptr(), _raw_stream(grads.gpu)), "gear_clip_grads")
    return norm
