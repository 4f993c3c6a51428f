"""Matrices of microscaled 4-bit floating point: thin binding of the sqllm_mx_* entry points.  Checks shapes, allocates outputs, marshals the
arguments (no arithmetic here); every call enqueues on the current stream of its tensors' device.

No call here is recorded by autograd: operands may require gradients, results never do, and what is written to a given `y` or `dw` autograd does not
see.  The gradients of a layer are mx_linear_backward's, which a program calls itself, for instance in a torch.autograd.Function of its own."""
from __future__ import annotations

import torch

from . import binding

ROW = 128       # columns a packed row is padded to
MOST_ROWS, MOST_COLUMNS = 2**31 - 1, 2**31 - 128     # the library counts in 32 bits
_TYPES = {torch.float16: binding.TYPE_F16, torch.bfloat16: binding.TYPE_BF16, torch.float32: binding.TYPE_F32}


def _refuse(name, message):
    raise binding.SqllmError(binding.STATUS_NAMES.index(name), message)


def _need_size(M, N):
    if not (0 <= M <= MOST_ROWS and 0 < N <= MOST_COLUMNS):
        _refuse("SQLLM_ERR_SHAPE", f"a packed matrix of {M} x {N}")


QUANTIZE, DEQUANTIZE, GEMV, GEMM = range(4)         # entries of binding._MX_ENTRIES


def _call(device, *args):
    """binding._mx(*args, current stream of the tensors' device) with that device as the current one"""
    if device == _current_device():
        stream = _raw_stream(device)
        status = binding._mx_call(*args, stream)
        if status != 0:
            binding._mx_not_ok(status, *args, stream)
    else:
        with torch.cuda.device(device):
            binding._mx(*args, None)


# Asked for tensors that are on a GPU, so the runtime is up: without the wrappers that start it 0.3 us less.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _empty(M, N, dtype, device):
    """torch.empty((M, N)); with its strides given it takes the host 1.3 us, not 1.7"""
    return torch.empty_strided((M, N), (N, 1), dtype=dtype, device=device)


def _type_of(dtype):
    if dtype not in _TYPES:
        _refuse("SQLLM_ERR_TYPE", f"{dtype} is none of float16, bfloat16 and float32")
    return _TYPES[dtype]


def _need(t, what, like=None, dtype=None, shape=None):
    """t is on a GPU (that of `like`), of that type and shape"""
    if not t.is_cuda:
        _refuse("SQLLM_ERR_DEVICE", f"{what} is not on a GPU")
    if like is not None and t.get_device() != like.get_device():
        _refuse("SQLLM_ERR_DEVICE", f"{what} is on {t.device}, not on {like.device}")
    if dtype is not None and t.dtype is not dtype:
        _refuse("SQLLM_ERR_TYPE", f"{what} is {t.dtype}, not {dtype}")
    if shape is not None and t.shape != shape:
        _refuse("SQLLM_ERR_SHAPE", f"{what} is {tuple(t.shape)}, not {shape}")


def _rows(t, what):
    """a matrix the library can walk by rows, and its row stride: t itself or a contiguous copy"""
    if t.dim() != 2:
        _refuse("SQLLM_ERR_SHAPE", f"{what} has {t.dim()} dimensions, not 2")
    if t.is_contiguous():
        return t, t.shape[1]
    if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        t = t.contiguous()
    return t, (t.stride(0) if t.shape[0] > 1 else t.shape[1])


class MxMatrix:
    """An M x N matrix of 4-bit codes (uint8 [M, P / 2], P = N rounded up to a multiple of 128) with one scale byte per 32 columns (uint8 [M, P / 32])."""

    __slots__ = ("M", "N", "codes", "scales")

    def __init__(self, M: int, N: int, codes: torch.Tensor, scales: torch.Tensor):
        _need_size(M, N)
        padded = -(-N // ROW) * ROW
        for t, what, width in ((codes, "codes", padded // 2), (scales, "scales", padded // 32)):
            _need(t, what, codes, torch.uint8, (M, width))
            if not t.is_contiguous():
                _refuse("SQLLM_ERR_SHAPE", f"{what} are not contiguous")
        self.M, self.N, self.codes, self.scales = M, N, codes, scales

    @staticmethod
    def empty(M, N, device):
        _need_size(M, N)
        return MxMatrix._empty(M, N, device)

    @staticmethod
    def _empty(M, N, device):
        padded = -(-N // ROW) * ROW
        m = object.__new__(MxMatrix)
        m.M, m.N = M, N
        m.codes = _empty(M, padded // 2, torch.uint8, device)
        m.scales = _empty(M, padded // 32, torch.uint8, device)
        return m

    @property
    def device(self):
        return self.codes.device

    def dequantize(self, dtype=torch.float16) -> torch.Tensor:
        """the numbers it holds, [M, N]"""
        ty = _type_of(dtype)
        codes = self.codes
        out = _empty(self.M, self.N, dtype, codes.device)
        if self.N == 0:
            return out
        _call(codes.get_device(), DEQUANTIZE, self.M, self.N, ty, codes, self.scales, out, self.N)
        return out


def mx_quantize(w: torch.Tensor, direction: str = "rows"):
    """w [M, N] packed with its blocks along the rows ("rows"), its transpose, an N x M matrix with blocks along the columns of w ("columns"), or
    the pair of both from one pass over w ("both").  A matrix without rows or columns is packed as one: the sums over nothing that its products are are zeros."""
    if direction not in ("rows", "columns", "both"):
        raise ValueError(f"direction = {direction!r} is none of 'rows', 'columns' and 'both'")
    _need(w, "w")
    ty = _type_of(w.dtype)
    w, ld = _rows(w, "w")
    M, N = w.shape
    device = w.device
    rows = columns = None
    if direction != "columns":
        _need_size(M, N or 1)
        rows = MxMatrix._empty(M, N, device)
    if direction != "rows":
        _need_size(N, M or 1)
        columns = MxMatrix._empty(N, M, device)
    if M and N:
        _call(w.get_device(), QUANTIZE, M, N, ty, w, ld, rows and rows.codes, rows and rows.scales, columns and columns.codes, columns and columns.scales)
    return (rows, columns) if direction == "both" else rows or columns


def mx_gemv(w: MxMatrix, x: torch.Tensor, y: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """W x for fp16 x [N, B], B = 1..16, as fp16 [M, B]; with accumulate, y + W x in y.  N is a multiple of 128, at most 28672, and x starts at a multiple of 16 bytes
    (mx_linear takes any N and any x); no gradient is recorded"""
    codes, B = w.codes, x.shape[1] if x.dim() == 2 else 0
    _need(x, "x", codes, torch.float16, (w.N, B))
    if y is None:
        if accumulate:
            _refuse("SQLLM_ERR_NULL", "accumulate needs y")
        y = _empty(w.M, B, torch.float16, codes.device)
    else:
        _need(y, "y", codes, torch.float16, (w.M, B))
        if not y.is_contiguous():
            _refuse("SQLLM_ERR_SHAPE", "y is not contiguous")
    _call(codes.get_device(), GEMV, w.M, w.N, B, codes, w.scales, x.contiguous(), y, 1 if accumulate else 0)
    return y


def mx_gemm(x: MxMatrix, w: MxMatrix, dtype=torch.float16, y: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """x w^T of two packed matrices with the same number of columns, [x.M, w.M]; y: where to (its type then counts), with accumulate added to what it holds"""
    if x.N != w.N:
        _refuse("SQLLM_ERR_SHAPE", f"x has {x.N} columns, w has {w.N}")
    codes = w.codes
    if x.codes.get_device() != codes.get_device():
        _refuse("SQLLM_ERR_DEVICE", f"x is on {x.device}, w on {w.device}")
    if y is None:
        if accumulate:
            _refuse("SQLLM_ERR_NULL", "accumulate needs y")
        ty = _type_of(dtype)
        y = _empty(x.M, w.M, dtype, codes.device)
        ld = w.M
    else:
        _need(y, "y", codes, None, (x.M, w.M))
        ty = _type_of(y.dtype)
        ld = y.stride(0) if x.M > 1 else w.M
        if w.M > 1 and y.stride(1) != 1 or ld < w.M:
            _refuse("SQLLM_ERR_SHAPE", f"y has strides {y.stride()}: its rows must be contiguous and must not overlap")
    if w.N == 0:                                                     # sums over nothing
        if not accumulate:
            y.detach().zero_()
        return y
    _call(codes.get_device(), GEMM, x.M, w.M, w.N, ty, x.codes, x.scales, codes, w.scales, y, ld, 1 if accumulate else 0)
    return y


def mx_linear(x: torch.Tensor, w: MxMatrix, dtype=None) -> torch.Tensor:
    """y = Q(x) W^T for tokens x [T, N] and a packed layer W [M, N], [T, M] in dtype (that of x if None); no gradient is recorded (mx_linear_backward)"""
    return mx_gemm(mx_quantize(x), w, x.dtype if dtype is None else dtype)


def mx_linear_backward(dy: torch.Tensor, x_t: MxMatrix, w_t: MxMatrix, dtype=None, dw: torch.Tensor | None = None):
    """Gradients of y = Q(x) Q(w)^T (rounding passes gradients through) for dy [T, M]: dx = Q(dy) Q(w) in dtype (that of dy if None), and dw = Q(dy)^T Q(x)
    in fp32, added to `dw` (fp32 too: sums of gradients are not rounded to fewer bits between steps) where that is given.  x_t and w_t are the packed
    transposes of x [T, N] and w [M, N]: mx_quantize(..., "both")[1].
    The blocks of dy lie along the rows for dx and along the columns for dw, as the sums run."""
    _need(dy, "dy", w_t.codes, None, (x_t.N, w_t.N))
    if x_t.M != w_t.M:
        _refuse("SQLLM_ERR_SHAPE", f"x has {x_t.M} columns, w has {w_t.M}")
    if dw is not None:
        _need(dw, "dw", w_t.codes, torch.float32, (w_t.N, x_t.M))
    rows, columns = mx_quantize(dy, "both")
    dx = mx_gemm(rows, w_t, dy.dtype if dtype is None else dtype)
    if dw is None:
        return dx, mx_gemm(columns, x_t, torch.float32)
    return dx, mx_gemm(columns, x_t, y=dw, accumulate=True)
