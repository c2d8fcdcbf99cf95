"""Operators on 8-bit rows, on torch tensors: thin calls of the spark_scaled_* entry points of include/spark.h.

    x = scaled_norm(h, gain, eps, y=y)          # h += y, RMSNorm, 8-bit rows
    qkv = scaled_matmul(x, ScaledWeights(wqkv)) # fp32 or bf16
    a = scaled_gated(x, ScaledWeights(wg, wu))  # silu(x Wg^T) * (x Wu^T), 8-bit rows
    o = scaled_matmul(scaled_rows(attn), ScaledWeights(wo))

Every call runs on the current stream of its tensors' device, allocates its results unless they are given
(`out`), and raises SparkError with nothing launched where a tensor does not fit.  There is no fallback: the
work is done by libspark.so's kernels.  The operators have no derivatives: a tensor that a gradient or tangent is wanted
of is refused (detach it, or call them under torch.no_grad()), and a tensor that they write counts as changed in place.
"""
from __future__ import annotations

import ctypes as C

import torch
from torch.autograd import forward_ad

from .binding import SparkError, load_library

BLOCK = 128
LONGEST, MOST_ROWS = 1 << 22, (1 << 31) - 1   # of a row; of the calls, whose sizes are 32-bit numbers (ctypes would cut larger ones)
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}
# The current device, its current stream's raw handle, and the versions of tensors that were written: torch.cuda.current_stream() and
# torch.autograd.graph.increment_version() take 3 and 0.4 us, the smallest launches here 2.
_device, _stream, _changed = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch._C._increment_version


def _refuse(why: str):
    raise SparkError(-1, why)


def _padded(k: int) -> tuple[int, int]:
    """codes and powers of a row of k values"""
    blocks = -(-k // BLOCK)
    return blocks * BLOCK, -(-blocks // 4) * 4


def _size(what: str, m: int, k: int):
    if not (0 <= m <= MOST_ROWS and 1 <= k <= LONGEST):
        _refuse(f"{what}: {m} x {k}, and up to {MOST_ROWS} rows of 1 to {LONGEST} values are taken")


def _matrix(t, what: str, shape=None):
    """(address, type, stride, rows, row's length) of a 2-d device tensor of a type the kernels read, rows contiguous"""
    try:
        code = _DTYPE[t.dtype]
        m, k = t.shape
        stride, step = t.stride()
        on_gpu = t.is_cuda
    except (AttributeError, KeyError, TypeError, ValueError):
        on_gpu = False
    if not on_gpu:
        _refuse(f"{what}: a 2-d fp32 or bf16 tensor on the GPU is wanted")
    if shape is not None and (m, k) != shape:
        _refuse(f"{what} is {m} x {k}, {shape[0]} x {shape[1]} is wanted")
    if m > MOST_ROWS or not 1 <= k <= LONGEST:
        _size(what, m, k)
    if m <= 1 and stride < k:
        stride = k              # (of a single row torch may say anything)
    if (step != 1 and k > 1) or stride < k:
        _refuse(f"{what}: the elements of a row must lie next to each other, and rows apart")
    return t.data_ptr(), code, stride, m, k


def _no_gradient(*tensors, what: str = "an operator on 8-bit rows"):
    """nothing may pass whose gradient or tangent would be lost without a word"""
    dual = forward_ad._current_level >= 0   # (outside a level of forward mode there are no tangents)
    for t in tensors:
        if t is not None and ((t.requires_grad and torch.is_grad_enabled()) or (dual and forward_ad.unpack_dual(t).tangent is not None)):
            _refuse(f"{what} has no derivatives, and a gradient or tangent of a tensor is wanted")


def _launch(what: str, tensors, written, call, *args):
    """call(*args, stream) with the tensors' (the first is one, others may be None) device current and on its current stream;
    `written`: those given tensors that it changes"""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None:
            if t.get_device() != dev:
                _refuse("the tensors are on different devices")
            if t.requires_grad:
                _no_gradient(t, what=what)
    if forward_ad._current_level >= 0:
        _no_gradient(*tensors, what=what)
    if dev == _device():
        rc = call(*args, _stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = call(*args, _stream(dev))
    if rc:
        raise SparkError(rc, what + " was refused or failed")
    if written:
        _changed(written)


class ScaledRows:
    """m rows of k values in 8 bits: `codes` float8_e4m3fn [m][k rounded up to 128s], `scales` float8_e8m0fnu, one
    for every 128 codes, padded to a multiple of four."""
    __slots__ = ("codes", "scales", "m", "k")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, k: int):
        _size("8-bit rows", codes.shape[0] if codes.dim() else 0, k)
        if codes.dim() != 2 or scales.dim() != 2 or codes.shape[0] != scales.shape[0] or \
                (codes.shape[1], scales.shape[1]) != _padded(k) or codes.dtype != torch.float8_e4m3fn or \
                scales.dtype != torch.float8_e8m0fnu or not codes.is_contiguous() or not scales.is_contiguous():
            _refuse("codes and scales do not make 8-bit rows")
        if codes.device.type != "cuda" or codes.device != scales.device:
            _refuse("8-bit rows: both tensors on one GPU are wanted")
        _no_gradient(codes, scales)
        self.codes, self.scales, self.m, self.k = codes, scales, codes.shape[0], k

    @classmethod
    def empty(cls, m: int, k: int, device="cuda") -> "ScaledRows":
        _size("8-bit rows", m, k)
        kp, pitch = _padded(k)
        return cls(torch.empty(m, kp, dtype=torch.float8_e4m3fn, device=device),
                   torch.empty(m, pitch, dtype=torch.float8_e8m0fnu, device=device), k)

    def values(self) -> torch.Tensor:
        """the numbers they stand for, fp32 [m][k]"""
        blocks = self.codes.shape[1] // BLOCK
        v = self.codes.float().view(self.m, blocks, BLOCK) * self.scales[:, :blocks].float().unsqueeze(-1)
        return v.view(self.m, blocks * BLOCK)[:, :self.k]


def _rows_out(out, m: int, k: int, like):
    """(the rows to write, beside `like`; those of its tensors that were given)"""
    if out is None:
        return ScaledRows.empty(m, k, like.device), ()
    if out.m != m or out.k != k:
        _refuse(f"out holds {out.m} x {out.k} values, {m} x {k} are written")
    return out, (out.codes, out.scales)


class ScaledWeights:
    """A projection matrix [n][k] (fp32 or bf16), or with `up` the pair of gate and up, laid out once in 8 bits in the
    order the matrix instructions take them."""

    def __init__(self, w: torch.Tensor, up: torch.Tensor | None = None):
        at, code, stride, self.n, self.k = _matrix(w, "w")
        self.pair = up is not None
        up_at = None
        if self.pair:
            up_at, up_code, up_stride, _, _ = _matrix(up, "up", (self.n, self.k))
            if (up_code, up_stride) != (code, stride):
                _refuse("up must have w's type and stride")
        lib, size = load_library(), C.c_size_t()
        if lib.spark_scaled_weight_bytes(self.n, self.k, int(self.pair), C.byref(size)):
            _refuse(f"weights of {self.n} x {self.k}")
        self.packed = torch.empty(size.value, dtype=torch.uint8, device=w.device)
        _launch("packing the weights", (w, up), None, lib.spark_scaled_pack, at, up_at, code, stride, self.n, self.k,
                self.packed.data_ptr(), size.value)
        self._workspace = {}   # rows -> bytes

    def workspace_bytes(self, m: int) -> int:
        """of a product with m rows"""
        need = self._workspace.get(m)
        if need is None:
            _size("a product's rows", m, self.k)
            size = C.c_size_t()
            with torch.cuda.device(self.packed.device):
                if load_library().spark_scaled_workspace_bytes(m, self.n, self.k, int(self.pair), C.byref(size)):
                    _refuse(f"a product of {m} rows")
            need = self._workspace[m] = size.value
        return need

    def workspace(self, m: int):
        """(tensor or None, its address, its bytes) for one call; torch's allocator hands it on in stream order"""
        need = self._workspace.get(m)
        if need is None:
            need = self.workspace_bytes(m)
        if not need:
            return None, None, 0
        t = torch.empty(need, dtype=torch.uint8, device=self.packed.device)
        return t, t.data_ptr(), need


def scaled_rows(x: torch.Tensor, out: ScaledRows | None = None) -> ScaledRows:
    """x [m][k], fp32 or bf16, as 8-bit rows"""
    at, code, stride, m, k = _matrix(x, "x")
    out, given = _rows_out(out, m, k, x)
    if m:
        _launch("scaled_rows", (x, out.codes), given, load_library().spark_scaled_rows, at, code, stride, m, k, out.codes.data_ptr(),
                out.scales.data_ptr())
    return out


def scaled_norm(h: torch.Tensor, gain: torch.Tensor, eps: float, y: torch.Tensor | None = None,
                h_out: torch.Tensor | None = None, out: ScaledRows | None = None) -> ScaledRows:
    """h' = h + y (in h's type, written to h_out, or to h where none is given), then the 8-bit rows of
    h' / sqrt(mean h'^2 + eps) * gain.  h, y, h_out [m][k] fp32 or bf16, gain fp32 [k]."""
    at, code, stride, m, k = _matrix(h, "h")
    y_at, y_code, y_stride, _, _ = (None, 0, 0, m, k) if y is None else _matrix(y, "y", (m, k))
    out_at, out_code, out_stride, _, _ = (at, code, stride, m, k) if h_out is None else _matrix(h_out, "h_out", (m, k))
    if out_code != code:
        _refuse("h_out must have h's type")
    if gain.dtype is not torch.float32 or gain.dim() != 1 or gain.numel() != k or not gain.is_contiguous():
        _refuse(f"gain: fp32 [{k}] is wanted")
    if not eps >= 0.0:
        _refuse("eps must not be negative")
    out, given = _rows_out(out, m, k, h)
    if m:
        if y is not None or out_at != at:   # (otherwise h' is h, where it lies)
            given = (h if h_out is None else h_out, *given)
        _launch("scaled_norm", (h, y, h_out, gain, out.codes), given, load_library().spark_scaled_norm, at, code, stride,
                y_at, y_code, y_stride, out_at, out_stride, gain.data_ptr(), eps, m, k, out.codes.data_ptr(), out.scales.data_ptr())
    return out


def scaled_matmul(x: ScaledRows, w: ScaledWeights, out: torch.Tensor | None = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """x W^T, [m][n] of `dtype` (fp32 or bf16; out's, where it is given)"""
    if w.pair or x.k != w.k:
        _refuse(f"rows of {x.k} and {'a pair of matrices' if w.pair else 'weights'} of {w.k}")
    given = None if out is None else (out,)
    if out is None:
        if dtype not in _DTYPE:
            _refuse("dtype: fp32 or bf16 is wanted")
        out = torch.empty(x.m, w.n, dtype=dtype, device=x.codes.device)
    at, code, stride, _, _ = _matrix(out, "out", (x.m, w.n))
    if x.m:
        keep, ws, need = w.workspace(x.m)
        _launch("scaled_matmul", (x.codes, w.packed, out), given, load_library().spark_scaled_matmul, x.codes.data_ptr(), x.scales.data_ptr(), x.m,
                w.packed.data_ptr(), w.n, w.k, at, code, stride, ws, need)
    return out


def scaled_gated(x: ScaledRows, w: ScaledWeights, out: ScaledRows | None = None) -> ScaledRows:
    """silu(x Wg^T) * (x Wu^T) as 8-bit rows [m][n]; w: a pair"""
    if not w.pair or x.k != w.k:
        _refuse(f"rows of {x.k} and {'a pair' if w.pair else 'one matrix'} of {w.k}: a pair of gate and up is wanted")
    out, given = _rows_out(out, x.m, w.n, x.codes)
    if x.m:
        if out.codes.data_ptr() == x.codes.data_ptr():
            _refuse("out must not be x")
        keep, ws, need = w.workspace(x.m)
        _launch("scaled_gated", (x.codes, w.packed, out.codes), given, load_library().spark_scaled_gated, x.codes.data_ptr(), x.scales.data_ptr(), x.m,
                w.packed.data_ptr(), w.n, w.k, out.codes.data_ptr(), out.scales.data_ptr(), ws, need)
    return out
