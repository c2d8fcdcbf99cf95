"""Operators on 8-bit rows, on torch tensors: thin calls of the spark_scaled_* entry points of include/spark.h.

    x = scaled_norm(h, gain, eps, y=y)          # h += y, RMSNorm, 8-bit rows
    qkv = scaled_matmul(x, ScaledWeights(wqkv)) # fp32 or bf16
    a = scaled_gated(x, ScaledWeights(wg, wu))  # silu(x Wg^T) * (x Wu^T), 8-bit rows
    o = scaled_matmul(scaled_rows(attn), ScaledWeights(wo))

Every call runs on the current stream of its tensors' device, allocates its results unless they are given
(`out`), and raises SparkError with nothing launched where a tensor does not fit.  There is no fallback: the
work is done by libspark.so's kernels.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import SparkError, load_library

BLOCK = 128
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}


def _refuse(why: str):
    raise SparkError(-1, why)


def _padded(k: int) -> tuple[int, int]:
    """codes and powers of a row of k values"""
    blocks = -(-k // BLOCK)
    return blocks * BLOCK, -(-blocks // 4) * 4


def _matrix(t, what: str, shape=None, dtypes=_DTYPE):
    """a 2-d device tensor of a type the kernels read, rows contiguous"""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dim() != 2 or t.dtype not in dtypes:
        _refuse(f"{what}: a 2-d fp32 or bf16 tensor on the GPU is wanted")
    if shape is not None and tuple(t.shape) != shape:
        _refuse(f"{what} is {tuple(t.shape)}, {shape} is wanted")
    if t.shape[1] < 1 or (t.stride(1) != 1 and t.shape[1] > 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        _refuse(f"{what}: the elements of a row must lie next to each other, and rows apart")
    return t


def _stride(t) -> int:
    return max(t.stride(0), t.shape[1])   # (of a single row torch may say anything)


class _on:
    """the device of a call's tensors, current while the call is made; its current stream"""
    __slots__ = ("device", "guard")

    def __init__(self, first, *others):
        self.device = first.get_device()
        for t in others:
            if t is not None and t.get_device() != self.device:
                _refuse("the tensors are on different devices")
        self.guard = torch.cuda.device(self.device) if self.device != torch.cuda.current_device() else None

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.device)   # (torch.cuda.current_stream() takes 3 us)

    def __exit__(self, *a):
        if self.guard is not None:
            self.guard.__exit__(*a)


def _check(rc: int, what: str):
    if rc:
        raise SparkError(rc, what + " was refused or failed")


class ScaledRows:
    """m rows of k values in 8 bits: `codes` float8_e4m3fn [m][k rounded up to 128s], `scales` float8_e8m0fnu, one
    for every 128 codes, padded to a multiple of four."""
    __slots__ = ("codes", "scales", "m", "k")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, k: int):
        if codes.dim() != 2 or scales.dim() != 2 or k < 1 or codes.shape[0] != scales.shape[0] or \
                (codes.shape[1], scales.shape[1]) != _padded(k) or codes.dtype != torch.float8_e4m3fn or \
                scales.dtype != torch.float8_e8m0fnu or not codes.is_contiguous() or not scales.is_contiguous():
            _refuse("codes and scales do not make 8-bit rows")
        if codes.device.type != "cuda" or codes.device != scales.device:
            _refuse("8-bit rows: both tensors on one GPU are wanted")
        self.codes, self.scales, self.m, self.k = codes, scales, codes.shape[0], k

    @classmethod
    def empty(cls, m: int, k: int, device="cuda") -> "ScaledRows":
        if m < 0 or k < 1:
            _refuse(f"8-bit rows of {m} x {k}")
        kp, pitch = _padded(k)
        return cls(torch.empty(m, kp, dtype=torch.float8_e4m3fn, device=device),
                   torch.empty(m, pitch, dtype=torch.float8_e8m0fnu, device=device), k)

    def values(self) -> torch.Tensor:
        """the numbers they stand for, fp32 [m][k]"""
        blocks = self.codes.shape[1] // BLOCK
        v = self.codes.float().view(self.m, blocks, BLOCK) * self.scales[:, :blocks].float().unsqueeze(-1)
        return v.view(self.m, blocks * BLOCK)[:, :self.k]


def _rows_out(out, m: int, k: int, device) -> ScaledRows:
    if out is None:
        return ScaledRows.empty(m, k, device)
    if out.m != m or out.k != k:
        _refuse(f"out holds {out.m} x {out.k} values, {m} x {k} are written")
    return out


class ScaledWeights:
    """A projection matrix [n][k] (fp32 or bf16), or with `up` the pair of gate and up, laid out once in 8 bits in the
    order the matrix instructions take them."""

    def __init__(self, w: torch.Tensor, up: torch.Tensor | None = None):
        _matrix(w, "w")
        if up is not None and (_matrix(up, "up", tuple(w.shape)).dtype != w.dtype or _stride(up) != _stride(w)):
            _refuse("up must have w's type and stride")
        self.n, self.k = w.shape
        self.pair = up is not None
        lib, size = load_library(), C.c_size_t()
        _check(lib.spark_scaled_weight_bytes(self.n, self.k, int(self.pair), C.byref(size)), "weights")
        with _on(w, up) as stream:
            self.packed = torch.empty(size.value, dtype=torch.uint8, device=w.device)
            _check(lib.spark_scaled_pack(w.data_ptr(), up.data_ptr() if self.pair else None, _DTYPE[w.dtype], _stride(w), self.n, self.k,
                                         self.packed.data_ptr(), size.value, stream), "packing the weights")
        self._workspace = {}   # rows -> bytes

    def workspace_bytes(self, m: int) -> int:
        """of a product with m rows"""
        need = self._workspace.get(m)
        if need is None:
            size = C.c_size_t()
            with _on(self.packed):
                _check(load_library().spark_scaled_workspace_bytes(m, self.n, self.k, int(self.pair), C.byref(size)), "workspace")
            need = self._workspace[m] = size.value
        return need


def scaled_rows(x: torch.Tensor, out: ScaledRows | None = None) -> ScaledRows:
    """x [m][k], fp32 or bf16, as 8-bit rows"""
    _matrix(x, "x")
    m, k = x.shape
    out = _rows_out(out, m, k, x.device)
    if m == 0:
        return out
    with _on(x, out.codes) as stream:
        _check(load_library().spark_scaled_rows(x.data_ptr(), _DTYPE[x.dtype], _stride(x), m, k, out.codes.data_ptr(),
                                                out.scales.data_ptr(), stream), "scaled_rows")
    return out


def scaled_norm(h: torch.Tensor, gain: torch.Tensor, eps: float, y: torch.Tensor | None = None,
                h_out: torch.Tensor | None = None, out: ScaledRows | None = None) -> ScaledRows:
    """h' = h + y (in h's type, written to h_out, or to h where none is given), then the 8-bit rows of
    h' / sqrt(mean h'^2 + eps) * gain.  h, y, h_out [m][k] fp32 or bf16, gain fp32 [k]."""
    _matrix(h, "h")
    m, k = h.shape
    if y is not None:
        _matrix(y, "y", (m, k))
    h_out = h if h_out is None else _matrix(h_out, "h_out", (m, k), (h.dtype,))
    if gain.dtype != torch.float32 or tuple(gain.shape) != (k,) or not gain.is_contiguous():
        _refuse(f"gain: fp32 [{k}] is wanted")
    if not eps >= 0.0:
        _refuse("eps must not be negative")
    out = _rows_out(out, m, k, h.device)
    if m == 0:
        return out
    with _on(h, y, h_out, gain, out.codes) as stream:
        _check(load_library().spark_scaled_norm(
            h.data_ptr(), _DTYPE[h.dtype], _stride(h), None if y is None else y.data_ptr(), 0 if y is None else _DTYPE[y.dtype],
            0 if y is None else _stride(y), h_out.data_ptr(), _stride(h_out), gain.data_ptr(), eps, m, k, out.codes.data_ptr(),
            out.scales.data_ptr(), stream), "scaled_norm")
    return out


def _workspace(x: ScaledRows, w: ScaledWeights):
    need = w.workspace_bytes(x.m)
    return (torch.empty(need, dtype=torch.uint8, device=x.codes.device), need) if need else (None, 0)


def scaled_matmul(x: ScaledRows, w: ScaledWeights, out: torch.Tensor | None = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """x W^T, [m][n] of `dtype` (fp32 or bf16; out's, where it is given)"""
    if w.pair or x.k != w.k:
        _refuse(f"rows of {x.k} and {'a pair of matrices' if w.pair else 'weights'} of {w.k}")
    if out is None:
        if dtype not in _DTYPE:
            _refuse("dtype: fp32 or bf16 is wanted")
        out = torch.empty(x.m, w.n, dtype=dtype, device=x.codes.device)
    else:
        _matrix(out, "out", (x.m, w.n))
    if x.m == 0:
        return out
    with _on(x.codes, w.packed, out) as stream:
        ws, need = _workspace(x, w)
        _check(load_library().spark_scaled_matmul(x.codes.data_ptr(), x.scales.data_ptr(), x.m, w.packed.data_ptr(), w.n, w.k, out.data_ptr(),
                                                  _DTYPE[out.dtype], _stride(out), ws.data_ptr() if need else None, need, stream),
               "scaled_matmul")
    return out


def scaled_gated(x: ScaledRows, w: ScaledWeights, out: ScaledRows | None = None) -> ScaledRows:
    """silu(x Wg^T) * (x Wu^T) as 8-bit rows [m][n]; w: a pair"""
    if not w.pair or x.k != w.k:
        _refuse(f"rows of {x.k} and {'a pair' if w.pair else 'one matrix'} of {w.k}: a pair of gate and up is wanted")
    out = _rows_out(out, x.m, w.n, x.codes.device)
    if x.m == 0:
        return out
    with _on(x.codes, w.packed, out.codes) as stream:
        ws, need = _workspace(x, w)
        _check(load_library().spark_scaled_gated(x.codes.data_ptr(), x.scales.data_ptr(), x.m, w.packed.data_ptr(), w.n, w.k,
                                                 out.codes.data_ptr(), out.scales.data_ptr(), ws.data_ptr() if need else None, need, stream),
               "scaled_gated")
    return out
