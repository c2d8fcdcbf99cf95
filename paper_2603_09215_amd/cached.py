"""Operators on a paged cache, on torch tensors: thin calls of the spark_cache_* entry points of include/spark.h.

    cache = PagedCache.empty(pages, kv_heads, head_dim)            # or PagedCache(pool): [page][layer][k|v][kv_head][token][head_dim]
    batch = CachedRows(starts, lengths, table)                     # which rows are whose, slots in use, pages
    turn = Rotation(rotary)                                        # angles per position
    q = cached_append(q, k, v, cache, batch, rotation=turn)        # norms, rotation, keys and values to their slots
    o = cached_attend(q, cache, batch, lse=lse)                    # attention over the slots
    w = cached_weigh(q, lse, cache, batch, before=w, out=w)        # the weight that every slot got
    kept, lengths = cached_evict(cache, batch, w, keep)            # the heaviest slots, next to each other

Every call runs on the current stream of its tensors' device, allocates its results unless they are given, and raises
SparkError with nothing launched where a tensor does not fit.  There is no fallback: the work is done by
libspark.so's kernels.  The operators have no derivatives: a tensor that a gradient or tangent is wanted of is refused,
and a tensor that they write counts as changed in place.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import SparkCache, SparkCacheBatch, SparkRotation, load_library
from .scaled import _DTYPE, _launch, _refuse


def _table(t, what: str, dims: int):
    """an int32 tensor on the GPU, without gaps"""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.dim() != dims or not t.is_cuda or not t.is_contiguous():
        _refuse(f"{what}: a contiguous {dims}-d int32 tensor on the GPU is wanted")
    return t


def _heads(t, what: str, head_dim: int, dtypes, shape=None):
    """(address, stride from row to row) of [rows][heads][head_dim], heads next to each other in a row"""
    try:
        m, heads, hd = t.shape
        stride, of_head, step = t.stride()
        on_gpu = t.is_cuda and t.dtype in dtypes
    except (AttributeError, TypeError, ValueError):
        on_gpu = False
    if not on_gpu:
        _refuse(f"{what}: a tensor [rows][heads][{head_dim}] on the GPU, of {' or '.join(str(d) for d in dtypes)}, is wanted")
    if hd != head_dim or (shape is not None and (m, heads) != shape):
        _refuse(f"{what} is {m} x {heads} x {hd}, {' x '.join(map(str, (*(shape or ('rows', 'heads')), head_dim)))} is wanted")
    if step != 1 or (of_head != hd and heads > 1) or (m > 1 and stride < heads * hd):
        _refuse(f"{what}: a row's heads must lie next to each other, and rows apart")
    return t.data_ptr(), stride if m > 1 else heads * hd   # (of a single row torch may say anything)


def _call(what: str, cache, batch, tensors, written, call, *args):
    """call(cache, batch, *args, stream) if all are on the cache's device; `written`: those given tensors that it changes"""
    if batch.device != cache.device:
        _refuse("the tensors are on different devices")
    _launch(what, (cache.pool, *tensors), written, call, *args)


_CACHE_BYTES, _BATCH_BYTES, _ROTATION_BYTES = C.sizeof(SparkCache), C.sizeof(SparkCacheBatch), C.sizeof(SparkRotation)


class PagedCache:
    """Keys and values in pages: `pool` [page][layer][k|v][kv_head][token in its page][head_dim], fp32 or bf16, head_dim 64 or 128,
    pages of a multiple of 16 tokens."""
    __slots__ = ("pool", "pages", "layers", "kv_heads", "page_tokens", "head_dim", "device", "_types", "_workspace")

    def __init__(self, pool: torch.Tensor):
        if not isinstance(pool, torch.Tensor) or pool.dim() != 6 or pool.shape[2] != 2 or not pool.is_cuda or not pool.is_contiguous() or pool.dtype not in _DTYPE:
            _refuse("pool: a contiguous fp32 or bf16 tensor [pages][layers][2][kv_heads][page_tokens][head_dim] on the GPU is wanted")
        self.pages, self.layers, _, self.kv_heads, self.page_tokens, self.head_dim = pool.shape
        if not (1 <= self.pages <= 1 << 24 and 1 <= self.layers <= 1 << 16 and 1 <= self.kv_heads <= 1 << 12 and 16 <= self.page_tokens <= 1 << 16 and
                self.page_tokens % 16 == 0 and self.head_dim in (64, 128)):
            _refuse(f"pool: {tuple(pool.shape)}; pages of 16 to 65536 tokens, a multiple of 16, and heads of 64 or 128 are taken")
        self.pool, self.device, self._types = pool, pool.device, (pool.dtype,)
        self._workspace = {}   # sizes -> bytes

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64, layers: int = 1, dtype=torch.bfloat16, device="cuda") -> "PagedCache":
        return cls(torch.empty(pages, layers, 2, kv_heads, page_tokens, head_dim, dtype=dtype, device=device))

    def _view(self, layer: int) -> SparkCache:
        if not 0 <= layer < self.layers:
            _refuse(f"layer {layer} of {self.layers}")
        return SparkCache(_CACHE_BYTES, _DTYPE[self.pool.dtype], self.pages, self.layers, self.kv_heads, self.page_tokens, self.head_dim, layer, self.pool.data_ptr())


class CachedRows:
    """A batch of n sequences: rows starts[s] .. starts[s + 1] - 1 are the new ones of sequence s, which are the last of its lengths[s]
    slots; table [n][pages a sequence has at most] holds its pages.  All int32 on the GPU; what they hold is read by each
    call (it may change between calls and between replays of a graph)."""
    __slots__ = ("starts", "lengths", "table", "n", "max_pages", "device")

    def __init__(self, starts: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor):
        self.starts, self.lengths, self.table = _table(starts, "starts", 1), _table(lengths, "lengths", 1), _table(table, "table", 2)
        self.n, self.max_pages = table.shape
        if starts.shape[0] != self.n + 1 or lengths.shape[0] != self.n:
            _refuse(f"starts has {starts.shape[0]} entries, lengths {lengths.shape[0]}: {self.n + 1} and {self.n} are wanted")
        if self.n > 1 << 16 or not 1 <= self.max_pages <= 1 << 24:
            _refuse(f"table: {self.n} sequences of {self.max_pages} pages; up to 65536 of 1 to 2^24 are taken")
        self.device = table.device
        if starts.device != self.device or lengths.device != self.device:
            _refuse("the tensors are on different devices")

    def _of(self, m: int, cache: PagedCache) -> SparkCacheBatch:
        """for calls on m rows"""
        if m > 1 << 22 or self.max_pages * cache.page_tokens > 1 << 23 or self.n * cache.kv_heads > 1 << 20:
            _refuse(f"{m} rows, {self.max_pages} pages of {cache.page_tokens}, {self.n} sequences with {cache.kv_heads} heads: up to 2^22 rows, 2^23 slots "
                    "a sequence and 2^20 heads of sequences are taken")
        return SparkCacheBatch(_BATCH_BYTES, m, self.n, self.max_pages, self.starts.data_ptr(), self.lengths.data_ptr(), self.table.data_ptr())


class Rotation:
    """The angles by which queries and keys are turned: the first `rotary` values of a head in pairs (j, j + rotary / 2), interleaved (2 j, 2 j + 1), by
    position * freqs[j], freqs[j] = base^(-2 j / rotary), and times `amplitude`.

    For contexts longer than the `original` one that a model was trained for: waves of fewer than `low` turns in it are drawn out by
    `factor`, those of more than `high` turns stay, and between them the share of each goes linearly with the turns (low == high: a
    step; both infinite: all waves are drawn out, which is positions divided by factor).  Or give `freqs` (rotary / 2 numbers)."""
    __slots__ = ("rotary", "interleaved", "amplitude", "freqs")

    def __init__(self, rotary: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                 original: int = 8192, amplitude: float = 1.0, freqs=None, device="cuda"):
        if rotary < 0 or rotary % 2 or rotary > 128:
            _refuse(f"rotary {rotary}: an even number up to the head's width is wanted")
        if not math.isfinite(amplitude):
            _refuse("amplitude must be finite")
        self.rotary, self.interleaved, self.amplitude = rotary, bool(interleaved), float(amplitude)
        if freqs is None:
            if not (base > 0 and factor > 0 and original > 0 and low <= high):
                _refuse("base, factor and original must be positive, low at most high")
            freqs = [self._drawn_out(base ** (-2 * j / rotary), factor, low, high, original) for j in range(rotary // 2)]
        freqs = torch.as_tensor(freqs, dtype=torch.float64)
        if freqs.shape != (rotary // 2,):
            _refuse(f"freqs: {rotary // 2} numbers are wanted")
        self.freqs = freqs.to(device).contiguous()

    @staticmethod
    def _drawn_out(f: float, factor: float, low: float, high: float, original: int) -> float:
        turns = original * f / (2 * math.pi)
        stay = (turns - low) / (high - low) if low < turns < high and high < math.inf else float(turns >= high)
        return f * (stay + (1 - stay) / factor)


def _gain(t, what: str, head_dim: int):
    return None if t is None else _plain(t, what, head_dim)


def _group(m: int, q_heads: int, cache: PagedCache):
    if not 1 <= q_heads <= 1 << 12 or q_heads % cache.kv_heads or m * q_heads > 1 << 26:
        _refuse(f"{m} rows of {q_heads} query heads and {cache.kv_heads} of keys: a multiple of these is wanted, up to 4096, and up to 2^26 with all rows'")


def cached_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cache: PagedCache, batch: CachedRows, layer: int = 0, rotation: Rotation | None = None,
                  q_gain: torch.Tensor | None = None, k_gain: torch.Tensor | None = None, eps: float = 1e-6, positions: torch.Tensor | None = None,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """q [m][q_heads][head_dim], k and v [m][kv_heads][head_dim] (fp32 or bf16, one type; views of one product's rows will do): heads of q and k
    normed where a gain (fp32 [head_dim]) is given, turned by position (positions int32 [m], or each row's slot), k and v written to their rows'
    slots of the cache; returns q in the cache's type (`out`; may be q itself), whose rows that are no sequence's are not written."""
    hd = cache.head_dim
    q_at, q_stride = _heads(q, "q", hd, _DTYPE)
    m, heads, _ = q.shape
    _group(m, heads, cache)
    types, of_kv = (q.dtype,), (m, cache.kv_heads)
    k_at, k_stride = _heads(k, "k", hd, types, of_kv)
    v_at, v_stride = _heads(v, "v", hd, types, of_kv)
    given = (cache.pool,) if out is None else (cache.pool, out)
    if out is None:
        out = torch.empty(m, heads, hd, dtype=cache.pool.dtype, device=q.device)
    out_at, out_stride = _heads(out, "out", hd, cache._types, (m, heads))
    if positions is not None and _table(positions, "positions", 1).shape[0] != m:
        _refuse(f"positions: {m} numbers are wanted")
    if not eps >= 0.0:
        _refuse("eps must not be negative")
    rotary = 0 if rotation is None else rotation.rotary
    if rotary > hd:
        _refuse(f"a rotation of {rotary} values and heads of {hd}")
    freqs = rotation.freqs if rotary else None
    turn = SparkRotation(_ROTATION_BYTES, rotary, rotary and rotation.interleaved, rotation.amplitude if rotary else 1.0, freqs.data_ptr() if rotary else None,
                         None if positions is None else positions.data_ptr(), _gain(q_gain, "q_gain", hd), _gain(k_gain, "k_gain", hd), eps)
    if m and batch.n:
        _call("cached_append", cache, batch, (q, k, v, out, freqs, positions, q_gain, k_gain), given, load_library().spark_cache_append, cache._view(layer),
              batch._of(m, cache), turn, heads, _DTYPE[q.dtype], q_at, q_stride, k_at, k_stride, v_at, v_stride, out_at, out_stride)
    return out


def _scale(scale, hd: int) -> float:
    if scale is None:
        return hd ** -0.5
    if not abs(scale) <= 2.0 ** 127 or C.c_float(scale).value == 0.0:
        _refuse("a scale up to 2^127, and not 0, is wanted")
    return scale


def _plain(t, what: str, *shape):
    """the address of a contiguous fp32 tensor of this shape"""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        _refuse(f"{what}: contiguous fp32 {shape} on the GPU is wanted")
    return t.data_ptr()


def _wide(what: str, at: int, stride: int):
    if at % 16 or stride % 8:
        _refuse(f"{what}: an address of 16 and a stride of 8 elements, or multiples, are wanted")


def attend_workspace_bytes(cache: PagedCache, batch: CachedRows, m: int, q_heads: int) -> int:
    """of cached_attend with m rows"""
    need = cache._workspace.get((m, q_heads, batch.n, batch.max_pages))
    if need is None:
        _group(m, q_heads, cache)
        size = C.c_size_t()
        with torch.cuda.device(cache.pool.device):
            if load_library().spark_cache_workspace_bytes(cache._view(0), batch._of(m, cache), q_heads, C.byref(size)):
                _refuse(f"attention of {m} rows of {q_heads} heads")
        if len(cache._workspace) >= 4096:   # (a program with ever new sizes)
            cache._workspace.clear()
        need = cache._workspace[m, q_heads, batch.n, batch.max_pages] = size.value
    return need


def cached_attend(q: torch.Tensor, cache: PagedCache, batch: CachedRows, layer: int = 0, scale: float | None = None, causal: bool = True,
                  out: torch.Tensor | None = None, lse: torch.Tensor | None = None) -> torch.Tensor:
    """softmax(scale q k^T) v over the slots that each row sees, [m][q_heads][head_dim] in the cache's type, q's too; scale: by default
    head_dim^-1/2; causal: a row sees the slots up to its own, else all of its sequence.  lse (fp32 [m][q_heads]) is given the
    logarithm of each row's sum.  A row that sees nothing: zeros, and minus infinity; rows that are no sequence's are not written."""
    hd = cache.head_dim
    at, stride = _heads(q, "q", hd, cache._types)
    m, heads, _ = q.shape
    _group(m, heads, cache)
    given = tuple(t for t in (out, lse) if t is not None)
    if out is None:
        out = torch.empty(m, heads, hd, dtype=q.dtype, device=q.device)
    out_at, out_stride = _heads(out, "out", hd, cache._types, (m, heads))
    _wide("q", at, stride)
    _wide("out", out_at, out_stride)
    lse_at = None if lse is None else _plain(lse, "lse", m, heads)
    scale = _scale(scale, hd)
    if m and batch.n:
        need = attend_workspace_bytes(cache, batch, m, heads)
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None   # (torch's allocator hands it on in stream order)
        _call("cached_attend", cache, batch, (q, out, lse), given, load_library().spark_cache_attend, cache._view(layer), batch._of(m, cache), heads, at, stride,
              scale, int(causal), out_at, out_stride, lse_at, None if ws is None else ws.data_ptr(), need)
    return out


def _weights(t, what: str, cache: PagedCache, batch: CachedRows):
    return _plain(t, what, batch.n, cache.kv_heads, batch.max_pages * cache.page_tokens)


def cached_weigh(q: torch.Tensor, lse: torch.Tensor, cache: PagedCache, batch: CachedRows, layer: int = 0, scale: float | None = None,
                 causal: bool = True, before: torch.Tensor | None = None, decay: float = 1.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """The attention weight of each slot, fp32 [n][kv_heads][slots a sequence has at most]: decay * before (zeros without) + the probabilities
    that the batch's rows gave it, summed over rows and the heads of its group; q, scale and causal as cached_attend had them, lse
    from it.  Slots behind a sequence's length are left alone (zeros in a new result).  out may be before.  (A batch of a long chunk and many single rows is
    faster in two calls.)"""
    hd = cache.head_dim
    at, stride = _heads(q, "q", hd, cache._types)
    m, heads, _ = q.shape
    _group(m, heads, cache)
    _wide("q", at, stride)
    lse_at = _plain(lse, "lse", m, heads)
    before_at = None if before is None else _weights(before, "before", cache, batch)
    if not math.isfinite(decay) or not math.isfinite(C.c_float(decay).value):
        _refuse("decay must be finite")
    given = None if out is None else (out,)
    if out is None:
        out = torch.zeros(batch.n, cache.kv_heads, batch.max_pages * cache.page_tokens, dtype=torch.float32, device=q.device)
    out_at = _weights(out, "out", cache, batch)
    scale = _scale(scale, hd)
    if batch.n:
        _call("cached_weigh", cache, batch, (q, lse, before, out), given, load_library().spark_cache_weigh, cache._view(layer), batch._of(m, cache), heads, at, stride,
              scale, int(causal), lse_at, before_at, decay, out_at)
    return out


def cached_evict(cache: PagedCache, batch: CachedRows, weights: torch.Tensor, keep: int, first: int = 0, recent: int = 0, layer: int = 0,
                 table_out: torch.Tensor | None = None, weights_out: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """Of sequences longer than `keep`, for each head of keys `keep` slots stay: the `first` first, the `recent` last, and of the others those of
    most weight (fp32 [n][kv_heads][slots]; equal ones: the lowest slot).  What stays moves to slots 0, 1, .. in its old order: keys and
    values in place, or to the pages of table_out (int32 [n][pages], none of them in batch.table); weights in place or to weights_out,
    with zeros from the new length to the old.  Returns (old slots int32 [n][kv_heads][keep], -1 behind the new length; new lengths int32 [n])."""
    at = _weights(weights, "weights", cache, batch)
    slots = batch.max_pages * cache.page_tokens
    if not (0 <= first and 0 <= recent and first + recent <= keep and 1 <= keep <= slots):
        _refuse(f"keep {keep}, first {first}, recent {recent}: first + recent <= keep, and keep of 1 to {slots} are wanted")
    out_pages = 0
    if table_out is not None:
        n, out_pages = _table(table_out, "table_out", 2).shape
        if n != batch.n or out_pages * cache.page_tokens < keep or out_pages > 1 << 24:
            _refuse(f"table_out is {n} x {out_pages}: pages for {keep} slots of {batch.n} sequences are wanted")
        if n and table_out.data_ptr() == batch.table.data_ptr():
            if n > 1 and out_pages != batch.max_pages:
                _refuse("table_out is a part of the batch's table")
            table_out = None
    out_at = at if weights_out is None else _weights(weights_out, "weights_out", cache, batch)
    kept = torch.empty(batch.n, cache.kv_heads, keep, dtype=torch.int32, device=weights.device)
    lengths = torch.empty(batch.n, dtype=torch.int32, device=weights.device)
    if batch.n:
        _call("cached_evict", cache, batch, (weights, weights_out, table_out), (cache.pool, weights if weights_out is None else weights_out),
              load_library().spark_cache_evict, cache._view(layer), batch._of(0, cache), at, keep, first, recent,
              None if table_out is None else table_out.data_ptr(), out_pages, out_at, kept.data_ptr(), lengths.data_ptr())
    return kept, lengths
