"""Operators on torch tensors: rotary positions, the 8-bit paged KV cache and causal
attention over it (the model-free calls of include/wici.h).

Argument marshalling only: every operator is a HIP kernel of libwici.so.  Tensors are on
one HIP GPU; a call enqueues on ``stream`` (default: the current stream of the tensors' GPU)
and returns without waiting.  On a stream other than the current one the caller orders the
inputs' producers before the call, as for any torch operation; results are allocated on
that stream.  Every call may be captured into a HIP graph.  The operators have no gradients: a
tensor that requires one is refused where gradients are recorded.

    table = ops.rope_table(n_pos, dim, base=500000.0, scaling="bands", factor=8, original=8192)
    cache = ops.KvCache.empty(n_pages, n_kv_heads, head_dim, page_table)
    q = cache.append(k, v, length, rope=table, q=q)      # one token of every sequence
    out = cache.attend(q, length)
"""

from __future__ import annotations

import contextlib
import ctypes

import torch

from . import binding
from .binding import WICI_BF16, WICI_F32, WICI_OK, WiciError

LAYOUTS = {"half": 0, "pairs": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}
_DTYPES = {torch.float32: WICI_F32, torch.bfloat16: WICI_BF16}

HeadRows = binding.WiciHeadRows
_NO_ROWS = HeadRows()


# The current stream of a GPU as the library takes it.  Of a small call's time on the host
# torch.cuda.current_stream is 2 us, its raw form 0.2.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


# Tells autograd that a call has written the caller's tensor, as operations in place do (0.3 us;
# tensors made in a call need none).
_written = torch.autograd.graph.increment_version


def _check(st: int, what: str) -> None:
    if st != WICI_OK:
        raise WiciError(st, what)


def _no_gradient(name: str) -> None:
    """For a tensor that requires a gradient."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{name}: requires a gradient, which these operators do not have (call "
                           "them under torch.no_grad(), or detach)")


def _rows(x: torch.Tensor, heads: int, head_dim: int, name: str, device) -> HeadRows:
    """x [rows, heads, head_dim] as the library takes it (strides of its own, dimensions
    side by side)."""
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise TypeError(f"{name}: dtype {x.dtype} (float32 or bfloat16)")
    if x.requires_grad:
        _no_gradient(name)
    shape = x.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != head_dim:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected [rows, {heads}, {head_dim}]")
    if x.device != device:
        raise ValueError(f"{name}: on {x.device}, expected {device}")
    r, h, d = x.stride()
    if d != 1:
        raise ValueError(f"{name}: the dimensions of a head must lie side by side")
    if heads == 1:
        h = head_dim
    if shape[0] <= 1:
        r = heads * max(h, head_dim)
    return HeadRows(x.data_ptr(), dtype, r, h)


def _ints(x: torch.Tensor, shape, name: str, device) -> int:
    if x.dtype != torch.int32 or tuple(x.shape) != shape or not x.is_contiguous():
        raise ValueError(f"{name}: {x.dtype} {tuple(x.shape)}, expected contiguous int32 {shape}")
    if x.device != device:
        raise ValueError(f"{name}: on {x.device}, expected {device}")
    return x.data_ptr()


def _like(x: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _new_rows(x: torch.Tensor) -> HeadRows:
    """A tensor made here (so contiguous, of a type and on a GPU already checked)."""
    _, h, d = x.shape
    return HeadRows(x.data_ptr(), _DTYPES[x.dtype], h * d, d)


def _on_gpu(x: torch.Tensor, name: str):
    if not x.is_cuda:
        raise ValueError(f"{name}: on {x.device}, expected a HIP GPU")
    return x.device


class _Here:
    """The raw current stream, where the tensors' GPU is current."""

    def __init__(self, raw):
        self.raw = raw

    def __enter__(self):
        return self.raw

    def __exit__(self, *exc):
        return False


@contextlib.contextmanager
def _elsewhere(stream, device, tensors):
    with torch.cuda.device(device):
        if stream is None:
            yield _raw_stream(device.index)
            return
        with torch.cuda.stream(stream):
            yield stream.cuda_stream
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)


def _launch_on(stream, device, *tensors):
    """Context giving the raw stream, with the tensors' GPU current and allocations made
    for that stream."""
    if stream is None and device.index == torch.cuda.current_device():
        return _Here(_raw_stream(device.index))
    if stream is not None and stream.device != device:
        raise ValueError(f"stream: on {stream.device}, expected {device}")
    return _elsewhere(stream, device, tensors)


class RopeTable:
    """Rotary tables: ``cos`` and ``sin`` [n_pos, dim / 2] (float32) and the pairs they turn:
    "half" (j, j + dim / 2) or "pairs" (2 j, 2 j + 1)."""

    def __init__(self, cos: torch.Tensor, sin: torch.Tensor, layout: str = "half"):
        device = _on_gpu(cos, "cos")
        for name, t in (("cos", cos), ("sin", sin)):
            if t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or \
                    t.shape != cos.shape or t.device != device:
                raise ValueError(f"{name}: contiguous float32 [n_pos, dim / 2] on one GPU expected")
        if layout not in LAYOUTS:
            raise ValueError(f"layout {layout!r} (one of {sorted(LAYOUTS)})")
        self.cos, self.sin, self.layout = cos, sin, layout
        self.dim = 2 * cos.shape[1]
        self.device = device
        self._c = binding.WiciRopeTab(cos.data_ptr(), sin.data_ptr(), cos.shape[0], self.dim,
                                      LAYOUTS[layout])


def rope_spec(dim: int, base: float = 10000.0, layout: str = "half", scaling: str = "plain",
              factor: float = 1.0, original: float = 0.0, low: float = 0.0,
              high: float = 0.0) -> "binding.WiciRope":
    """A rotary embedding (wici_rope): ``dim`` rotated dimensions, its base, and how its
    angle steps are scaled for contexts longer than the ``original`` positions:
    "plain", "linear", "base", "bands" or "ramp"."""
    if layout not in LAYOUTS:
        raise ValueError(f"layout {layout!r} (one of {sorted(LAYOUTS)})")
    if scaling not in SCALINGS:
        raise ValueError(f"scaling {scaling!r} (one of {sorted(SCALINGS)})")
    return binding.WiciRope(dim, LAYOUTS[layout], SCALINGS[scaling], base, factor, original, low,
                            high)


def rope_table(n_pos: int, dim: int, *, device=None, stream=None, layout: str = "half",
               **spec) -> RopeTable:
    """Tables of positions 0 .. n_pos - 1 (wici_rope_table); ``spec`` as for rope_spec."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else \
        torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"device {device}, expected a HIP GPU")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    c = rope_spec(dim, layout=layout, **spec)
    if n_pos < 1 or dim < 2:
        raise ValueError(f"n_pos {n_pos}, dim {dim}")
    lib = binding.load_library()
    with _launch_on(stream, device) as raw:
        cos = torch.empty(n_pos, dim // 2, dtype=torch.float32, device=device)
        sin = torch.empty_like(cos)
        _check(lib.wici_rope_table(ctypes.byref(c), n_pos, cos.data_ptr(), sin.data_ptr(), raw),
               f"rope_table: dim {dim}, {spec}")
    return RopeTable(cos, sin, layout)


def rope(x: torch.Tensor, positions: torch.Tensor, table: RopeTable,
         out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x [rows, heads, head_dim] rotated at ``positions`` [rows] (int32) into ``out`` (default: a
    new tensor like x; x itself is allowed).  wici_rope_rows."""
    device = _on_gpu(x, "x")
    if x.dim() != 3:
        raise ValueError(f"x: shape {tuple(x.shape)}, expected [rows, heads, head_dim]")
    n, h, d = x.shape
    if table.device != device:
        raise ValueError(f"table: on {table.device}, expected {device}")
    if table.cos.requires_grad or table.sin.requires_grad:
        _no_gradient("table")
    lib = binding.load_library()
    with _launch_on(stream, device, x, positions, out, table.cos, table.sin) as raw:
        xr = _rows(x, h, d, "x", device)
        given = out is not None
        if not given:
            out = _like(x)
            outr = _new_rows(out)
        elif out.shape[0] != n:
            raise ValueError(f"out: {out.shape[0]} rows, expected {n}")
        else:
            outr = _rows(out, h, d, "out", device)
        if n == 0:
            return out
        st = lib.wici_rope_rows(table._c, d, n, h, _ints(positions, (n,), "positions", device), xr,
                                outr, raw)
        if st:
            _check(st, f"rope: {h} heads of {d}, {table.dim} rotated (strides multiples of 8, "
                   "16-byte aligned rows)")
        if given:
            _written(out)
    return out


class KvCache:
    """An 8-bit paged KV cache (wici_kv8): ``pool`` uint8 [n_pages, 2, n_kv_heads,
    page * (head_dim + 4)] and ``table`` int32 [n_seqs, max_pages] naming each sequence's
    pages in order.  Both stay the caller's: pages are handed out by writing the table.

    ``length`` [n_seqs] (int32) counts each sequence's positions, the call's new rows
    included; without ``row_start`` [n_seqs + 1] (int32) a sequence has one new row, else rows
    row_start[b] .. row_start[b + 1].  Rows of no sequence are not used, and not written in
    outputs (a new output tensor holds nothing in particular there)."""

    def __init__(self, pool: torch.Tensor, table: torch.Tensor, *, page: int, head_dim: int):
        device = _on_gpu(pool, "pool")
        if pool.dtype != torch.uint8 or pool.dim() != 4 or not pool.is_contiguous() or \
                pool.shape[1] != 2 or pool.shape[3] != page * (head_dim + 4):
            raise ValueError(f"pool: {pool.dtype} {tuple(pool.shape)}, expected contiguous uint8 "
                             f"[n_pages, 2, n_kv_heads, {page * (head_dim + 4)}]")
        if table.dtype != torch.int32 or table.dim() != 2 or table.stride(1) != 1 or \
                table.shape[1] < 1 or table.device != device:
            raise ValueError(f"table: {table.dtype} {tuple(table.shape)}, expected int32 "
                             "[n_seqs, max_pages] on the pool's GPU")
        self.pool, self.table, self.page, self.head_dim = pool, table, page, head_dim
        self.n_kv_heads, self.device = pool.shape[2], device
        self.lib = binding.load_library()
        stride = table.stride(0) if table.shape[0] > 1 else table.shape[1]
        self._c = binding.WiciKv8(pool.data_ptr(), pool.shape[0], page, self.n_kv_heads, head_dim,
                                  table.data_ptr(), stride, table.shape[1])
        size = ctypes.c_size_t()
        _check(self.lib.wici_kv8_bytes(ctypes.byref(self._c), ctypes.byref(size)),
               f"KvCache: page {page}, head_dim {head_dim}, {self.n_kv_heads} KV heads")

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, table: torch.Tensor,
              page: int = 64) -> "KvCache":
        """A cache with a new pool on the table's GPU."""
        pool = torch.empty(n_pages, 2, n_kv_heads, page * (head_dim + 4), dtype=torch.uint8,
                           device=_on_gpu(table, "table"))
        return cls(pool, table, page=page, head_dim=head_dim)

    def _on(self, stream, *tensors):
        return _launch_on(stream, self.device, self.pool, self.table, *tensors)

    def _batch(self, n_rows, length, row_start, max_rows=0, max_length=0):
        n = length.shape[0]
        if n > self.table.shape[0]:
            raise ValueError(f"length: {n} sequences, the table has {self.table.shape[0]}")
        if row_start is None and n_rows != n:
            raise ValueError(f"{n_rows} rows for {n} sequences need row_start")
        start = None if row_start is None else _ints(row_start, (n + 1,), "row_start", self.device)
        return binding.WiciKv8Batch(n, n_rows, start, _ints(length, (n,), "length", self.device),
                                    max_rows, max_length)

    def append(self, k: torch.Tensor, v: torch.Tensor, length: torch.Tensor, *,
               row_start: torch.Tensor | None = None, rope: RopeTable | None = None,
               q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, stream=None):
        """Quantise the rows k and v [rows, n_kv_heads, head_dim] into the cache.  With ``rope``
        the keys are rotated at their positions first, and ``q`` [rows, heads, head_dim] into
        ``q_out`` (default: a new tensor like q; q itself is allowed), which is returned
        (None without q).  wici_kv8_append."""
        n, d, dev = k.shape[0], self.head_dim, self.device
        if v.shape[0] != n or (q is not None and q.shape[0] != n):
            raise ValueError("k, v and q have different numbers of rows")
        if q is not None and rope is None:
            raise ValueError("q is only rotated: it needs rope")
        if rope is not None and rope.device != dev:
            raise ValueError(f"rope: on {rope.device}, expected {dev}")
        if rope is not None and (rope.cos.requires_grad or rope.sin.requires_grad):
            _no_gradient("rope")
        with self._on(stream, k, v, length, row_start, q, q_out, rope and rope.cos,
                      rope and rope.sin) as raw:
            qr, qo, heads, given = _NO_ROWS, _NO_ROWS, 0, q is not None and q_out is not None
            if q is not None:
                heads = q.shape[1]
                qr = _rows(q, heads, d, "q", dev)
                if q_out is None:
                    q_out = _like(q)
                    qo = _new_rows(q_out)
                elif q_out.shape[0] != n:
                    raise ValueError(f"q_out: {q_out.shape[0]} rows, expected {n}")
                else:
                    qo = _rows(q_out, heads, d, "q_out", dev)
            kr, vr = _rows(k, self.n_kv_heads, d, "k", dev), _rows(v, self.n_kv_heads, d, "v", dev)
            _check(self.lib.wici_kv8_append(
                self._c, self._batch(n, length, row_start), None if rope is None else rope._c, heads,
                qr, qo, kr, vr, raw),
                "append (strides multiples of 8, 16-byte aligned rows, rope.dim <= head_dim)")
            _written((self.pool, q_out) if given else self.pool)
        return q_out if q is not None else None

    def read(self, length: torch.Tensor, *, row_start: torch.Tensor | None = None,
             n_rows: int | None = None, dtype: torch.dtype = torch.bfloat16,
             k: torch.Tensor | None = None, v: torch.Tensor | None = None, stream=None):
        """The values the cache holds for the rows: (k, v), each [rows, n_kv_heads, head_dim].  New
        tensors of ``dtype`` with ``n_rows`` rows (default: one a sequence) unless given.
        wici_kv8_read."""
        dev, d = self.device, self.head_dim
        if n_rows is None:
            n_rows = k.shape[0] if k is not None else v.shape[0] if v is not None else \
                length.shape[0]
        with self._on(stream, length, row_start, k, v) as raw:
            if dtype not in _DTYPES:
                raise TypeError(f"dtype {dtype} (float32 or bfloat16)")
            rows, given = [], [x for x in (k, v) if x is not None]
            for name, x in (("k", k), ("v", v)):
                if x is None:
                    x = torch.empty((n_rows, self.n_kv_heads, d), dtype=dtype, device=dev)
                    rows += [x, _new_rows(x)]
                elif x.shape[0] != n_rows:
                    raise ValueError(f"{name}: {x.shape[0]} rows, expected {n_rows}")
                else:
                    rows += [x, _rows(x, self.n_kv_heads, d, name, dev)]
            k, kr, v, vr = rows
            _check(self.lib.wici_kv8_read(self._c, self._batch(n_rows, length, row_start), kr, vr,
                                          raw),
                   "read (strides multiples of 8, 16-byte aligned rows)")
            if given:
                _written(given)
        return k, v

    def attend(self, q: torch.Tensor, length: torch.Tensor, *,
               row_start: torch.Tensor | None = None, scale: float | None = None,
               max_rows: int = 0, max_length: int = 0, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Causal attention of the rows q [rows, heads, head_dim] over the cache (append first):
        a row sees its sequence's positions up to its own; zeros where that is none.  ``scale``
        defaults to head_dim^-1/2.  ``max_rows`` and ``max_length`` (the most new rows and
        positions of a sequence, 0: unknown) only shape the launch.  ``out`` (default: a new
        tensor like q) and ``workspace`` (uint8, attend_workspace bytes; default: a new one) may
        be given.  wici_kv8_attend."""
        dev, d = self.device, self.head_dim
        if q.dim() != 3:
            raise ValueError(f"q: shape {tuple(q.shape)}, expected [rows, heads, {d}]")
        n, heads = q.shape[0], q.shape[1]
        with self._on(stream, q, length, row_start, out, workspace) as raw:
            b = self._batch(n, length, row_start, max_rows, max_length)
            qr = _rows(q, heads, d, "q", dev)
            given = out is not None
            if not given:
                out = _like(q)
                outr = _new_rows(out)
            elif out.shape[0] != n:
                raise ValueError(f"out: {out.shape[0]} rows, expected {n}")
            else:
                outr = _rows(out, heads, d, "out", dev)
            need = self._workspace(b, heads)
            if workspace is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
            elif workspace.device != dev or not workspace.is_contiguous():
                raise ValueError(f"workspace: contiguous on {dev} expected")
            size = 0 if workspace is None else workspace.numel() * workspace.element_size()
            st = self.lib.wici_kv8_attend(
                self._c, b, heads, d ** -0.5 if scale is None else scale, qr, outr,
                None if workspace is None else workspace.data_ptr(), size, raw)
            if st:
                _check(st, f"attend: {heads} query heads on {self.n_kv_heads}, {need} workspace "
                       "bytes (strides multiples of 8, 16-byte aligned rows)")
            if given:
                _written(out)
        return out

    def _workspace(self, batch, heads: int) -> int:
        size = ctypes.c_size_t()
        st = self.lib.wici_kv8_attend_workspace(self._c, batch, heads, size)
        if st:
            _check(st, f"attend: {heads} query heads on {self.n_kv_heads}")
        return size.value

    def attend_workspace(self, n_rows: int, heads: int, n_seqs: int, *, row_start: bool = False,
                         max_rows: int = 0, max_length: int = 0) -> int:
        """Bytes of workspace attend needs for such a call (0: none)."""
        return self._workspace(binding.WiciKv8Batch(n_seqs, n_rows, 1 if row_start else None, None,
                                                    max_rows, max_length), heads)
