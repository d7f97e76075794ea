"""Python binding of the attention calls of libspconv.so (C ABI declared in
include/spconv_attention.h): rotary positions, the paged cache's append, block
scores, block selection and attention over the listed blocks.

Argument marshalling only, as in ``spconv``: device buffers are torch CUDA (HIP)
tensors, streams are torch streams, every computation happens in the library, and
errors are ``SpconvError``, ``TypeError`` and ``ValueError``. ``BlockAttention``
strings the calls of one step together.

Queries, keys and outputs are [tokens, heads, dim] tensors with any strides whose
last is 1; caches are [pages, heads, block, dim], key sums [pages, heads, dim].
No gradients are recorded: tensors that require them are refused while torch records.
"""
from __future__ import annotations

import ctypes
from contextlib import contextmanager
from functools import lru_cache
from operator import index

import numpy as np
import torch

from . import spconv
from .spconv import SPCONV_EINVAL, SPCONV_EHIP, SPCONV_OK, SpconvError  # noqa: F401

EXPORTED = ("spconv_batch_rows", "spconv_rope_frequencies", "spconv_rope", "spconv_cache_append", "spconv_block_scores",
            "spconv_select_blocks", "spconv_attention_workspace", "spconv_block_attention")
SPCONV_F32 = 0
SPCONV_F16 = 1
SPCONV_BF16 = 2
SPCONV_ROPE_INTERLEAVED = 1
SPCONV_ROPE_INVERSE = 2
SPCONV_ROPE_PLAIN = 0
SPCONV_ROPE_LINEAR = 1
SPCONV_ROPE_BASE = 2
SPCONV_ROPE_BY_PARTS = 3

_DTYPES = {torch.float32: SPCONV_F32, torch.float16: SPCONV_F16, torch.bfloat16: SPCONV_BF16}


class spconv_batch(ctypes.Structure):
    """Mirror of ``struct spconv_batch``."""
    _fields_ = [("sequences", ctypes.c_int32), ("block", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("q_block", ctypes.c_int32), ("tokens", ctypes.c_int64), ("pages", ctypes.c_int64),
                ("table_stride", ctypes.c_int64), ("table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("q_start", ctypes.c_void_p)]


class spconv_rope_scaling(ctypes.Structure):
    """Mirror of ``struct spconv_rope_scaling``."""
    _fields_ = [("kind", ctypes.c_int32), ("factor", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("original", ctypes.c_double)]


_int, _i64, _u32, _f32, _vp = ctypes.c_int, ctypes.c_int64, ctypes.c_uint32, ctypes.c_float, ctypes.c_void_p
_batch_p = ctypes.POINTER(spconv_batch)


def _bind(lib):
    """Declare the C signatures on the loaded libspconv.so and return it."""
    lib.spconv_batch_rows.argtypes = [_batch_p, ctypes.POINTER(_i64)]
    lib.spconv_rope_frequencies.argtypes = [_int, ctypes.c_double, ctypes.POINTER(spconv_rope_scaling), _vp]
    lib.spconv_rope.argtypes = [_int, _vp, _i64, _i64, _i64, _int, _int, _vp, _vp, _int, _u32, _f32, _vp, _i64, _i64, _vp]
    lib.spconv_cache_append.argtypes = [_int, _batch_p, _vp, _i64, _i64, _vp, _i64, _i64, _int, _int, _vp, _vp, _int,
                                        _u32, _f32, _vp, _vp, _vp, _vp]
    lib.spconv_block_scores.argtypes = [_int, _batch_p, _vp, _i64, _i64, _int, _int, _int, _vp, _vp, _vp]
    lib.spconv_select_blocks.argtypes = [_batch_p, _int, _vp, _int, _int, _int, _vp, _vp, _vp]
    lib.spconv_attention_workspace.argtypes = [_int, _batch_p, _int, _int, _int, _int, ctypes.POINTER(_i64)]
    lib.spconv_block_attention.argtypes = [_int, _batch_p, _vp, _i64, _i64, _int, _int, _int, _vp, _vp, _f32, _vp, _vp,
                                           _int, _vp, _i64, _i64, _vp, _vp, _i64, _vp]
    for name in EXPORTED:
        getattr(lib, name).restype = _int
    return lib


_lib = _bind(spconv._lib)
_check = spconv._check


def _device(t, name):
    """The device of a call: that of its first tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    return t.device


def _refuse_grad(name):
    raise ValueError(f"{name} requires grad, and the calls record no gradients: use torch.no_grad() or detach() (the "
                     "gradient of spconv_rope is the call with inverse=True)")


def _rows(t, name, dtype, shape, device):
    """Pointer and strides of a [tokens, heads, dim] tensor of these."""
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    a, b, c = t.stride()
    if c != 1 and shape[2] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse_grad(name)
    # A dimension of one element is never stepped over: its stride says nothing.
    return t.data_ptr(), a if shape[0] > 1 else shape[2], b if shape[1] > 1 else shape[2]


def _whole(t, name, dtype, shape, device):
    """Pointer of a contiguous tensor of these."""
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype is not dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse_grad(name)
    return t.data_ptr()


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, not {t.dtype}")
    return code


def _dims(t, name, what):
    """Shape of a tensor of such dimensions."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dim() != len(what):
        raise ValueError(f"{name} must be [{', '.join(what)}]")
    return t.shape


_QUERIES = ("tokens", "heads", "dim")
_CACHE = ("pages", "heads", "block", "dim")


class _Here:
    """A call on the current device and its current stream: nothing to switch."""
    __slots__ = ("_raw",)

    def __init__(self, raw):
        self._raw = raw

    def __enter__(self):
        return self._raw

    def __exit__(self, *exc):
        return False


@contextmanager
def _elsewhere(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream(device).cuda_stream
        else:
            if stream.device != device:
                raise ValueError(f"stream belongs to {stream.device}, the tensors to {device}")
            with torch.cuda.stream(stream):
                yield stream.cuda_stream


def _on(device, stream):
    """The device a call runs on made current, and its raw stream (torch's current one without ``stream``).
    Outputs and scratch memory are allocated inside, so that they belong to that stream."""
    # (The usual case asks torch for two numbers: its Python classes for them take 4 us, as long as a launch.)
    if stream is None and device.index == torch._C._cuda_getDevice():
        return _Here(torch._C._cuda_getCurrentRawStream(device.index))
    return _elsewhere(device, stream)


@lru_cache(maxsize=1024)
def _batch_rows(sequences, block, max_blocks, q_block, tokens, stride, one_each):
    """Rows of a batch, and its checks: a function of these sizes alone (the batch's arrays are not looked at)."""
    rows = _i64()
    batch = spconv_batch(sequences, block, max_blocks, q_block, tokens, 1, stride, None, None, None if one_each else 16)
    _check(_lib.spconv_batch_rows(batch, rows), "spconv_batch_rows")
    return rows.value


class CacheBatch:
    """The sequences of a step (``struct spconv_batch``): ``table`` int32 [sequences, blocks] (pages), ``kv_len``
    int32 [sequences] (keys, the new ones among them), ``block`` keys to a page, ``q_start`` int32 [sequences + 1] (the
    tokens of each; without it one each), ``tokens`` of the packed tensors (default: ``sequences``), ``q_block`` tokens
    to a row. The tensors are read when a call's kernels run, so they may be updated in place between steps."""

    def __init__(self, table, kv_len, block: int, q_start=None, tokens: int | None = None, q_block: int = 1):
        self.device = _device(table, "table")
        if table.dtype is not torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise TypeError("table must be an int32 [sequences, blocks] tensor with contiguous rows")
        B, nb = table.shape
        block, q_block = index(block), index(q_block)  # (an equal float would find what is remembered for the number)
        tokens = None if tokens is None else index(tokens)
        stride = table.stride(0) if B > 1 else nb
        _whole(kv_len, "kv_len", torch.int32, (B,), self.device)
        if q_start is not None:
            _whole(q_start, "q_start", torch.int32, (B + 1,), self.device)
        elif tokens is None:
            tokens = B
        if tokens is None:
            raise ValueError("a batch with q_start needs the number of tokens")
        self.table, self.kv_len, self.q_start = table, kv_len, q_start  # kept alive
        self.sequences, self.max_blocks, self.block, self.q_block, self.tokens = B, nb, block, q_block, tokens
        self._fields = (B, block, nb, q_block, tokens, stride, table.data_ptr(), kv_len.data_ptr(),
                        None if q_start is None else q_start.data_ptr())
        self.rows = _batch_rows(B, block, nb, q_block, tokens, stride, q_start is None)
        self._last = (0, None)

    def with_pages(self, pages: int) -> spconv_batch:
        """The struct for a call on a cache of this many pages (never changed: calls and threads may share it)."""
        last = self._last
        if last[0] != pages:
            f = self._fields
            self._last = last = (pages, spconv_batch(f[0], f[1], f[2], f[3], f[4], pages, f[5], f[6], f[7], f[8]))
        return last[1]


def _scaling(scaling):
    if scaling is None:
        return None
    if isinstance(scaling, spconv_rope_scaling):
        return scaling
    kinds = {"plain": SPCONV_ROPE_PLAIN, "linear": SPCONV_ROPE_LINEAR, "base": SPCONV_ROPE_BASE, "by_parts": SPCONV_ROPE_BY_PARTS}
    values = dict(scaling)
    kind = values.pop("kind")
    if kind not in kinds:
        raise ValueError(f"unknown scaling {kind!r}")
    if set(values) - {"factor", "low", "high", "original"}:
        raise ValueError(f"unknown scaling fields {sorted(set(values) - {'factor', 'low', 'high', 'original'})}")
    return spconv_rope_scaling(kinds[kind], values.get("factor", 1.0), values.get("low", 0.0), values.get("high", 0.0),
                               values.get("original", 0.0))


def spconv_rope_frequencies(rot: int, base: float = 10000.0, scaling=None, device=None):
    """Angle per position of each of ``rot``/2 pairs: float64 numpy array, or a tensor on ``device``. ``scaling``: a
    ``spconv_rope_scaling`` or a dict with ``kind`` "linear", "base" (both with ``factor``) or "by_parts" (also ``low``,
    ``high``, ``original``)."""
    freq = np.empty(max(rot // 2, 1), np.float64)
    s = _scaling(scaling)
    _check(_lib.spconv_rope_frequencies(rot, base, None if s is None else ctypes.byref(s), freq.ctypes.data),
           "spconv_rope_frequencies")
    return freq if device is None else torch.from_numpy(freq).to(device)


def _freq(freq, device):
    if freq is None:
        return None, 0
    if not isinstance(freq, torch.Tensor) or freq.device != device or freq.dtype is not torch.float64 or freq.dim() != 1 \
            or not freq.is_contiguous():
        raise TypeError(f"freq must be a contiguous one-dimensional float64 tensor on {device}")
    if freq.requires_grad and torch.is_grad_enabled():
        _refuse_grad("freq")
    n = freq.numel()
    return (freq.data_ptr(), 2 * n) if n else (None, 0)


def spconv_rope(x, positions, freq, interleaved: bool = False, inverse: bool = False, amplitude: float = 1.0, out=None,
                stream=None):
    """``x`` [tokens, heads, dim] rotated by ``positions`` (int32 [tokens]) in its first 2*len(``freq``) components.
    ``inverse`` turns back: with the same ``amplitude`` it is the gradient, with 1 / ``amplitude`` it undoes the rotation.
    ``out`` may be ``x``."""
    device = _device(x, "x")
    T, H, D = _dims(x, "x", _QUERIES)
    code = _dtype(x, "x")
    xp, xt, xh = _rows(x, "x", x.dtype, (T, H, D), device)
    pp = _whole(positions, "positions", torch.int32, (T,), device)
    fp, rot = _freq(freq, device)
    flags = (SPCONV_ROPE_INTERLEAVED if interleaved else 0) | (SPCONV_ROPE_INVERSE if inverse else 0)
    with _on(device, stream) as raw:
        if out is None:
            out = x.new_empty((T, H, D))
        op, ot, oh = _rows(out, "out", x.dtype, (T, H, D), device)
        _check(_lib.spconv_rope(code, xp, xt, xh, T, H, D, pp, fp, rot, flags, amplitude, op, ot, oh, raw), "spconv_rope")
    return out


def _cache(k_cache, v_cache, batch, heads, dim, dtype, device):
    shape = (_dims(k_cache, "k_cache", _CACHE)[0], heads, batch.block, dim)
    return _whole(k_cache, "k_cache", dtype, shape, device), _whole(v_cache, "v_cache", dtype, shape, device), shape[0]


def spconv_cache_append(k, v, k_cache, v_cache, batch: CacheBatch, sums=None, freq=None, interleaved: bool = False,
                        amplitude: float = 1.0, positions=None, stream=None):
    """Store the step's ``k`` and ``v`` [tokens, heads, dim] in the cache (keys rotated on the way with ``freq``, by their
    place in the sequence or by ``positions``) and set ``sums`` of the pages that got keys."""
    device = batch.device
    T, H, D = _dims(k, "k", _QUERIES)
    if T != batch.tokens:
        raise ValueError(f"k has {T} tokens, the batch {batch.tokens}")
    code = _dtype(k, "k")
    kp, kt, kh = _rows(k, "k", k.dtype, (T, H, D), device)
    vp, vt, vh = _rows(v, "v", k.dtype, (T, H, D), device)
    kc, vc, pages = _cache(k_cache, v_cache, batch, H, D, k.dtype, device)
    sp = None if sums is None else _whole(sums, "sums", torch.float32, (pages, H, D), device)
    pp = None if positions is None else _whole(positions, "positions", torch.int32, (T,), device)
    fp, rot = _freq(freq, device)
    flags = SPCONV_ROPE_INTERLEAVED if interleaved else 0
    with _on(device, stream) as raw:
        _check(_lib.spconv_cache_append(code, batch.with_pages(pages), kp, kt, kh, vp, vt, vh, H, D, pp, fp, rot, flags,
                                        amplitude, kc, vc, sp, raw), "spconv_cache_append")


def spconv_block_scores(q, sums, batch: CacheBatch, out=None, stream=None):
    """Scores [rows, heads, blocks] of every block of the cache for every row of ``q`` [tokens, q_heads, dim], by the
    blocks' key ``sums`` [pages, heads, dim]."""
    device = batch.device
    T, HQ, D = _dims(q, "q", _QUERIES)
    if T != batch.tokens:
        raise ValueError(f"q has {T} tokens, the batch {batch.tokens}")
    pages, H, _ = _dims(sums, "sums", ("pages", "heads", "dim"))
    code = _dtype(q, "q")
    qp, qt, qh = _rows(q, "q", q.dtype, (T, HQ, D), device)
    sp = _whole(sums, "sums", torch.float32, (pages, H, D), device)
    shape = (batch.rows, H, batch.max_blocks)
    with _on(device, stream) as raw:
        if out is None:
            out = sums.new_empty(shape)
        op = _whole(out, "out", torch.float32, shape, device)
        _check(_lib.spconv_block_scores(code, batch.with_pages(pages), qp, qt, qh, HQ, H, D, sp, op, raw),
               "spconv_block_scores")
    return out


def spconv_select_blocks(scores, batch: CacheBatch, keep: int, sink: int = 1, local: int = 1, out=None, stream=None):
    """(blocks int32 [rows, heads, keep], counts int32 [rows, heads]): the blocks that each row reads, ascending, -1 behind
    them: the first ``sink``, the row's own and the ``local`` - 1 before them, and the best scored others. ``out``: such a
    pair to write into."""
    device = batch.device
    H = _dims(scores, "scores", ("rows", "heads", "blocks"))[1]
    sp = _whole(scores, "scores", torch.float32, (batch.rows, H, batch.max_blocks), device)
    with _on(device, stream) as raw:
        if out is None:
            # Only sizes that the call accepts are allocated.
            if not 1 <= keep < 1 << 31:
                raise SpconvError(SPCONV_EINVAL, "spconv_select_blocks")
            out = (scores.new_empty((batch.rows, H, keep), dtype=torch.int32),
                   scores.new_empty((batch.rows, H), dtype=torch.int32))
        bp = _whole(out[0], "blocks", torch.int32, (batch.rows, H, keep), device)
        cp = _whole(out[1], "counts", torch.int32, (batch.rows, H), device)
        _check(_lib.spconv_select_blocks(batch.with_pages(1), H, sp, keep, sink, local, bp, cp, raw), "spconv_select_blocks")
    return out


@lru_cache(maxsize=1024)
def _workspace(code, sequences, block, max_blocks, q_block, tokens, one_each, q_heads, heads, dim, keep):
    """Bytes of scratch memory: a function of these sizes alone (the batch's arrays are not looked at)."""
    n = _i64()
    batch = spconv_batch(sequences, block, max_blocks, q_block, tokens, 1, max_blocks, None, None, None if one_each else 16)
    _check(_lib.spconv_attention_workspace(code, batch, q_heads, heads, dim, keep, n), "spconv_attention_workspace")
    return n.value


def spconv_attention_workspace(dtype, batch: CacheBatch, q_heads: int, heads: int, dim: int, keep: int = 0) -> int:
    """Bytes of scratch memory of a ``spconv_block_attention`` call of these sizes."""
    if dtype not in _DTYPES:
        raise TypeError(f"dtype must be float32, float16 or bfloat16, not {dtype}")
    q_heads, heads, dim, keep = index(q_heads), index(heads), index(dim), index(keep)  # (equal floats are remembered sizes, too)
    return _workspace(_DTYPES[dtype], batch.sequences, batch.block, batch.max_blocks, batch.q_block, batch.tokens,
                      batch.q_start is None, q_heads, heads, dim, keep)


def spconv_block_attention(q, k_cache, v_cache, batch: CacheBatch, blocks=None, counts=None, scale: float | None = None,
                           out=None, lse=None, workspace=None, stream=None):
    """Causal softmax attention of ``q`` [tokens, q_heads, dim] over the blocks that each row lists (``blocks`` int32
    [rows, heads, keep], ``counts`` int32 [rows, heads] or None), or over every block that it sees. ``scale`` defaults to
    dim**-0.5. ``lse`` True, or a float32 [tokens, q_heads] tensor, asks for the log-sum-exp: the call then returns (out,
    lse). ``workspace``: a uint8 tensor of ``spconv_attention_workspace`` bytes; without it one is allocated on the stream.
    Tokens that no sequence has are left as they are (in new outputs: unset)."""
    device = batch.device
    T, HQ, D = _dims(q, "q", _QUERIES)
    if T != batch.tokens:
        raise ValueError(f"q has {T} tokens, the batch {batch.tokens}")
    H = _dims(k_cache, "k_cache", _CACHE)[1]
    code = _dtype(q, "q")
    qp, qt, qh = _rows(q, "q", q.dtype, (T, HQ, D), device)
    kc, vc, pages = _cache(k_cache, v_cache, batch, H, D, q.dtype, device)
    keep, bp, cp = 0, None, None
    if blocks is not None:
        keep = _dims(blocks, "blocks", ("rows", "heads", "keep"))[2]
        if keep == 0:  # (it has no address, which would stand for no lists: all blocks)
            raise SpconvError(SPCONV_EINVAL, "spconv_block_attention")
        bp = _whole(blocks, "blocks", torch.int32, (batch.rows, H, keep), device)
    if counts is not None:
        cp = _whole(counts, "counts", torch.int32, (batch.rows, H), device)
    struct = batch.with_pages(pages)
    need = _workspace(code, batch.sequences, batch.block, batch.max_blocks, batch.q_block, batch.tokens,
                      batch.q_start is None, HQ, H, D, keep)
    with _on(device, stream) as raw:
        if out is None:
            out = q.new_empty((T, HQ, D))
        op, ot, oh = _rows(out, "out", q.dtype, (T, HQ, D), device)
        if lse is True:
            lse = q.new_empty((T, HQ), dtype=torch.float32)
        lp = None if lse is None or lse is False else _whole(lse, "lse", torch.float32, (T, HQ), device)
        wp, size = None, 0
        if need:
            if workspace is None:
                workspace = q.new_empty(need, dtype=torch.uint8)
            if not isinstance(workspace, torch.Tensor) or workspace.device != device or not workspace.is_contiguous():
                raise TypeError(f"workspace must be a contiguous tensor on {device}")
            wp, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        _check(_lib.spconv_block_attention(code, struct, qp, qt, qh, HQ, H, D, kc, vc,
                                           D ** -0.5 if scale is None else scale, bp, cp, keep, op, ot, oh, lp, wp, size,
                                           raw), "spconv_block_attention")
    return out if lp is None else (out, lse)


class BlockAttention:
    """One attention layer's device state: its paged cache, key sums and rotary table, ready to run.

    ``step(q, k, v, batch)`` queues what a step of the layer needs on the current stream: rotates the queries, appends keys
    and values, scores and selects ``keep`` blocks for each row and attends over them; ``keep`` 0 attends over all blocks
    without a selection. The caller owns the pages: which sequence has which is the ``batch``'s table."""

    def __init__(self, pages: int, heads: int, dim: int, block: int = 64, keep: int = 0, sink: int = 1, local: int = 1,
                 rot: int | None = None, base: float = 10000.0, scaling=None, interleaved: bool = False,
                 amplitude: float = 1.0, scale: float | None = None, dtype=torch.bfloat16, device="cuda"):
        self.heads, self.dim, self.block, self.keep, self.sink, self.local = heads, dim, block, keep, sink, local
        self.interleaved, self.amplitude, self.scale = interleaved, amplitude, scale
        rot = dim if rot is None else rot
        self.freq = spconv_rope_frequencies(rot, base, scaling, device) if rot else None
        self.k_cache = torch.empty((pages, heads, block, dim), dtype=dtype, device=device)
        self.v_cache = torch.empty_like(self.k_cache)
        self.sums = torch.empty((pages, heads, dim), dtype=torch.float32, device=device) if keep else None

    def rotate(self, q, positions, out=None, stream=None):
        """Queries rotated by their ``positions``."""
        return spconv_rope(q, positions, self.freq, self.interleaved, amplitude=self.amplitude, out=out, stream=stream)

    def append(self, k, v, batch: CacheBatch, stream=None, positions=None):
        """Keys and values of a step into the cache, keys rotated by their place in the sequence or by ``positions``."""
        spconv_cache_append(k, v, self.k_cache, self.v_cache, batch, self.sums, self.freq, self.interleaved,
                            self.amplitude, positions, stream=stream)

    def select(self, q, batch: CacheBatch, stream=None):
        """(blocks, counts) that the rows of the rotated ``q`` read; (None, None) without a selection."""
        if not self.keep:
            return None, None
        scores = spconv_block_scores(q, self.sums, batch, stream=stream)
        return spconv_select_blocks(scores, batch, self.keep, self.sink, self.local, stream=stream)

    def attend(self, q, batch: CacheBatch, blocks=None, counts=None, out=None, lse=None, stream=None):
        """Attention of the rotated ``q`` over the listed blocks of the cache."""
        return spconv_block_attention(q, self.k_cache, self.v_cache, batch, blocks, counts, self.scale, out, lse,
                                      stream=stream)

    def step(self, q, k, v, positions, batch: CacheBatch, out=None, lse=None, stream=None):
        """One step: ``q`` [tokens, q_heads, dim], ``k`` and ``v`` [tokens, heads, dim] as projected, ``positions`` int32
        [tokens] by which queries and keys are rotated (those of the tokens in their sequences, or others that the model
        counts in; where keys lie and what a token sees goes by the batch alone). Returns the attention's output (and
        log-sum-exp, if asked for)."""
        if self.freq is None:
            positions = None
        else:
            q = self.rotate(q, positions, stream=stream)
        self.append(k, v, batch, stream=stream, positions=positions)
        blocks, counts = self.select(q, batch, stream=stream)
        return self.attend(q, batch, blocks, counts, out, lse, stream=stream)
