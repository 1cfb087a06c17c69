"""Binding of the 8-bit paged key/value cache, its attention, its pages, and the choice of the next token (include/sfmp.h).

Arguments are torch tensors on the GPU; a tensor of another type, shape or layout than a call takes raises ValueError (the
library's own refusals raise SfmpError).  Launches are marshalled by the extension where it takes them, else here."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional

from .binding import (SfmpKvBatch, SfmpKvLayout, SfmpKvTables, _check, _launcher, _stream_ptr, load_library)

KV_PAGE = 64
KV_FORMATS = {"int8": 0, "fp8": 1}


@dataclass
class DeviceKvCache:
    """The pool: codes uint8 [layers, pages, kv_heads, 2, 64 * head_dim], scales fp32 [layers, pages, kv_heads, 2]."""
    layout: SfmpKvLayout
    codes: object
    scales: object


@dataclass
class DeviceKvTables:
    """page_table int32 [sequences, table_pages], lengths int32 [sequences], refs int32 [pages]."""
    page_table: object
    lengths: object
    refs: object


def _int(x, what: str) -> int:
    """A number that the C call takes as int32 (ctypes would cut it off)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{what} has to fit 32 bits, got {x}")
    return x


def sfmp_kv_query(pages: int, kv_heads: int, head_dim: int, format: str = "int8", layers: int = 1) -> SfmpKvLayout:
    """Layout of a pool; format "int8", "fp8" or the header's integer."""
    out = SfmpKvLayout()
    fmt = KV_FORMATS[format] if isinstance(format, str) else _int(format, "format")
    _check(load_library().sfmp_kv_query(_int(pages, "pages"), _int(kv_heads, "kv_heads"), _int(head_dim, "head_dim"), fmt,
                                        _int(layers, "layers"), C.byref(out)))
    return out


def make_kv_cache(layout: SfmpKvLayout, device="cuda:0") -> DeviceKvCache:
    """A pool of this layout, its contents not initialised (no call reads a slot that no token was written to)."""
    import torch
    shape = (layout.layers, layout.pages, layout.kv_heads, 2)
    return DeviceKvCache(layout, torch.empty((*shape, KV_PAGE * layout.head_dim), dtype=torch.uint8, device=device),
                         torch.empty(shape, dtype=torch.float32, device=device))


def make_kv_tables(layout: SfmpKvLayout, sequences: int, table_pages: int, device="cuda:0") -> DeviceKvTables:
    """Tables of `sequences` empty sequences of up to 64 * table_pages tokens over a pool of free pages."""
    import torch
    z = dict(dtype=torch.int32, device=device)
    return DeviceKvTables(torch.full((sequences, table_pages), -1, **z), torch.zeros(sequences, **z),
                          torch.zeros(layout.pages, **z))


def _types():
    import torch
    return {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


def _tensor(t, what: str, dtype: str, *shape):
    """Address of a contiguous GPU tensor of this type and shape (None in `shape`: any extent); None stays None."""
    if t is None:
        return None
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} has to be a tensor on the GPU")
    if t.dtype != getattr(torch, dtype):
        raise ValueError(f"{what} has to be {dtype}, got {t.dtype}")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{what} has to be of shape {['any' if n is None else n for n in shape]}, got {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} has to be contiguous")
    return t.data_ptr() or None


def _rows(t, what: str, types, heads: Optional[int], dim: int):
    """(address, type, row stride) of [rows, heads, dim] whose rows are contiguous inside but may lie apart."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} has to be a tensor on the GPU")
    if t.dtype not in types:
        raise ValueError(f"{what} has to be one of {[str(x) for x in types]}, got {t.dtype}")
    if t.dim() != 3 or (heads is not None and t.shape[1] != heads) or t.shape[2] != dim:
        raise ValueError(f"{what} has to be of shape [rows, {heads or 'heads'}, {dim}], got {list(t.shape)}")
    width = t.shape[1] * dim
    if t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != dim):
        raise ValueError(f"{what}: the heads of a row have to be contiguous")
    return t.data_ptr() or None, _types()[t.dtype], t.stride(0) if t.shape[0] > 1 else (width + 7) // 8 * 8


def _cache(cache: DeviceKvCache):
    L = cache.layout
    shape = (L.layers, L.pages, L.kv_heads, 2)
    return (C.byref(L), _tensor(cache.codes, "codes", "uint8", *shape, KV_PAGE * L.head_dim),
            _tensor(cache.scales, "scales", "float32", *shape))


def _tables(layout: SfmpKvLayout, t: DeviceKvTables):
    table = _tensor(t.page_table, "page_table", "int32", None, None)
    sequences, width = (0, 0) if t.page_table is None else t.page_table.shape
    return SfmpKvTables(table, _tensor(t.lengths, "lengths", "int32", sequences), _tensor(t.refs, "refs", "int32", layout.pages),
                        _int(sequences, "sequences"), _int(width, "table_pages"))


def _length(t, what: str) -> int:
    """Elements of a vector."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dim() != 1:
        raise ValueError(f"{what} has to be a vector on the GPU, got {type(t).__name__ if not isinstance(t, torch.Tensor) else list(t.shape)}")
    return t.shape[0]


def _batch(tables: DeviceKvTables, slots, row_start, rows: int, max_rows: int) -> SfmpKvBatch:
    batch = _length(slots, "slots") if slots is not None else _length(row_start, "row_start") - 1 if row_start is not None else rows
    return SfmpKvBatch(_tensor(slots, "slots", "int32", None), _tensor(row_start, "row_start", "int32", batch + 1), _int(batch, "batch"),
                       _int(rows, "rows"), _int(max_rows, "max_rows"), 0)


def _workspace(t):
    """(address, bytes) of a contiguous GPU tensor of any type; None and an empty one are left to the library's check."""
    import torch
    if t is None or (isinstance(t, torch.Tensor) and t.numel() == 0):
        return None, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise ValueError("workspace has to be a contiguous tensor on the GPU")
    return C.c_void_p(t.data_ptr()), t.numel() * t.element_size()


def sfmp_kv_append(cache: DeviceKvCache, layer: int, tables: DeviceKvTables, slots, row_start, K, V, max_rows: int,
                   stream=None) -> None:
    """K, V: fp16 or bf16 [rows, kv_heads, head_dim], the last tokens of the sequences slots (None: 0, 1, ...); entry b owns
    the rows row_start[b] .. row_start[b + 1] - 1 (None: row b), max_rows of them at most."""
    rc = _launcher().kv_append(cache, layer, tables, slots, row_start, K, V, max_rows, stream)
    if rc is not None:
        return _check(rc)
    import torch
    L = cache.layout
    layout, codes, scales = _cache(cache)
    types = (torch.float16, torch.bfloat16)
    k, dtype, k_stride = _rows(K, "K", types, L.kv_heads, L.head_dim)
    v, v_dtype, v_stride = _rows(V, "V", types, L.kv_heads, L.head_dim)
    if V.shape != K.shape or v_dtype != dtype:
        raise ValueError("K and V have to be of one shape and type")
    t, b = _tables(L, tables), _batch(tables, slots, row_start, K.shape[0], max_rows)
    _check(load_library().sfmp_kv_append(layout, _int(layer, "layer"), codes, scales, C.byref(t), C.byref(b), k, v, dtype, k_stride, v_stride,
                                         _stream_ptr(stream)))


def sfmp_kv_gather(cache: DeviceKvCache, layer: int, tables: DeviceKvTables, slots, first, row_start, K, V, max_rows: int,
                   stream=None) -> None:
    """Reads the tokens from first[b] on into the rows of entry b of K and V (fp16, bf16 or fp32)."""
    rc = _launcher().kv_gather(cache, layer, tables, slots, first, row_start, K, V, max_rows, stream)
    if rc is not None:
        return _check(rc)
    L = cache.layout
    layout, codes, scales = _cache(cache)
    k, dtype, k_stride = _rows(K, "K", _types(), L.kv_heads, L.head_dim)
    v, v_dtype, v_stride = _rows(V, "V", _types(), L.kv_heads, L.head_dim)
    if V.shape != K.shape or v_dtype != dtype:
        raise ValueError("K and V have to be of one shape and type")
    t, b = _tables(L, tables), _batch(tables, slots, row_start, K.shape[0], max_rows)
    _check(load_library().sfmp_kv_gather(layout, _int(layer, "layer"), codes, scales, C.byref(t), C.byref(b),
                                         _tensor(first, "first", "int32", b.batch), k, v, dtype, k_stride, v_stride, _stream_ptr(stream)))


def sfmp_kv_attention_workspace(layout: SfmpKvLayout, batch: int, rows: int, q_heads: int, max_rows: int, max_tokens: int) -> int:
    """Bytes that are enough for these sizes and for smaller ones."""
    n = C.c_int64(0)
    _check(load_library().sfmp_kv_attention_workspace(C.byref(layout), _int(batch, "batch"), _int(rows, "rows"), _int(q_heads, "q_heads"),
                                                      _int(max_rows, "max_rows"), _int(max_tokens, "max_tokens"), C.byref(n)))
    return int(n.value)


def sfmp_kv_attention(cache: DeviceKvCache, layer: int, tables: DeviceKvTables, slots, row_start, Q, O, max_rows: int,
                      max_tokens: int, scale: float, workspace, window: int = 0, lse=None, stream=None) -> None:
    """Attention of the rows Q (fp16 or bf16 [rows, q_heads, head_dim]) over their sequences' cached tokens into O (same type
    and shape) and, if given, lse (fp32 [rows, q_heads])."""
    rc = _launcher().kv_attention(cache, layer, tables, slots, row_start, Q, O, max_rows, max_tokens, scale, workspace, window,
                                  lse, stream)
    if rc is not None:
        return _check(rc)
    import torch
    L = cache.layout
    layout, codes, scales = _cache(cache)
    types = (torch.float16, torch.bfloat16)
    q, dtype, q_stride = _rows(Q, "Q", types, None, L.head_dim)
    o, o_dtype, o_stride = _rows(O, "O", types, None, L.head_dim)
    if O.shape != Q.shape or o_dtype != dtype:
        raise ValueError("Q and O have to be of one shape and type")
    t, b = _tables(L, tables), _batch(tables, slots, row_start, Q.shape[0], max_rows)
    at, size = _workspace(workspace)
    _check(load_library().sfmp_kv_attention(layout, _int(layer, "layer"), codes, scales, C.byref(t), C.byref(b), q, _int(Q.shape[1], "q_heads"),
                                            dtype, q_stride, _int(max_tokens, "max_tokens"), _int(window, "window"), float(scale), o, o_stride,
                                            _tensor(lse, "lse", "float32", Q.shape[0], Q.shape[1]), at, size, _stream_ptr(stream)))


def sfmp_kv_pages_workspace(layout: SfmpKvLayout) -> int:
    n = C.c_int64(0)
    _check(load_library().sfmp_kv_pages_workspace(C.byref(layout), C.byref(n)))
    return int(n.value)


def sfmp_kv_reserve(cache: DeviceKvCache, tables: DeviceKvTables, slots, counts, status, workspace, stream=None) -> None:
    """Room for counts[i] (None: one) more tokens of sequence slots[i]; status: int32 [1]."""
    rc = _launcher().kv_reserve(cache, tables, slots, counts, status, workspace, stream)
    if rc is not None:
        return _check(rc)
    layout, codes, scales = _cache(cache)
    t, n = _tables(cache.layout, tables), _length(slots, "slots")
    at, size = _workspace(workspace)
    _check(load_library().sfmp_kv_reserve(layout, codes, scales, C.byref(t), _tensor(slots, "slots", "int32", n),
                                          _tensor(counts, "counts", "int32", n), n, _tensor(status, "status", "int32", 1), at, size,
                                          _stream_ptr(stream)))


def sfmp_kv_fork(cache: DeviceKvCache, tables: DeviceKvTables, parents, children, stream=None) -> None:
    """children[i] (empty before) holds the tokens of parents[i], in the same pages."""
    rc = _launcher().kv_fork(cache, tables, parents, children, stream)
    if rc is not None:
        return _check(rc)
    t, n = _tables(cache.layout, tables), _length(parents, "parents")
    _check(load_library().sfmp_kv_fork(C.byref(cache.layout), C.byref(t), _tensor(parents, "parents", "int32", n),
                                       _tensor(children, "children", "int32", n), n, _stream_ptr(stream)))


def sfmp_kv_free(cache: DeviceKvCache, tables: DeviceKvTables, slots, keep=None, stream=None) -> None:
    """Sequence slots[i] keeps its first keep[i] tokens (None: none)."""
    rc = _launcher().kv_free(cache, tables, slots, keep, stream)
    if rc is not None:
        return _check(rc)
    t, n = _tables(cache.layout, tables), _length(slots, "slots")
    _check(load_library().sfmp_kv_free(C.byref(cache.layout), C.byref(t), _tensor(slots, "slots", "int32", n),
                                       _tensor(keep, "keep", "int32", n), n, _stream_ptr(stream)))


def sfmp_kv_compact(cache: DeviceKvCache, tables: DeviceKvTables, status, workspace, stream=None) -> None:
    """Moves the live pages to the low end of the pool; status: int32 [1], their number."""
    rc = _launcher().kv_compact(cache, tables, status, workspace, stream)
    if rc is not None:
        return _check(rc)
    layout, codes, scales = _cache(cache)
    t = _tables(cache.layout, tables)
    at, size = _workspace(workspace)
    _check(load_library().sfmp_kv_compact(layout, codes, scales, C.byref(t), _tensor(status, "status", "int32", 1), at, size,
                                          _stream_ptr(stream)))


def sfmp_sample_workspace(rows: int, vocab: int) -> int:
    """Bytes that are enough for so many rows of so many tokens and for fewer."""
    n = C.c_int64(0)
    _check(load_library().sfmp_sample_workspace(_int(rows, "rows"), _int(vocab, "vocab"), C.byref(n)))
    return int(n.value)


def sfmp_sample(logits, temperature, top_k, top_p, min_p, uniform, tokens, logprobs, workspace, stream=None) -> None:
    """logits fp16, bf16 or fp32 [rows, vocab] (rows may lie apart); temperature, top_p, min_p fp32 [rows] or None, top_k int32
    [rows] or None, uniform fp32 [rows]; tokens int32 [rows], logprobs fp32 [rows] or None."""
    rc = _launcher().sample(logits, temperature, top_k, top_p, min_p, uniform, tokens, logprobs, workspace, stream)
    if rc is not None:
        return _check(rc)
    import torch
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise ValueError("logits has to be a tensor on the GPU")
    if logits.dtype not in _types() or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits has to be fp16, bf16 or fp32 [rows, vocab] with contiguous rows")
    n, vocab = _int(logits.shape[0], "rows"), _int(logits.shape[1], "vocab")
    at, size = _workspace(workspace)
    _check(load_library().sfmp_sample(logits.data_ptr() or None, _types()[logits.dtype], n, vocab, logits.stride(0) if n > 1 else vocab,
                                      _tensor(temperature, "temperature", "float32", n), _tensor(top_k, "top_k", "int32", n),
                                      _tensor(top_p, "top_p", "float32", n), _tensor(min_p, "min_p", "float32", n),
                                      _tensor(uniform, "uniform", "float32", n), _tensor(tokens, "tokens", "int32", n),
                                      _tensor(logprobs, "logprobs", "float32", n), at, size, _stream_ptr(stream)))
