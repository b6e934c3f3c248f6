"""Heads between a decoder layer's products: rotation, paged key/value caches in 4 and in 8 bits, attention over them, and of a prompt over its own keys and values.

Same names as the C ABI (``include/macko.h``, from "between the products of a decoder layer" on), argument checks and marshalling only.  For inference: results have no
gradient, also where an argument requires one.
"""
from __future__ import annotations

import contextlib
import ctypes
import math

from . import binding
from .binding import _check, _dev_ptr, _made, _need_torch, _stream_ptr, load_library

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float


class _CCache(ctypes.Structure):
    _fields_ = [("data", _vp), ("pages", _i64), ("page_size", _i32), ("kv_heads", _i32), ("head_dim", _i32)]


class _CRotation(ctypes.Structure):
    _fields_ = [("positions", _vp), ("table", _vp), ("table_rows", _i64), ("rot", _i32), ("interleaved", _i32), ("eps", _f32)]


class _CAppend(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("type", _i32), ("q", _vp), ("q_token", _i64), ("q_head", _i64),
                ("q_out", _vp), ("q_out_token", _i64), ("q_out_head", _i64), ("k", _vp), ("k_token", _i64), ("k_head", _i64),
                ("v", _vp), ("v_token", _i64), ("v_head", _i64), ("slots", _vp), ("q_weight", _vp), ("k_weight", _vp),
                ("rotation", _CRotation)]


class _CCache8(ctypes.Structure):
    _fields_ = [("codes", _vp), ("scales", _vp), ("pages", _i64), ("page_size", _i32), ("kv_heads", _i32), ("head_dim", _i32)]


class _CAppend8(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("type", _i32), ("batch", _i32), ("q", _vp), ("q_token", _i64), ("q_head", _i64),
                ("q_out", _vp), ("q_out_token", _i64), ("q_out_head", _i64), ("k", _vp), ("k_token", _i64), ("k_head", _i64),
                ("v", _vp), ("v_token", _i64), ("v_head", _i64), ("tables", _vp), ("table_stride", _i64), ("table_width", _i32),
                ("lengths", _vp), ("start", _vp), ("q_weight", _vp), ("k_weight", _vp), ("rotation", _CRotation)]


class _CAttention(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("type", _i32), ("batch", _i32), ("q", _vp), ("q_token", _i64), ("q_head", _i64),
                ("out", _vp), ("out_token", _i64), ("out_head", _i64), ("sums", _vp), ("tables", _vp), ("table_stride", _i64),
                ("table_width", _i32), ("lengths", _vp), ("start", _vp), ("most_queries", _i32), ("window", _i32), ("longest", _i64),
                ("scale", _f32)]


class _CPrompt(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("type", _i32), ("batch", _i32), ("q", _vp), ("q_token", _i64),
                ("q_head", _i64), ("k", _vp), ("k_token", _i64), ("k_head", _i64), ("v", _vp), ("v_token", _i64), ("v_head", _i64), ("out", _vp),
                ("out_token", _i64), ("out_head", _i64), ("sums", _vp), ("start", _vp), ("window", _i32), ("longest", _i64), ("scale", _f32)]


def _declare(lib) -> None:
    """Argument types of the calls of this file (load_library)."""
    cp = ctypes.POINTER(_CCache)
    lib.macko_kv_cache_bytes.argtypes = [cp]
    lib.macko_kv_cache_bytes.restype = _i64
    lib.macko_rope_table.argtypes = [_i64, _i64, ctypes.c_int] + [ctypes.c_double] * 6 + [_vp, _vp]
    lib.macko_rotate.argtypes = [_i64, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp, _i64, _i64, ctypes.POINTER(_CRotation), _vp, _vp, _i64, _i64, _vp]
    lib.macko_kv_append.argtypes = [cp, ctypes.POINTER(_CAppend), _vp]
    lib.macko_kv_read.argtypes = [cp, _i64, _vp, ctypes.c_int, _vp, _i64, _i64, _vp, _i64, _i64, _vp]
    lib.macko_kv_attention_workspace.argtypes = [cp, ctypes.POINTER(_CAttention)]
    lib.macko_kv_attention_workspace.restype = _i64
    lib.macko_kv_attention.argtypes = [cp, ctypes.POINTER(_CAttention), _vp, _i64, _vp]
    cp = ctypes.POINTER(_CCache8)
    lib.macko_kv8_cache_bytes.argtypes = [cp, ctypes.POINTER(_i64)]
    lib.macko_kv8_cache_bytes.restype = _i64
    lib.macko_kv8_append.argtypes = [cp, ctypes.POINTER(_CAppend8), _vp]
    lib.macko_kv8_read.argtypes = [cp, _i64, _vp, ctypes.c_int, _vp, _i64, _i64, _vp, _i64, _i64, _vp]
    lib.macko_kv8_attention_workspace.argtypes = [cp, ctypes.POINTER(_CAttention)]
    lib.macko_kv8_attention_workspace.restype = _i64
    lib.macko_kv8_attention.argtypes = [cp, ctypes.POINTER(_CAttention), _vp, _i64, _vp]
    lib.macko_prompt_attention.argtypes = [ctypes.POINTER(_CPrompt), _vp]


def _type_of(x) -> int:
    torch = _need_torch()
    if x.dtype == torch.float16:
        return 0
    if x.dtype == torch.bfloat16:
        return 1
    raise TypeError(f"16-bit tensors are float16 or bfloat16, not {x.dtype}")


def _heads(x, name, shape, like=None):
    """A [tokens, heads, head_dim] tensor on the GPU whose channels lie next to each other: its address and strides."""
    if x.dim() != 3 or tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(x.shape)}")
    if not x.is_cuda or (like is not None and (x.device != like.device or x.dtype != like.dtype)):
        raise ValueError(f"{name} must be on the GPU, on the device and of the type of the other tensors")
    if x.shape[2] > 1 and x.stride(2) != 1:
        raise ValueError(f"the channels of {name} must lie next to each other")
    return x.data_ptr(), x.stride(0), x.stride(1)


def _made_heads(x, name, shape, like):
    """_heads of a tensor that is written: no two elements share a place."""
    got = _heads(x, name, shape, like)
    token, head = got[1:]
    t, h, d = shape
    if t * h > 1 and not ((t <= 1 or token >= ((h - 1) * head + d if h > 1 else d)) and (h <= 1 or head >= d)
                          or (h <= 1 or head >= (t - 1) * token + d) and (t <= 1 or token >= d)):
        raise ValueError(f"rows of {name} overlap")
    return got


def _ints(x, name, shape, like):
    torch = _need_torch()
    if x.dtype != torch.int32:
        raise TypeError(f"{name} must be int32, not {x.dtype}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(x.shape)}")
    if x.device != like.device or (x.numel() > 1 and x.shape[-1] > 1 and x.stride(-1) != 1):
        raise ValueError(f"{name} must lie on {like.device}, its elements next to each other")
    return x.data_ptr()


def _whole(value, name, bits=32):
    """A whole number as the C interface takes it; ctypes would cut off what does not fit."""
    value = int(value)
    if not -2 ** (bits - 1) <= value < 2 ** (bits - 1):
        raise ValueError(f"{name} = {value} does not fit {bits} bits")
    return value


def _weight(w, name, like):
    if w is None:
        return None
    if w.dtype != like.dtype or w.device != like.device or tuple(w.shape) != (like.shape[2],) or (w.numel() > 1 and w.stride(0) != 1):
        raise ValueError(f"{name} must be [{like.shape[2]}] of the heads' type, on their device, elements next to each other")
    return w.data_ptr()


def _rotation(x, positions, table, interleaved, eps) -> _CRotation:
    torch = _need_torch()
    if table is None:
        return _CRotation(None, None, 0, 0, 0, eps)
    if table.dtype != torch.float32:
        raise TypeError("table must be float32 (rope_table)")
    if table.dim() != 3 or table.shape[1] != 2 or not table.is_contiguous() or table.device != x.device:
        raise ValueError("table must be a contiguous [positions, 2, rot / 2] tensor on the heads' device (rope_table)")
    if positions is None:
        raise ValueError("positions are needed with a table")
    return _CRotation(_ints(positions, "positions", (x.shape[0],), x), table.data_ptr(), table.shape[0], 2 * table.shape[2], int(bool(interleaved)), eps)


@contextlib.contextmanager
def _on(device, stream):
    """Allocations of the call belong to the stream that it runs on; its tensors must be on the current device, whose streams these are."""
    torch = _need_torch()
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    if stream is None:
        yield
        return
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        yield


def rope_table(length, rot, base=10000.0, first=0, factor=1.0, trained=0, low=1.0, high=32.0, amplitude=1.0, device="cuda", stream=None):
    """macko_rope_table: float32 [length, 2, rot / 2], cosines and sines of the positions first, first + 1, ...

    factor > 1 scales for contexts longer than the `trained` length: frequencies that turn more than `high` times within it stay, those
    below `low` are divided by the factor, others are blended; with trained = 0 all are divided."""
    torch = _need_torch()
    length, rot, first = _whole(length, "length", 64), _whole(rot, "rot"), _whole(first, "first", 64)
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    with _on(device, stream):
        table = torch.empty((max(length, 0), 2, max(rot, 0) // 2), dtype=torch.float32, device=device)
        _check(load_library().macko_rope_table(first, length, rot, base, factor, trained, low, high, amplitude,
                                               _dev_ptr(table), _stream_ptr(stream)), "macko_rope_table")
    return table


def rotate(x, positions, table, weight=None, eps=1e-6, interleaved=False, out=None, stream=None):
    """macko_rotate: the heads x [tokens, heads, head_dim] normalised (with a weight [head_dim]) and turned by their tokens' positions.

    positions: int32 [tokens], rows of the table (rope_table); table None: the norm alone.  `out` may be x."""
    if stream is None and binding._native is not None:
        y = binding._native.rotate(x, positions, table, weight, eps, interleaved, out)
        if y is not None:                    # None: something to be refused, a forked child or anything out of the ordinary
            return _made(y, "macko_rotate")
    torch = _need_torch()
    kind = _type_of(x)
    src = _heads(x, "x", x.shape)
    r = _rotation(x, positions, table, interleaved, eps)
    w = _weight(weight, "weight", x)
    with _on(x.device, stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dst = _made_heads(out, "out", x.shape, x)
        _check(load_library().macko_rotate(x.shape[0], x.shape[1], x.shape[2], kind, *src, ctypes.byref(r), w, *dst, _stream_ptr(stream)), "macko_rotate")
    return out


def attend_prompt(q, k, v, start=None, longest=None, scale=None, window=0, sums=False, out=None, stream=None):
    """macko_prompt_attention: causal attention of packed sequences, q [tokens, heads, head_dim] over k and v [tokens, kv_heads, head_dim] of the same type.

    start: int32 [sequences + 1], the rows that are each sequence's; None: all rows are one.  longest: a bound on the rows of one sequence, all rows unless
    given.  scale: head_dim ** -0.5 unless given.  window > 0: a row sees that many tokens at most, itself among them.  Returns out, or (out, sums) with sums = True: float32 [tokens, heads], the logarithm of each row's
    sum, to join results with those over a cached prefix."""
    if stream is None and binding._native is not None:
        y = binding._native.attend_prompt(q, k, v, start, longest, scale, window, sums, out)
        if y is not None:
            return _made(y, "macko_prompt_attention")
    torch = _need_torch()
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q must be [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim]")
    kind, shape = _type_of(q), tuple(q.shape)
    held = (shape[0], k.shape[1], shape[2])
    a = _CPrompt(*shape[:2], held[1], shape[2], kind)
    a.q, a.q_token, a.q_head = _heads(q, "q", shape)
    a.k, a.k_token, a.k_head = _heads(k, "k", held, q)
    a.v, a.v_token, a.v_head = _heads(v, "v", held, q)
    if start is not None:
        a.batch = start.shape[0] - 1 if start.dim() == 1 else -1
        a.start = _ints(start, "start", (a.batch + 1,), q)
    a.window = _whole(window, "window")
    a.longest = shape[0] if longest is None else _whole(longest, "longest", 64)
    a.scale = 1.0 / math.sqrt(shape[2]) if scale is None else scale
    with _on(q.device, stream):
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        a.out, a.out_token, a.out_head = _made_heads(out, "out", shape, q)
        total = torch.empty(shape[:2], dtype=torch.float32, device=q.device) if sums else None
        if sums:
            a.sums = total.data_ptr()
        _check(load_library().macko_prompt_attention(ctypes.byref(a), _stream_ptr(stream)), "macko_prompt_attention")
    return (out, total) if sums else out


def _read(cache, name, slots, dtype, k_out, v_out, stream):
    """The general way of a cache's read."""
    torch = _need_torch()
    shape = (slots.shape[0], cache.kv_heads, cache.head_dim)
    with _on(cache.data.device, stream):
        made = [torch.empty(shape, dtype=dtype, device=cache.data.device) if x is None else x for x in (k_out, v_out)]
        if made[0].dtype != dtype:
            raise ValueError("k_out and v_out must be of the type that is asked for")
        kind = _type_of(made[0])
        at = _ints(slots, "slots", (shape[0],), cache.data)
        to = [_made_heads(x, what, shape, made[0]) for x, what in zip(made, ("k_out", "v_out"))]
        cache._same(made[0])
        _check(getattr(load_library(), name)(cache._p, shape[0], at, kind, *to[0], *to[1], _stream_ptr(stream)), name)
    return made[0], made[1]


def _attend(cache, name, q, tables, lengths, start, most_queries, longest, scale, window, sums, out, stream):
    """The general way of a cache's attend."""
    torch = _need_torch()
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, head_dim]")
    kind, shape = _type_of(q), (q.shape[0], q.shape[1], cache.head_dim)
    batch = lengths.shape[0] if lengths.dim() == 1 else -1
    if tables.dim() != 2:
        raise ValueError("tables must be [batch, pages]")
    a = _CAttention(shape[0], shape[1], kind, batch)
    a.q, a.q_token, a.q_head = _heads(q, "q", shape, cache._same(q))
    a.lengths = _ints(lengths, "lengths", (batch,), q)
    a.tables = _ints(tables, "tables", (batch, tables.shape[1]), q)
    a.table_stride, a.table_width = tables.stride(0), tables.shape[1]
    if start is not None:
        a.start = _ints(start, "start", (batch + 1,), q)
    elif batch != shape[0]:
        raise ValueError("without start, q has one row a sequence")
    a.most_queries, a.window = _whole(most_queries, "most_queries"), _whole(window, "window")
    a.longest = a.table_width * cache.page_size if longest is None else _whole(longest, "longest", 64)
    a.scale = 1.0 / math.sqrt(cache.head_dim) if scale is None else scale
    lib = load_library()
    with _on(q.device, stream):
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        a.out, a.out_token, a.out_head = _made_heads(out, "out", shape, q)
        total = torch.empty(shape[:2], dtype=torch.float32, device=q.device) if sums else None
        if sums:
            a.sums = total.data_ptr()
        size = getattr(lib, name + "_workspace")(cache._p, ctypes.byref(a))
        if size < 0:
            _check(int(size), name)
        work = torch.empty(size, dtype=torch.uint8, device=q.device) if size else None
        _check(getattr(lib, name)(cache._p, ctypes.byref(a), work.data_ptr() if size else None, size, _stream_ptr(stream)), name)
    return (out, total) if sums else out


class KvCache:
    """A pool of pages of keys and values in 4 bits (macko_kv_cache_t).

    data: uint8 [pages, kv_heads, page_size * head_dim * 17 / 16] on the GPU, allocated unless given (a loaded or shared pool)."""

    def __init__(self, pages, page_size, kv_heads, head_dim, data=None, device="cuda"):
        torch = _need_torch()
        c = _CCache(None, _whole(pages, "pages", 64), _whole(page_size, "page_size"), _whole(kv_heads, "kv_heads"), _whole(head_dim, "head_dim"))
        size = load_library().macko_kv_cache_bytes(ctypes.byref(c))
        if size < 0:
            _check(int(size), "macko_kv_cache_bytes")
        shape = (c.pages, c.kv_heads, c.page_size * c.head_dim * 17 // 16)
        if data is None:
            data = torch.empty(shape, dtype=torch.uint8, device=device)
        if data.dtype != torch.uint8:
            raise TypeError("data must be uint8")
        if tuple(data.shape) != shape or not data.is_contiguous() or not data.is_cuda:
            raise ValueError(f"data must be a contiguous {list(shape)} tensor on the GPU")
        c.data = data.data_ptr()
        self.data, self._c, self._p = data, c, ctypes.byref(c)
        self._address, self._device = ctypes.addressof(c), data.device.index
        self.pages, self.page_size, self.kv_heads, self.head_dim = c.pages, c.page_size, c.kv_heads, c.head_dim

    def append(self, q, k, v, positions, slots, table=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None, stream=None):
        """macko_kv_append: q and k [tokens, heads, head_dim] normalised (weights) and turned (table, positions), k and v into the slots
        (int32 [tokens], below 0: none).  Returns q_out, which may be q; None without queries."""
        if stream is None and binding._native is not None:
            y = binding._native.kv_append(self._address, self._device, q, k, v, positions, slots, table, q_weight, k_weight, eps, interleaved, q_out)
            if y is not None:
                return None if y is True else _made(y, "macko_kv_append")
        torch = _need_torch()
        kind, tokens = _type_of(k), k.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        a = _CAppend(tokens, 0, kind)
        a.k, a.k_token, a.k_head = _heads(k, "k", shape, self._same(k))
        a.v, a.v_token, a.v_head = _heads(v, "v", shape, k)
        a.slots = _ints(slots, "slots", (tokens,), k)
        a.k_weight = _weight(k_weight, "k_weight", k)
        a.rotation = _rotation(k, positions, table, interleaved, eps)
        with _on(k.device, stream):
            if q is not None:
                shape = (tokens, q.shape[1] if q.dim() == 3 else 0, self.head_dim)
                a.heads = shape[1]
                a.q, a.q_token, a.q_head = _heads(q, "q", shape, k)
                a.q_weight = _weight(q_weight, "q_weight", q)
                if q_out is None:
                    q_out = torch.empty(shape, dtype=q.dtype, device=q.device)
                a.q_out, a.q_out_token, a.q_out_head = _made_heads(q_out, "q_out", shape, q)
            _check(load_library().macko_kv_append(self._p, ctypes.byref(a), _stream_ptr(stream)), "macko_kv_append")
        return q_out if q is not None else None

    def read(self, slots, dtype=None, k_out=None, v_out=None, stream=None):
        """macko_kv_read: keys and values [tokens, kv_heads, head_dim] of the slots (int32, below 0: zeros), in dtype (float16 by default)."""
        torch = binding._torch or _need_torch()
        if dtype is None:
            given = k_out if k_out is not None else v_out
            dtype = torch.float16 if given is None else given.dtype
        if stream is None and binding._native is not None and (dtype == torch.float16 or dtype == torch.bfloat16):
            pair = binding._native.kv_read(self._address, self._device, slots, dtype == torch.bfloat16, k_out, v_out)
            if pair is not None:
                return _made(pair, "macko_kv_read")
        return _read(self, "macko_kv_read", slots, dtype, k_out, v_out, stream)

    def attend(self, q, tables, lengths, start=None, most_queries=1, longest=None, scale=None, window=0, sums=False, out=None, stream=None):
        """macko_kv_attention of q [tokens, heads, head_dim] over the sequences' cached tokens.

        tables: int32 [batch, most pages], lengths: int32 [batch], counting the query tokens (append them first); start: int32 [batch + 1],
        the rows of q that are each sequence's, up to most_queries; None: one row a sequence.  longest: a bound on the lengths, of all
        that the tables can hold unless given.  scale: head_dim ** -0.5 unless given.  Returns out, or (out, sums) with sums = True:
        float32 [tokens, heads], the logarithm of each row's sum, to join results over parts of a context."""
        if stream is None and binding._native is not None:
            y = binding._native.kv_attend(self._address, self._device, q, tables, lengths, start, most_queries, longest, scale, window, sums, out)
            if y is not None:
                return _made(y, "macko_kv_attention")
        return _attend(self, "macko_kv_attention", q, tables, lengths, start, most_queries, longest, scale, window, sums, out, stream)

    def _same(self, x):
        if x.device != self.data.device:
            raise ValueError(f"tensors must lie on {self.data.device}, with the cache")
        return x


class KvCache8:
    """A pool of pages of keys and values in 8 bits (macko_kv8_cache_t), a power of two for each block of 16 tokens and head.

    data: uint8 [pages, kv_heads, page_size / 16, 2, 16 * head_dim], the codes of keys and values, and scales: uint8 [pages, kv_heads, page_size / 16, 2], both
    on the GPU, allocated unless given (a loaded or shared pool: both)."""

    def __init__(self, pages, page_size, kv_heads, head_dim, data=None, scales=None, device="cuda"):
        torch = _need_torch()
        c = _CCache8(None, None, _whole(pages, "pages", 64), _whole(page_size, "page_size"), _whole(kv_heads, "kv_heads"), _whole(head_dim, "head_dim"))
        size = load_library().macko_kv8_cache_bytes(ctypes.byref(c), None)
        if size < 0:
            _check(int(size), "macko_kv8_cache_bytes")
        if (data is None) != (scales is None):
            raise ValueError("data and scales are given together")
        blocks = (c.pages, c.kv_heads, c.page_size // 16, 2)
        made = []
        for x, name, shape in ((data, "data", blocks + (16 * c.head_dim,)), (scales, "scales", blocks)):
            if x is None:
                x = torch.empty(shape, dtype=torch.uint8, device=device)
            if x.dtype != torch.uint8:
                raise TypeError(f"{name} must be uint8")
            if tuple(x.shape) != shape or not x.is_contiguous() or not x.is_cuda:
                raise ValueError(f"{name} must be a contiguous {list(shape)} tensor on the GPU")
            made.append(x)
        if made[0].device != made[1].device:
            raise ValueError("data and scales must lie on one device")
        c.codes, c.scales = made[0].data_ptr(), made[1].data_ptr()
        self.data, self.scales, self._c, self._p = *made, c, ctypes.byref(c)
        self._address, self._device = ctypes.addressof(c), self.data.device.index
        self.pages, self.page_size, self.kv_heads, self.head_dim = c.pages, c.page_size, c.kv_heads, c.head_dim

    def append(self, q, k, v, positions, tables, lengths, start=None, table=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None, stream=None):
        """macko_kv8_append: q and k [tokens, heads, head_dim] normalised (weights) and turned (table, positions), k and v into the cache as the last tokens
        of the sequences that tables, lengths (with the new tokens) and start say, as in attend.  Returns q_out, which may be q; None without queries."""
        if stream is None and binding._native is not None:
            y = binding._native.kv8_append(self._address, self._device, q, k, v, positions, tables, lengths, start, table, q_weight, k_weight, eps, interleaved, q_out)
            if y is not None:
                return None if y is True else _made(y, "macko_kv8_append")
        torch = _need_torch()
        kind, tokens = _type_of(k), k.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        batch = lengths.shape[0] if lengths.dim() == 1 else -1
        if tables.dim() != 2:
            raise ValueError("tables must be [batch, pages]")
        a = _CAppend8(tokens, 0, kind, batch)
        a.k, a.k_token, a.k_head = _heads(k, "k", shape, self._same(k))
        a.v, a.v_token, a.v_head = _heads(v, "v", shape, k)
        a.lengths = _ints(lengths, "lengths", (batch,), k)
        a.tables = _ints(tables, "tables", (batch, tables.shape[1]), k)
        a.table_stride, a.table_width = tables.stride(0), tables.shape[1]
        if start is not None:
            a.start = _ints(start, "start", (batch + 1,), k)
        elif batch != tokens:
            raise ValueError("without start, there is one row a sequence")
        a.k_weight = _weight(k_weight, "k_weight", k)
        a.rotation = _rotation(k, positions, table, interleaved, eps)
        with _on(k.device, stream):
            if q is not None:
                shape = (tokens, q.shape[1] if q.dim() == 3 else 0, self.head_dim)
                a.heads = shape[1]
                a.q, a.q_token, a.q_head = _heads(q, "q", shape, k)
                a.q_weight = _weight(q_weight, "q_weight", q)
                if q_out is None:
                    q_out = torch.empty(shape, dtype=q.dtype, device=q.device)
                a.q_out, a.q_out_token, a.q_out_head = _made_heads(q_out, "q_out", shape, q)
            _check(load_library().macko_kv8_append(self._p, ctypes.byref(a), _stream_ptr(stream)), "macko_kv8_append")
        return q_out if q is not None else None

    def read(self, slots, dtype=None, k_out=None, v_out=None, stream=None):
        """macko_kv8_read: keys and values [tokens, kv_heads, head_dim] of the slots (int32, below 0: zeros), in dtype (float16 by default)."""
        torch = binding._torch or _need_torch()
        if dtype is None:
            given = k_out if k_out is not None else v_out
            dtype = torch.float16 if given is None else given.dtype
        if stream is None and binding._native is not None and (dtype == torch.float16 or dtype == torch.bfloat16):
            pair = binding._native.kv8_read(self._address, self._device, slots, dtype == torch.bfloat16, k_out, v_out)
            if pair is not None:
                return _made(pair, "macko_kv8_read")
        return _read(self, "macko_kv8_read", slots, dtype, k_out, v_out, stream)

    def attend(self, q, tables, lengths, start=None, most_queries=1, longest=None, scale=None, window=0, sums=False, out=None, stream=None):
        """macko_kv8_attention: KvCache.attend over this cache."""
        if stream is None and binding._native is not None:
            y = binding._native.kv8_attend(self._address, self._device, q, tables, lengths, start, most_queries, longest, scale, window, sums, out)
            if y is not None:
                return _made(y, "macko_kv8_attention")
        return _attend(self, "macko_kv8_attention", q, tables, lengths, start, most_queries, longest, scale, window, sums, out, stream)

    def _same(self, x):
        if x.device != self.data.device:
            raise ValueError(f"tensors must lie on {self.data.device}, with the cache")
        return x
