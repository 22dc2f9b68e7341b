"""Python binding of the paged key-value cache (``include/saf3r_paged.h``).

The functions take torch tensors on the GPU and run on the tensors' device, on
its current stream unless ``stream`` names another. As in ``binding``, every
computation runs in the HIP library; the outputs and workspaces that a caller
does not pass are allocated here.

With ``stream``, what the caller passes is the caller's to order: inputs still
being written on another stream, and tensors let go while ``stream`` reads them.
Memory that the call allocates is ordered here, which makes ``stream`` wait for
the device's current one; a call that allocates nothing does not wait.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding
from .binding import Saf3rError  # noqa: F401

E4M3, E2M1 = 2, 4  # cache types beside binding.F32 and binding.BF16

EXPORTS = (
    "saf3r_page_tables_workspace_bytes",
    "saf3r_page_tables",
    "saf3r_cache_append",
    "saf3r_paged_attention_workspace_bytes",
    "saf3r_paged_attention",
)

_INT_MAX = 2 ** 31 - 1


class PageStep(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("requests", "page_size", "max_pages", "pages", "tokens", "in_place")]


class PageLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("pages", "page_size", "kv_heads", "head_dim", "dtype", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("page_stride", "head_stride", "token_stride")]


class TokenLayout(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("reserved", ctypes.c_int32), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


class Decode(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("requests", "q_heads", "max_pages", "anchor", "window")] + \
               [("scale", ctypes.c_float)] + \
               [(n, ctypes.c_int64) for n in ("q_head_stride", "q_request_stride", "out_head_stride", "out_request_stride")]


def _declare(lib):
    V, I64, I32, P = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER
    lib.saf3r_page_tables_workspace_bytes.argtypes = [P(PageStep)]
    lib.saf3r_page_tables_workspace_bytes.restype = I64
    lib.saf3r_page_tables.argtypes = [P(PageStep)] + [V] * 10 + [I64, V]
    lib.saf3r_page_tables.restype = I32
    lib.saf3r_cache_append.argtypes = [P(PageLayout), P(TokenLayout)] + [V] * 8
    lib.saf3r_cache_append.restype = I32
    lib.saf3r_paged_attention_workspace_bytes.argtypes = [P(PageLayout), P(Decode)]
    lib.saf3r_paged_attention_workspace_bytes.restype = I64
    lib.saf3r_paged_attention.argtypes = [P(PageLayout), P(Decode)] + [V] * 10 + [I64, V]
    lib.saf3r_paged_attention.restype = I32
    return lib


torch = None  # with the library, by _lib(), which every call goes through first
_LIB = None
_TYPES = {}  # of a cache: its code, and the type of tokens, queries and outputs


def _lib():
    global torch, _LIB
    if _LIB is None or _LIB is not binding._LIB:
        import torch as module

        torch = module
        _TYPES.update({torch.float32: (binding.F32, torch.float32), torch.bfloat16: (binding.BF16, torch.bfloat16),
                       torch.float8_e4m3fn: (E4M3, torch.bfloat16)})
        if hasattr(torch, "float4_e2m1fn_x2"):
            _TYPES[torch.float4_e2m1fn_x2] = (E2M1, torch.bfloat16)
        _LIB = _declare(binding.load())
    return _LIB


def _call(function, device, stream, *args):
    """``function(*args, stream)`` with the tensors' device current, on the stream
    given or the device's current one; its status is checked."""
    if device.index != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return _call(function, device, stream, *args)
    # the handle alone: a Stream object takes 2.6 us
    status = function(*args, torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream)
    if status != 0:
        raise Saf3rError(status, function.__name__)


def _check_int(name, x, low):
    if not low <= x <= _INT_MAX:
        raise ValueError(f"{name} must be in [{low}, 2^31)")


def _check_cap(cap):
    """The library takes it as fp32, and 0 there as none."""
    if cap != 0 and ctypes.c_float(cap).value == 0:
        raise ValueError("cap must be 0 or at least fp32's least number")


def _check_sizes(together):
    """The library takes sizes as int32, and ctypes drops what does not fit. `together`:
    the bits of several."""
    if together > _INT_MAX:
        raise ValueError("sizes must be below 2^31")


def _check_words(name, t, shape, device):
    if t.dtype != torch.int32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {list(shape)} on {device}")


def _check_device(device):
    if device.type != "cuda":
        raise ValueError("expected device tensors")


def _allocated(stream, device, tensors):
    """Memory that the call allocated on the device's current stream, for use on
    `stream`: not before the current one is done with what lay there, and not
    handed out again before `stream` is."""
    current = torch.cuda.current_stream(device)
    if tensors and stream.cuda_stream != current.cuda_stream:
        binding._torch_stream(stream).wait_stream(current)
        binding._keep_until_done(stream, *tensors)


def _given_workspace(t, device):
    if not t.is_contiguous() or t.device != device:
        raise ValueError(f"the workspace must be a contiguous tensor on {device}")
    return t.numel() * t.element_size()


@functools.lru_cache(maxsize=256)
def _step_workspace(*sizes) -> int:
    """The library's own answer, which these sizes alone decide."""
    return _lib().saf3r_page_tables_workspace_bytes(ctypes.byref(PageStep(*sizes)))


def page_tables_workspace_bytes(requests, page_size, max_pages, pages, tokens, in_place=False) -> int:
    """Bytes of the workspace of ``page_tables``, 0 for the steps that are one launch."""
    _check_sizes(max(abs(x) for x in (requests, page_size, max_pages, pages, tokens)))
    r = _step_workspace(requests, page_size, max_pages, pages, tokens, int(in_place))
    binding._check(min(r, 0), "saf3r_page_tables_workspace_bytes")
    return int(r)


def page_tables(lengths, new_tokens, free_pages, free_count, page_table, page_size, tokens, lengths_out=None,
                token_start=None, slots=None, free_count_out=None, workspace=None, stream=None):
    """One step's bookkeeping: ``(lengths_out [R], token_start [R + 1], slots
    [tokens], free_count_out [1])``, all int32, with the entries of the pages
    taken written into ``page_table [R, max_pages]`` and those of ended sequences
    pushed into ``free_pages [pages]``.

    ``new_tokens[r]`` tokens follow the ``lengths[r]`` of request r, or fewer than
    0: it ends. Pages come from the top of the stack ``free_pages[:free_count]``,
    in the order of the requests. A request that does not fit keeps its length,
    and its slots are -1. ``lengths_out`` may be ``lengths`` and ``free_count_out``
    ``free_count``."""
    lib = _lib()
    _check_int("page_size", page_size, 1)
    _check_int("tokens", tokens, 0)
    if lengths.dim() != 1 or free_pages.dim() != 1 or page_table.dim() != 2:
        raise ValueError("lengths must be [requests], free_pages [pages] and page_table [requests, max_pages]")
    R, width, pages = lengths.shape[0], page_table.shape[1], free_pages.shape[0]
    _check_sizes(R | width | pages)
    dev = lengths.device
    _check_device(dev)
    _check_words("lengths", lengths, (R,), dev)
    _check_words("new_tokens", new_tokens, (R,), dev)
    _check_words("free_pages", free_pages, (pages,), dev)
    _check_words("free_count", free_count, (1,), dev)
    _check_words("page_table", page_table, (R, width), dev)
    outs, made = [lengths_out, token_start, slots, free_count_out], []
    sizes = (R, R + 1, tokens, 1)
    if lengths_out is None and token_start is None and slots is None and free_count_out is None:
        # one allocation and its parts: a microsecond less than four
        made.append(torch.empty(2 * R + tokens + 2, dtype=torch.int32, device=dev))
        outs = made[0].split(sizes)
    else:
        for i, name in enumerate(("lengths_out", "token_start", "slots", "free_count_out")):
            if outs[i] is None:
                outs[i] = torch.empty(sizes[i], dtype=torch.int32, device=dev)
                made.append(outs[i])
            else:
                _check_words(name, outs[i], (sizes[i],), dev)
    lengths_at, count_at = lengths.data_ptr(), free_count.data_ptr()
    lengths_to, count_to = outs[0].data_ptr(), outs[3].data_ptr()
    in_place = 1 if lengths_at == lengths_to or count_at == count_to else 0
    step = PageStep(R, page_size, width, pages, tokens, in_place)
    if workspace is None:
        nbytes = _step_workspace(R, page_size, width, pages, tokens, in_place)
        binding._check(min(nbytes, 0), "saf3r_page_tables")
        if nbytes > 0:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            made.append(workspace)
    else:
        nbytes = _given_workspace(workspace, dev)
    if stream is not None:
        _allocated(stream, dev, made)
    _call(lib.saf3r_page_tables, dev, stream, ctypes.byref(step), lengths_at, new_tokens.data_ptr(), free_pages.data_ptr(),
          count_at, page_table.data_ptr(), lengths_to, count_to, outs[1].data_ptr(), outs[2].data_ptr(), _ptr(workspace), nbytes)
    return tuple(outs)


def _same_strides(s, t):
    """Whether two tensors of one shape have the same strides but along single entries, where they say nothing."""
    return all(x == y or n == 1 for x, y, n in zip(s.stride(), t.stride(), s.shape))


def _check_exps(exps, shape, device, what):
    for t in exps:
        if t is None or t.dtype != torch.uint8 or not t.is_contiguous() or t.shape != shape or t.device != device:
            raise ValueError(what)


def _layout(k_pages, v_pages, k_exp, v_exp):
    """The pages' layout, and the type of tokens and queries beside them."""
    dtype, dev, shape, strides = k_pages.dtype, k_pages.device, k_pages.shape, k_pages.stride()
    if dtype not in _TYPES:
        raise ValueError(f"unsupported cache dtype {dtype}")
    code, kind = _TYPES[dtype]
    if len(shape) != 4 or strides[3] != 1:
        raise ValueError("pages must be [pages, kv_heads, page_size, head_dim], head_dim contiguous")
    n, H, ps, D = shape
    _check_sizes(n | H | ps | D)
    _check_device(dev)
    if v_pages.shape != shape or v_pages.dtype != dtype or v_pages.device != dev \
            or (v_pages.stride() != strides and not _same_strides(k_pages, v_pages)):
        raise ValueError("k_pages and v_pages must share shape, strides, dtype and device")
    if code == E4M3:
        _check_exps((k_exp, v_exp), (n, H, ps), dev, "an e4m3 cache needs k_exp and v_exp, contiguous uint8 [pages, kv_heads, page_size]")
    elif code == E2M1:
        D *= 2  # two values an element
        _check_exps((k_exp, v_exp), (n, H, ps, D // 32), dev,
                    "an e2m1 cache needs k_exp and v_exp, contiguous uint8 [pages, kv_heads, page_size, head_dim / 32]")
    elif k_exp is not None or v_exp is not None:
        raise ValueError("k_exp and v_exp belong to an e4m3 or e2m1 cache")
    return PageLayout(n, ps, H, D, code, 0, strides[0], strides[1], strides[2]), kind


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check_apart(name, t):
    """Entries that a call writes must not share memory."""
    if 0 in t.stride() and any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape)):
        raise ValueError(f"{name} must not share memory among their entries")


def cache_append(k, v, slots, k_pages, v_pages, k_exp=None, v_exp=None, stream=None):
    """K and V of new tokens, ``[kv_heads, tokens, head_dim]`` with head_dim
    contiguous and the same strides, into their ``slots [tokens]`` of
    ``k_pages`` and ``v_pages`` (``[pages, kv_heads, page_size, head_dim]``).
    fp32 tokens into an fp32 cache, bf16 ones into a bf16, ``float8_e4m3fn`` or
    ``float4_e2m1fn_x2`` one, the last two with the exponents ``k_exp`` and ``v_exp``:
    uint8, one for each token and head, and for each 32 values of 4 bits. A
    ``float4_e2m1fn_x2`` element holds two values, so such pages' last dimension is half
    of head_dim. Slots outside the cache (-1) are skipped; the others must be distinct."""
    lib = _lib()
    dev, shape, strides = k.device, k.shape, k.stride()
    if len(shape) != 3:
        raise ValueError("k and v must be [kv_heads, tokens, head_dim]")
    H, T, D = shape
    _check_sizes(T)
    layout, kind = _layout(k_pages, v_pages, k_exp, v_exp)
    if k.dtype != kind or dev != k_pages.device or strides[2] != 1:
        raise ValueError(f"k and v must be {kind} tensors [kv_heads, tokens, head_dim] on {k_pages.device}, head_dim contiguous")
    if v.shape != shape or v.dtype != kind or v.device != dev or (v.stride() != strides and not _same_strides(k, v)):
        raise ValueError("k and v must share shape, strides, dtype and device")
    if H != layout.kv_heads or D != layout.head_dim:
        raise ValueError("k and v must have the cache's kv_heads and head_dim")
    _check_apart("the pages", k_pages)
    _check_words("slots", slots, (T,), dev)
    rows = TokenLayout(T, 0, strides[0], strides[1])
    _call(lib.saf3r_cache_append, dev, stream, ctypes.byref(layout), ctypes.byref(rows), k.data_ptr(), v.data_ptr(),
          slots.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_exp), _ptr(v_exp))


@functools.lru_cache(maxsize=256)
def _attention_workspace(code, kv_heads, page_size, head_dim, q_heads, requests, width) -> int:
    """The library's own answer, which these sizes alone decide."""
    layout = PageLayout(1, page_size, kv_heads, head_dim, code, 0, 0, 0, 0)
    step = Decode(requests, q_heads, width, 0, 0, 1.0, 0, 0, 0, 0)
    return _lib().saf3r_paged_attention_workspace_bytes(ctypes.byref(layout), ctypes.byref(step))


def paged_attention_workspace_bytes(q, k_pages, v_pages, page_table, k_exp=None, v_exp=None) -> int:
    """Bytes of the workspace of ``paged_attention``, 0 where the table's rows are short."""
    _lib()
    _check_sizes(q.shape[0] | q.shape[1] | page_table.shape[1])
    c, _ = _layout(k_pages, v_pages, k_exp, v_exp)
    r = _attention_workspace(c.dtype, c.kv_heads, c.page_size, c.head_dim, q.shape[0], q.shape[1], page_table.shape[1])
    binding._check(min(r, 0), "saf3r_paged_attention_workspace_bytes")
    return int(r)


def _check_slopes(t, heads, device):
    if t.dtype != torch.float32 or t.device != device or t.shape != (heads,) or not t.is_contiguous():
        raise ValueError(f"slopes must be a contiguous float32 tensor of shape [{heads}] on {device}")


def paged_attention(q, k_pages, v_pages, page_table, lengths, k_exp=None, v_exp=None, anchor=0, window=0, scale=None,
                    out=None, want_lse=False, workspace=None, stream=None, cap=0.0, slopes=None):
    """Attention of one token per request over its cached tokens: ``(out
    [q_heads, requests, head_dim], lse [q_heads, requests] float32 or None)``.

    ``q [q_heads, requests, head_dim]`` (head_dim contiguous, bf16, or fp32 with an
    fp32 cache); query head h reads key-value head ``h // (q_heads //
    kv_heads)``. ``lengths [requests]`` tokens are attended, with ``window > 0``
    only the first ``anchor`` and the last ``window`` of them; a request without a
    token gives zeros and -inf. ``scale`` is ``head_dim ** -0.5`` by default. With ``cap >
    0`` a score z becomes ``cap * tanh(z / cap)``; ``slopes [q_heads]`` float32 times the
    distance of the query, the request's last token, and the key are then taken off it."""
    lib = _lib()
    _check_int("anchor", anchor, 0)
    _check_int("window", window, 0)
    _check_cap(cap)
    dev, shape, strides, table = k_pages.device, q.shape, q.stride(), page_table.shape
    if len(shape) != 3 or len(table) != 2:
        raise ValueError("q must be [q_heads, requests, head_dim] and page_table [requests, max_pages]")
    Hq, R, D = shape
    width = table[1]
    _check_sizes(Hq | R | width)
    layout, kind = _layout(k_pages, v_pages, k_exp, v_exp)
    if q.dtype != kind or q.device != dev or strides[2] != 1 or D != layout.head_dim:
        raise ValueError(f"q must be a {kind} tensor [q_heads, requests, {layout.head_dim}] on {dev}, head_dim contiguous")
    _check_words("page_table", page_table, (R, width), dev)
    _check_words("lengths", lengths, (R,), dev)
    if slopes is not None:
        _check_slopes(slopes, Hq, dev)
    made = []
    if out is None:
        out = torch.empty_like(q)
        made.append(out)
    elif out.shape != shape or out.dtype != kind or out.device != dev:
        raise ValueError("out must be like q")
    to = out.stride()
    if to[2] != 1:
        raise ValueError("out's head_dim must be contiguous")
    _check_apart("the rows of out", out)
    lse = None
    if want_lse:
        lse = torch.empty(Hq, R, dtype=torch.float32, device=dev)
        made.append(lse)
    step = Decode(R, Hq, width, anchor, window, D ** -0.5 if scale is None else scale, strides[0], strides[1], to[0], to[1])
    if workspace is None:
        nbytes = _attention_workspace(layout.dtype, layout.kv_heads, layout.page_size, D, Hq, R, width)
        binding._check(min(nbytes, 0), "saf3r_paged_attention")
        if nbytes > 0:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            made.append(workspace)
    else:
        nbytes = _given_workspace(workspace, dev)
    if stream is not None:
        _allocated(stream, dev, made)
    call, scores = lib.saf3r_paged_attention, ()
    if cap != 0 or slopes is not None:
        from . import prompt

        call, scores = prompt._lib().saf3r_paged_attention_scored, (cap, _ptr(slopes))
    _call(call, dev, stream, ctypes.byref(layout), ctypes.byref(step), *scores, q.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), _ptr(k_exp), _ptr(v_exp), page_table.data_ptr(), lengths.data_ptr(), out.data_ptr(), _ptr(lse),
          _ptr(workspace), nbytes)
    return out, lse
