"""Python binding of what ``include/saf3r_prompt.h`` adds to the paged cache of
``paged``, whose conventions hold."""
from __future__ import annotations

import ctypes
import functools

from . import binding, paged
from .paged import Decode, PageLayout, TokenLayout

EXPORTS = (
    "saf3r_cache_read",
    "saf3r_paged_attention_scored",
    "saf3r_prompt_attention_workspace_bytes",
    "saf3r_prompt_attention",
)


class Prompt(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("requests", "tokens", "q_heads", "max_pages", "anchor", "window")] + \
               [(n, ctypes.c_float) for n in ("scale", "cap")] + \
               [(n, ctypes.c_int64) for n in ("q_head_stride", "q_token_stride", "out_head_stride", "out_token_stride")]



def _declare(lib):
    V, I64, I32, F, P = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.POINTER
    lib.saf3r_cache_read.argtypes = [P(PageLayout), P(TokenLayout)] + [V] * 8
    lib.saf3r_cache_read.restype = I32
    lib.saf3r_paged_attention_scored.argtypes = [P(PageLayout), P(Decode), F] + [V] * 11 + [I64, V]
    lib.saf3r_paged_attention_scored.restype = I32
    lib.saf3r_prompt_attention_workspace_bytes.argtypes = [P(PageLayout), P(Prompt)]
    lib.saf3r_prompt_attention_workspace_bytes.restype = I64
    lib.saf3r_prompt_attention.argtypes = [P(PageLayout), P(Prompt)] + [V] * 13 + [I64, V]
    lib.saf3r_prompt_attention.restype = I32
    return lib


_LIB = None


def _lib():
    global _LIB
    if _LIB is None or _LIB is not binding._LIB:
        _LIB = _declare(paged._lib())
    return _LIB


def _within(gap, dims, dim) -> bool:
    """Whether two rows of ``dim`` entries, each at a multiple of every stride of ``dims`` from its tensor's start, share
    one, the starts lying ``gap`` apart."""
    if not dims:
        return abs(gap) < dim
    (stride, n), rest = dims[0], dims[1:]
    reach = sum(s * (m - 1) for s, m in rest) + dim - 1
    least, most = max(1 - n, -((reach - gap) // stride)), min(n - 1, (gap + reach) // stride)
    return any(_within(gap - x * stride, rest, dim) for x in range(least, most + 1))


def _meet(a, b) -> bool:
    """Whether two tensors ``[heads, tokens, dim]`` of the same strides, dim contiguous, share an entry."""
    dims = sorted(((s, n) for s, n in zip(a.stride()[:2], a.shape[:2]) if n > 1), reverse=True)
    return a.numel() > 0 and _within((b.data_ptr() - a.data_ptr()) // a.element_size(), dims, a.shape[2])


def cache_read(slots, k_pages, v_pages, k_exp=None, v_exp=None, k=None, v=None, stream=None):
    """The tokens that ``slots [tokens]`` hold: ``(k, v)``, each ``[kv_heads, tokens,
    head_dim]``, fp32 of an fp32 cache and bf16 of the others, which hold nothing that
    bf16 does not. Zeros for slots outside the cache (-1); slots may repeat. ``k`` and
    ``v``, where they are passed, have head_dim contiguous, the same strides and no memory
    in common."""
    lib = _lib()
    layout, kind = paged._layout(k_pages, v_pages, k_exp, v_exp)
    dev = k_pages.device
    if slots.dim() != 1:
        raise ValueError("slots must be [tokens]")
    T = slots.shape[0]
    paged._check_sizes(T)
    paged._check_words("slots", slots, (T,), dev)
    shape = (layout.kv_heads, T, layout.head_dim)
    made = []
    if k is None and v is None:
        made.append(paged.torch.empty((2, *shape), dtype=kind, device=dev))
        k, v = made[0].unbind(0)
    elif k is None or v is None:
        raise ValueError("k and v are passed together")
    for t in (k, v):
        if t.shape != shape or t.dtype != kind or t.device != dev or t.stride(2) != 1:
            raise ValueError(f"k and v must be {kind} tensors {list(shape)} on {dev}, head_dim contiguous")
    if k.stride() != v.stride() and not paged._same_strides(k, v):
        raise ValueError("k and v must have the same strides")
    paged._check_apart("k and v", k)
    if not made and _meet(k, v):
        raise ValueError("k and v must not share memory")
    rows = TokenLayout(T, 0, k.stride(0), k.stride(1))
    if stream is not None:
        paged._allocated(stream, dev, made)
    paged._call(lib.saf3r_cache_read, dev, stream, ctypes.byref(layout), ctypes.byref(rows), slots.data_ptr(), k_pages.data_ptr(),
                v_pages.data_ptr(), paged._ptr(k_exp), paged._ptr(v_exp), k.data_ptr(), v.data_ptr())
    return k, v


@functools.lru_cache(maxsize=256)
def _prompt_workspace(code, kv_heads, page_size, head_dim, q_heads, requests, tokens, width) -> int:
    """The library's own answer, which these sizes alone decide."""
    layout = PageLayout(1, page_size, kv_heads, head_dim, code, 0, 0, 0, 0)
    return _lib().saf3r_prompt_attention_workspace_bytes(
        ctypes.byref(layout), ctypes.byref(Prompt(requests, tokens, q_heads, width, 0, 0, 1.0, 0.0, 0, 0, 0, 0)))


def prompt_attention_workspace_bytes(q, k_pages, v_pages, page_table, k_exp=None, v_exp=None) -> int:
    """Bytes of the workspace of ``prompt_attention``, 0 where the rows alone fill the GPU."""
    _lib()
    paged._check_sizes(q.shape[0] | q.shape[1] | page_table.shape[0] | page_table.shape[1])
    c, _ = paged._layout(k_pages, v_pages, k_exp, v_exp)
    r = _prompt_workspace(c.dtype, c.kv_heads, c.page_size, c.head_dim, q.shape[0], page_table.shape[0], q.shape[1],
                          page_table.shape[1])
    binding._check(min(r, 0), "saf3r_prompt_attention_workspace_bytes")
    return int(r)


def prompt_attention(q, k_pages, v_pages, page_table, lengths, token_start, k_exp=None, v_exp=None, prefix=None, anchor=0,
                     window=0, cap=0.0, slopes=None, scale=None, out=None, want_lse=False, workspace=None, stream=None):
    """Attention of several new tokens per request over its cached tokens, their own among
    them: ``(out [q_heads, tokens, head_dim], lse [q_heads, tokens] float32 or None)``.

    ``q [q_heads, tokens, head_dim]`` (head_dim contiguous, bf16, or fp32 with an fp32 cache)
    holds the new tokens of all requests one after another, those of r from
    ``token_start[r]`` to ``token_start[r + 1]`` (int32 ``[requests + 1]``, as ``page_tables``
    gives it); they are the last ones of its ``lengths[r]`` tokens. A token sees those up to
    itself, with ``window > 0`` only the first ``anchor`` and the last ``window`` of them,
    and, whatever its place, the first ``prefix[r]`` (int32 ``[requests]``) of its sequence:
    with ``prefix=lengths`` all of it. ``cap`` and ``slopes`` change scores as in
    ``paged_attention``, the distance being that of query and key in either direction. Rows
    from ``token_start[requests]`` on stay as they were; a token that sees nothing gives
    zeros and -inf."""
    lib = _lib()
    torch = paged.torch
    paged._check_int("anchor", anchor, 0)
    paged._check_int("window", window, 0)
    paged._check_cap(cap)
    dev, shape, strides, table = k_pages.device, q.shape, q.stride(), page_table.shape
    if len(shape) != 3 or len(table) != 2:
        raise ValueError("q must be [q_heads, tokens, head_dim] and page_table [requests, max_pages]")
    Hq, T, D = shape
    R, width = table
    paged._check_sizes(Hq | T | R | width)
    layout, kind = paged._layout(k_pages, v_pages, k_exp, v_exp)
    if q.dtype != kind or q.device != dev or strides[2] != 1 or D != layout.head_dim:
        raise ValueError(f"q must be a {kind} tensor [q_heads, tokens, {layout.head_dim}] on {dev}, head_dim contiguous")
    paged._check_words("page_table", page_table, (R, width), dev)
    paged._check_words("lengths", lengths, (R,), dev)
    paged._check_words("token_start", token_start, (R + 1,), dev)
    if prefix is not None:
        paged._check_words("prefix", prefix, (R,), dev)
    if slopes is not None:
        paged._check_slopes(slopes, Hq, dev)
    made = []
    if out is None:
        out = torch.empty_like(q)
        made.append(out)
    elif out.shape != shape or out.dtype != kind or out.device != dev:
        raise ValueError("out must be like q")
    to = out.stride()
    if to[2] != 1:
        raise ValueError("out's head_dim must be contiguous")
    paged._check_apart("the rows of out", out)
    lse = None
    if want_lse:
        lse = torch.empty(Hq, T, dtype=torch.float32, device=dev)
        made.append(lse)
    step = Prompt(R, T, Hq, width, anchor, window, D ** -0.5 if scale is None else scale, cap, strides[0], strides[1], to[0], to[1])
    if workspace is None:
        nbytes = _prompt_workspace(layout.dtype, layout.kv_heads, layout.page_size, D, Hq, R, T, width)
        binding._check(min(nbytes, 0), "saf3r_prompt_attention")
        if nbytes > 0:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            made.append(workspace)
    else:
        nbytes = paged._given_workspace(workspace, dev)
    if stream is not None:
        paged._allocated(stream, dev, made)
    paged._call(lib.saf3r_prompt_attention, dev, stream, ctypes.byref(layout), ctypes.byref(step), paged._ptr(slopes), q.data_ptr(),
                k_pages.data_ptr(), v_pages.data_ptr(), paged._ptr(k_exp), paged._ptr(v_exp), page_table.data_ptr(),
                lengths.data_ptr(), token_start.data_ptr(), paged._ptr(prefix), out.data_ptr(), paged._ptr(lse),
                paged._ptr(workspace), nbytes)
    return out, lse
