"""Python binding of the paged key-value cache (``include/saf3r_paged.h``).

The functions take torch tensors on the GPU and run on the tensors' device, on
its current stream unless ``stream`` names another. As in ``binding``, every
computation runs in the HIP library; the outputs and workspaces that a caller
does not pass are allocated here.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import Saf3rError  # noqa: F401

E4M3 = 2  # cache type beside binding.F32 and binding.BF16

EXPORTS = (
    "saf3r_page_tables_workspace_bytes",
    "saf3r_page_tables",
    "saf3r_cache_append",
    "saf3r_paged_attention_workspace_bytes",
    "saf3r_paged_attention",
)

_INT_MAX = 2 ** 31 - 1


class PageStep(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("requests", "page_size", "max_pages", "pages", "tokens")]


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


_DECLARED = None


def _lib():
    global _DECLARED
    lib = binding.load()
    if _DECLARED is not lib:
        _DECLARED = _declare(lib)
    return lib


class _Call:
    """Device and stream of a call: the tensors' device is made current for it
    where it is not, and the stream is the device's current one by default."""

    def __init__(self, device, stream):
        import torch

        self.device, self.given = device, stream
        self.guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        import torch

        if self.guard is not None:
            self.guard.__enter__()
        return (torch.cuda.current_stream() if self.given is None else self.given).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _check_int(name, x, low):
    if not low <= x <= _INT_MAX:
        raise ValueError(f"{name} must be in [{low}, 2^31)")


def _check_words(name, t, shape, device):
    import torch

    if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.shape == shape and t.device == device):
        raise ValueError(f"{name} must be a contiguous int32 device tensor of shape {list(shape)} on {device}")


def _workspace(nbytes, device, stream):
    import torch

    t = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    binding._keep_until_done(stream, t)
    return t


def _given_workspace(t, device):
    if not (t.is_cuda and t.is_contiguous() and t.device == device):
        raise ValueError(f"the workspace must be a contiguous device tensor on {device}")
    return t.numel() * t.element_size()


def page_tables_workspace_bytes(requests, page_size, max_pages, pages, tokens) -> int:
    step = PageStep(requests, page_size, max_pages, pages, tokens)
    r = _lib().saf3r_page_tables_workspace_bytes(ctypes.byref(step))
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
    import torch

    _check_int("page_size", page_size, 1)
    _check_int("tokens", tokens, 0)
    dev = lengths.device
    R = lengths.shape[0]
    _check_words("lengths", lengths, (R,), dev)
    _check_words("new_tokens", new_tokens, (R,), dev)
    if free_pages.dim() != 1 or page_table.dim() != 2:
        raise ValueError("free_pages must be [pages] and page_table [requests, max_pages]")
    _check_words("free_pages", free_pages, free_pages.shape, dev)
    _check_words("free_count", free_count, (1,), dev)
    _check_words("page_table", page_table, (R, page_table.shape[1]), dev)
    outs = []
    for name, t, n in (("lengths_out", lengths_out, R), ("token_start", token_start, R + 1), ("slots", slots, tokens),
                       ("free_count_out", free_count_out, 1)):
        if t is None:
            t = torch.empty(n, dtype=torch.int32, device=dev)
        else:
            _check_words(name, t, (n,), dev)
        outs.append(t)
    step = PageStep(R, page_size, page_table.shape[1], free_pages.shape[0], tokens)
    if workspace is None:
        nbytes = 16 * R
        workspace = _workspace(nbytes, dev, stream)
    else:
        nbytes = _given_workspace(workspace, dev)
    with _Call(dev, stream) as st:
        binding._check(_lib().saf3r_page_tables(
            ctypes.byref(step), lengths.data_ptr(), new_tokens.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
            page_table.data_ptr(), outs[0].data_ptr(), outs[3].data_ptr(), outs[1].data_ptr(), outs[2].data_ptr(),
            workspace.data_ptr(), nbytes, st), "saf3r_page_tables")
    return tuple(outs)


def _layout(k_pages, v_pages, k_exp, v_exp):
    """The pages' layout, and the type of tokens and queries beside them."""
    import torch

    kind = torch.bfloat16
    if k_pages.dtype == torch.float8_e4m3fn:
        code = E4M3
    else:
        code = binding._torch_dtype_code(k_pages)
        kind = k_pages.dtype
    if not (k_pages.is_cuda and k_pages.dim() == 4 and k_pages.stride(3) == 1):
        raise ValueError("pages must be device tensors [pages, kv_heads, page_size, head_dim], head_dim contiguous")
    if v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype or v_pages.device != k_pages.device \
            or v_pages.stride() != k_pages.stride():
        raise ValueError("k_pages and v_pages must share shape, strides, dtype and device")
    n, H, ps, D = k_pages.shape
    if code == E4M3:
        for t in (k_exp, v_exp):
            if t is None or not (t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous() and t.shape == (n, H, ps)
                                 and t.device == k_pages.device):
                raise ValueError("an e4m3 cache needs k_exp and v_exp, contiguous uint8 [pages, kv_heads, page_size]")
    elif k_exp is not None or v_exp is not None:
        raise ValueError("k_exp and v_exp belong to an e4m3 cache")
    sp, sh, st, _ = k_pages.stride()
    return PageLayout(n, ps, H, D, code, 0, sp, sh, st), kind


def _ptr(t):
    return None if t is None else t.data_ptr()


def cache_append(k, v, slots, k_pages, v_pages, k_exp=None, v_exp=None, stream=None):
    """K and V of new tokens, ``[kv_heads, tokens, head_dim]`` with head_dim
    contiguous and the same strides, into their ``slots [tokens]`` of
    ``k_pages`` and ``v_pages`` (``[pages, kv_heads, page_size, head_dim]``).
    fp32 tokens into an fp32 cache, bf16 ones into a bf16 or ``float8_e4m3fn``
    one, the latter with the exponents ``k_exp`` and ``v_exp``. Slots outside the
    cache (-1) are skipped; the others must be distinct."""
    layout, kind = _layout(k_pages, v_pages, k_exp, v_exp)
    H, T, D = k.shape
    if not (k.is_cuda and k.dtype == kind and k.stride(2) == 1 and k.device == k_pages.device):
        raise ValueError(f"k and v must be {kind} tensors on {k_pages.device}, head_dim contiguous")
    if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or v.stride() != k.stride():
        raise ValueError("k and v must share shape, strides, dtype and device")
    if H != layout.kv_heads or D != layout.head_dim:
        raise ValueError("k and v must be [kv_heads, tokens, head_dim] with the cache's kv_heads and head_dim")
    if any(s == 0 and n > 1 for s, n in zip(k_pages.stride(), k_pages.shape)):
        raise ValueError("the pages' entries must not share memory")
    _check_words("slots", slots, (T,), k.device)
    rows = TokenLayout(T, 0, k.stride(0), k.stride(1))
    with _Call(k.device, stream) as st:
        binding._check(_lib().saf3r_cache_append(
            ctypes.byref(layout), ctypes.byref(rows), k.data_ptr(), v.data_ptr(), slots.data_ptr(), k_pages.data_ptr(),
            v_pages.data_ptr(), _ptr(k_exp), _ptr(v_exp), st), "saf3r_cache_append")


def paged_attention_workspace_bytes(q, k_pages, v_pages, page_table, k_exp=None, v_exp=None) -> int:
    layout, _ = _layout(k_pages, v_pages, k_exp, v_exp)
    step = Decode(q.shape[1], q.shape[0], page_table.shape[1], 0, 0, 1.0, 0, 0, 0, 0)
    r = _lib().saf3r_paged_attention_workspace_bytes(ctypes.byref(layout), ctypes.byref(step))
    binding._check(min(r, 0), "saf3r_paged_attention_workspace_bytes")
    return int(r)


def paged_attention(q, k_pages, v_pages, page_table, lengths, k_exp=None, v_exp=None, anchor=0, window=0, scale=None,
                    out=None, want_lse=False, workspace=None, stream=None):
    """Attention of one token per request over its cached tokens: ``(out
    [q_heads, requests, head_dim], lse [q_heads, requests] float32 or None)``.

    ``q [q_heads, requests, head_dim]`` (head_dim contiguous, bf16, or fp32 with an
    fp32 cache); query head h reads key-value head ``h // (q_heads //
    kv_heads)``. ``lengths [requests]`` tokens are attended, with ``window > 0``
    only the first ``anchor`` and the last ``window`` of them; a request without a
    token gives zeros and -inf. ``scale`` is ``head_dim ** -0.5`` by default."""
    import torch

    _check_int("anchor", anchor, 0)
    _check_int("window", window, 0)
    layout, kind = _layout(k_pages, v_pages, k_exp, v_exp)
    dev = k_pages.device
    Hq, R, D = q.shape
    if not (q.is_cuda and q.dtype == kind and q.stride(2) == 1 and q.device == dev and D == layout.head_dim):
        raise ValueError(f"q must be a {kind} tensor [q_heads, requests, {layout.head_dim}] on {dev}, head_dim contiguous")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [requests, max_pages]")
    _check_words("page_table", page_table, (R, page_table.shape[1]), dev)
    _check_words("lengths", lengths, (R,), dev)
    if out is None:
        out = torch.empty_like(q)
    elif not (out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.stride(2) == 1):
        raise ValueError("out must be like q, head_dim contiguous")
    if any(s == 0 and n > 1 for s, n in zip(out.stride(), out.shape)):
        raise ValueError("the rows of out must not share memory")
    lse = torch.empty((Hq, R), dtype=torch.float32, device=dev) if want_lse else None
    step = Decode(R, Hq, page_table.shape[1], anchor, window, D ** -0.5 if scale is None else scale, q.stride(0),
                  q.stride(1), out.stride(0), out.stride(1))
    lib = _lib()
    if workspace is None:
        nbytes = lib.saf3r_paged_attention_workspace_bytes(ctypes.byref(layout), ctypes.byref(step))
        binding._check(min(nbytes, 0), "saf3r_paged_attention")
        workspace = _workspace(nbytes, dev, stream)
    else:
        nbytes = _given_workspace(workspace, dev)
    with _Call(dev, stream) as st:
        binding._check(lib.saf3r_paged_attention(
            ctypes.byref(layout), ctypes.byref(step), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_exp),
            _ptr(v_exp), page_table.data_ptr(), lengths.data_ptr(), out.data_ptr(), _ptr(lse), workspace.data_ptr(),
            nbytes, st), "saf3r_paged_attention")
    return out, lse
