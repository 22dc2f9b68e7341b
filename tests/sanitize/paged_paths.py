"""Calls of the paged cache's C ABI that pass validation, and its integer
arithmetic, for the sanitizer build only (its launches are stand-ins). Run by
tests/test_paged_cpu.py in a process with AddressSanitizer preloaded."""
import ctypes
import random

import pytest

from paper_2607_03612_amd import binding
from paper_2607_03612_amd import paged as G

OK = ctypes.c_void_p(0x10000)  # never dereferenced by the stand-ins
OTHER = ctypes.c_void_p(0x20000)


def lib():
    return G._declare(binding.load())


@pytest.mark.parametrize("size", list(range(16, 1025, 16)))
def test_page_division_is_exact(size):
    div = lib().saf3r_stub_div_page
    rng = random.Random(size)
    top = (1 << 29) + 1023
    xs = [0, 1, size - 1, size, size + 1, top, top - 1] + [rng.randint(0, top) for _ in range(300)]
    for _ in range(300):  # around multiples, and the largest of them
        m = rng.randint(1, top // size) * size
        xs += [m - 1, m, min(m + size - 1, top)]
    m = top // size * size
    for x in xs + [m - 1, m]:
        assert div(size, x) == x // size, (size, x)


@pytest.mark.parametrize("size", list(range(16, 1025, 16)))
def test_page_division_is_exact_for_every_slot(size):
    """Slots go up to 2^31 - 1. A reciprocal that is rounded up gives a page too many first at a page's last
    place, and the later the page the sooner."""
    div = lib().saf3r_stub_div_page
    rng = random.Random(-size)
    top = 2 ** 31 - 1
    most = (top + 1) // size  # whole pages
    firsts = [1, 2, most - 1, most] + [rng.randint(1, most) for _ in range(300)] + [most - i for i in range(300) if most > i]
    xs = [top] + [m * size + d for m in firsts for d in (-1, 0)] + [rng.randint(0, top) for _ in range(300)]
    for x in xs:
        if x <= top:
            assert div(size, x) == x // size, (size, x)


@pytest.mark.parametrize("requests,tokens,in_place,launches", [
    (1, 0, 0, 1), (1024, 1 << 30, 0, 1), (1024, 4096, 1, 1), (1024, 4097, 1, 2), (1025, 1, 0, 2), (65536, 1 << 30, 1, 2)])
def test_page_tables(requests, tokens, in_place, launches):
    step = G.PageStep(requests, 1024, 1 << 19, 2097151, tokens, in_place)
    need = lib().saf3r_page_tables_workspace_bytes(ctypes.byref(step))
    assert need == (0 if launches == 1 else 12 * requests)
    call = lib().saf3r_page_tables
    outs = (OK, OK) if in_place else (OTHER, OTHER)
    args = [OK, OK, OK, OK, OK, *outs, OK, OK]
    assert call(ctypes.byref(step), *args, OK, need, None) == 0
    assert lib().saf3r_stub_paged_launches() == launches
    if need == 0:
        assert call(ctypes.byref(step), *args, None, 0, None) == 0
    # in place only where the step says so
    if not in_place:
        assert call(ctypes.byref(step), OK, OK, OK, OK, OK, OK, OTHER, OK, OK, OK, need, None) == -1
        assert call(ctypes.byref(step), OK, OK, OK, OK, OK, OTHER, OK, OK, OK, OK, need, None) == -1


@pytest.mark.parametrize("dtype,size,dim,page,width,launches", [
    (0, 4, 64, 64, 12, 1), (0, 4, 64, 64, 13, 2), (1, 2, 128, 16, 48, 1), (1, 2, 128, 16, 49, 2), (2, 1, 128, 1024, 1, 1),
    (2, 1, 128, 1024, 2, 2), (2, 1, 64, 128, 16, 1), (2, 1, 64, 128, 17, 2), (1, 2, 64, 1024, 1 << 19, 2)])
@pytest.mark.parametrize("heads", [(1, 1), (256, 1), (256, 256), (96, 2)])
def test_attention(dtype, size, dim, page, width, launches, heads):
    hq, hk = heads
    # whole rows only while a launch's threads can be counted: 65536 requests with up to 128 rows each
    requests = 65536 // max(1, hk // 128) // max(1, hq // hk // 16)
    layout = G.PageLayout(2097151 if page == 1024 else 9, page, hk, dim, dtype, 0, hk * page * dim, page * dim, dim)
    step = G.Decode(requests, hq, width, 2 ** 31 - 1, 2 ** 31 - 1, 0.125, 65536 * dim, dim, dim, hq * dim)
    need = lib().saf3r_paged_attention_workspace_bytes(ctypes.byref(layout), ctypes.byref(step))
    assert need == (0 if launches == 1 else 512 * 16 + 1024 * min(hq // hk, 16) * (8 + 4 * dim))
    exps = (OK, OK) if dtype == 2 else (None, None)
    call = lib().saf3r_paged_attention
    assert call(ctypes.byref(layout), ctypes.byref(step), OK, OK, OK, *exps, OK, OK, OK, OK, OK, need, None) == 0
    assert lib().saf3r_stub_paged_launches() == launches
    assert call(ctypes.byref(layout), ctypes.byref(step), OK, OK, OK, *exps, OK, OK, OK, None, None if need == 0 else OK, need,
                None) == 0
    if heads == (256, 256):
        step.requests += 1
        assert lib().saf3r_paged_attention_workspace_bytes(ctypes.byref(layout), ctypes.byref(step)) > 0
        step.requests = 65536
        assert call(ctypes.byref(layout), ctypes.byref(step), OK, OK, OK, *exps, OK, OK, OK, OK, OK, 1 << 30, None) == 0
        assert lib().saf3r_stub_paged_launches() == 2
    rows = G.TokenLayout(1 << 26, 0, dim, 0)
    assert lib().saf3r_cache_append(ctypes.byref(layout), ctypes.byref(rows), OK, OK, OK, OK, OK, *exps, None) == 0


def test_far_apart_is_no_reason_to_refuse():
    """Any stride that two entries in a device's memory can have; what would pass 63 bits is none."""
    def run(pages, page_stride, tokens, token_stride):
        layout = G.PageLayout(pages, 16, 2, 64, binding.BF16, 0, page_stride // 2, 1024, 64)
        rows = G.TokenLayout(tokens, 0, 64, token_stride // 2)
        return lib().saf3r_cache_append(ctypes.byref(layout), ctypes.byref(rows), OK, OK, OK, OK, OK, None, None, None)

    for pages, tokens in ((2, 2), (1 << 24, 1 << 24)):
        assert run(pages, 1 << 36, tokens, 4096) == 0 and run(pages, 4096, tokens, 1 << 36) == 0, pages
    assert run(2, 1 << 44, 2, 1 << 44) == 0 and run(2, (1 << 44) + 16, 2, 16) == -1 and run(2, 16, 2, (1 << 44) + 16) == -1
    assert run(1 << 26, 1 << 34, 1 << 26, 1 << 34) == 0
    assert run(1 << 26, (1 << 34) + 16, 2, 16) == -1 and run(2, 16, 1 << 26, (1 << 34) + 16) == -1
