"""The paged cache's Python binding where no GPU is needed: what torch lacks, and arguments that the library cannot see."""
import os
import random

import pytest
import torch


@pytest.fixture(scope="module")
def paged():
    from paper_2607_03612_amd import binding, build, paged

    if not os.path.exists(binding.LIB_PATH):
        build.build()
    paged._lib()
    return paged


@pytest.fixture
def afresh(paged):
    """The binding as at its first call, before and after a test."""
    paged._LIB = None
    paged._TYPES.clear()
    yield paged
    paged._LIB = None
    paged._TYPES.clear()


def test_torch_without_a_4_bit_type(afresh, monkeypatch):
    """The other cache types do not need it."""
    monkeypatch.delattr(torch, "float4_e2m1fn_x2")
    afresh._lib()
    assert set(afresh._TYPES) == {torch.float32, torch.bfloat16, torch.float8_e4m3fn}
    pages = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        afresh.cache_append(pages[:, 0, :5].contiguous(), pages[:, 0, :5].contiguous(), torch.zeros(5, dtype=torch.int32), pages, pages)


def test_shared_entries_are_found(paged):
    """Against the sets of entries, for tensors in one buffer: heads first, tokens first, side by side, one inside another."""
    from paper_2607_03612_amd import prompt

    rng = random.Random(2)
    buffer = torch.zeros(4096, dtype=torch.bfloat16)
    met = apart = beside = 0
    for _ in range(3000):
        H, T, D = rng.randint(1, 5), rng.randint(1, 6), rng.choice([1, 4, 8])
        strides = [rng.choice([D, 2 * D, D * T, D * T + 8, 3 * D, D + 1]), rng.choice([D, 2 * D, D * H, D * H + 8, D + 4])]
        at = [rng.randint(0, 400) for _ in range(2)]
        if rng.random() < 0.5:
            at[1] = at[0] + rng.choice([0, 1, D - 1, D, strides[0], strides[1], D * T, D * H])
        a, b = (torch.as_strided(buffer, (H, T, D), (*strides, 1), x) for x in at)
        entries = [{x + h * strides[0] + t * strides[1] + d for h in range(H) for t in range(T) for d in range(D)} for x in at]
        want = bool(entries[0] & entries[1])
        assert prompt._meet(a, b) == prompt._meet(b, a) == want, (H, T, D, strides, at)
        met, apart = met + want, apart + (not want)
        beside += not want and max(map(min, entries)) < min(map(max, entries))
    assert met > 500 and apart > 500 and beside > 100
    assert not prompt._meet(buffer[:0].view(1, 0, 8), buffer[:0].view(1, 0, 8))
    kv = buffer.view(4, 2, 8, 64)
    assert not prompt._meet(kv[:, 0], kv[:, 1]) and prompt._meet(kv[:, 0], kv[:, 0])
    dims = [(1 << 33, 256), (128, 1 << 26)]  # the largest sizes, 2^42 entries in all
    assert prompt._within((5 << 33) + 128 * 77 + 127, dims, 128) and not prompt._within((256 << 33) + 5, dims, 128)
    assert not prompt._within((1 << 33) - 128, dims[:1] + [(256, 1 << 24)], 128)


@pytest.mark.parametrize("cap", [1e-46, -1e-46, 1e-300, 5e-324])
def test_a_cap_below_fp32(paged, cap):
    """The library takes it as fp32, where it would be 0: no cap."""
    from paper_2607_03612_amd import prompt

    pages, q = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    words = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="cap"):
        paged.paged_attention(q, pages, pages, words(1, 2), words(1), cap=cap)
    with pytest.raises(ValueError, match="cap"):
        prompt.prompt_attention(q, pages, pages, words(1, 2), words(1), words(2), cap=cap)
