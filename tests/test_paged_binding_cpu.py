"""The paged cache's Python binding where no GPU is needed: what torch lacks, and arguments that the library cannot see."""
import os

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
