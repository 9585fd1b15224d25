"""Calls of the paged cache that are refused before any launch, and what its
offsets hold (no GPU)."""
import ctypes

import pytest

from paper_2509_01190_amd import zsa
from tests.test_paged_cpu import append, attend, cu


@pytest.mark.parametrize("offs", [(0, 2 ** 31 - 1, -2 ** 31), (0, -2 ** 31), (0, 1, -1), (0, 2 ** 31 - 1, -2)])
def test_offsets_that_fall_are_refused(offs):
    # also where the difference of the two has no place in 32 bits
    assert append(offs=offs) == zsa.ESHAPE
    assert attend(offs=offs) == zsa.ESHAPE
    h, c = cu(*offs), zsa.PagedKvStruct(page_stride=4096, n_pages=8, page_size=16, max_pages=4, n_kv_heads=2, head_dim=64,
                                        dtype=zsa.BF16)
    assert zsa.lib().zsa_paged_attention_workspace_size(ctypes.byref(c), 4, len(offs) - 1, zsa._hp32(h), 64, 40000) == 0
