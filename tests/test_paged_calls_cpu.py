"""Calls of the paged cache that are refused before any launch, and what its
offsets hold (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_01190_amd import zsa
from tests.test_paged_cpu import PTR, append, attend, cu


@pytest.mark.parametrize("offs", [(0, 2 ** 31 - 1, -2 ** 31), (0, -2 ** 31), (0, 1, -1), (0, 2 ** 31 - 1, -2)])
def test_offsets_that_fall_are_refused(offs):
    # also where the difference of the two has no place in 32 bits
    assert append(offs=offs) == zsa.ESHAPE
    assert attend(offs=offs) == zsa.ESHAPE
    h, c = cu(*offs), zsa.PagedKvStruct(page_stride=4096, n_pages=8, page_size=16, max_pages=4, n_kv_heads=2, head_dim=64,
                                        dtype=zsa.BF16)
    assert zsa.lib().zsa_paged_attention_workspace_size(ctypes.byref(c), 4, len(offs) - 1, zsa._hp32(h), 64, 40000) == 0


def test_wrapped_offsets_are_the_calls_own():
    # the rows that a call checks its tensors for and those that the library is
    # given are the same, whatever the caller does with the array afterwards
    host = np.array([0, 1, 3], dtype=np.int32)
    seqs = zsa.Seqs.wrap(host, torch.tensor([0, 1, 3], dtype=torch.int32))
    pointer = seqs.host_ptr()
    host[1:] = 100, 3000
    assert seqs.total == 3 and seqs.lengths == [1, 2]
    assert [pointer[i] for i in range(3)] == [0, 1, 3] == [int(c) for c in seqs.host]


@pytest.mark.parametrize("cu", [[], [[0, 1], [1, 2]]])
def test_wrapped_offsets_that_are_none(cu):
    dev = torch.tensor(cu, dtype=torch.int32).reshape(-1)
    with pytest.raises(ValueError):
        zsa.Seqs.wrap(cu, dev)


def test_queries_rotated_in_place_keep_their_stride():
    # with another one a row would be written before it is read
    q = dict(q=PTR[2], qs=512, H=4, qo=PTR[2], pos=PTR[4])
    assert append(qos=256, **q) == zsa.ESHAPE
    assert append(qos=768, **q) == zsa.ESHAPE
