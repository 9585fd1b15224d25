"""Calls of the paged cache that its documentation allows, beyond those of
test_gpu_paged.py."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_01190_amd import zsa
from tests.helpers import dev, f64
from tests.test_gpu_paged import TYPES, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,hd", [(8, 2, 64), (4, 4, 16), (4, 1, 128)])
@pytest.mark.parametrize("new", [[1], [3, 0, 40]])
def test_queries_rotated_in_place(dtype, H, kv, hd, new):
    b = Batch(dtype, H, kv, hd, 16, new, [n + 20 for n in new], seed=hd)
    T, kvd = sum(new), kv * hd
    g = torch.Generator(device=dev()).manual_seed(hd)
    rows = torch.randn((T, (H + 2 * kv) * hd), device=dev(), generator=g).to(TYPES[dtype])
    pos = torch.arange(T, dtype=torch.int32, device=dev()) * 31
    k, v = rows[:, H * hd:H * hd + kvd], rows[:, H * hd + kvd:]
    want = zsa.paged_append(b.kvc, k, v, b.seqs, b.len_dev, pos=pos, q=rows[:, :H * hd], n_heads=H)
    pool, fused, p = b.pool.clone(), rows.clone(), lambda t: ctypes.c_void_p(t.data_ptr())
    e, d = fused.element_size(), fused.stride(0)
    rc = zsa.lib().zsa_paged_append(
        ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), b.kvc._ref, ctypes.c_void_p(fused.data_ptr() + H * hd * e), d,
        ctypes.c_void_p(fused.data_ptr() + (H * hd + kvd) * e), d, p(fused), d, H, p(fused), d, p(pos), 10000.0, len(new),
        b.seqs.host_ptr(), p(b.seqs.dev), p(b.len_dev))
    assert rc == zsa.OK
    assert torch.equal(fused[:, :H * hd], want) and torch.equal(fused[:, H * hd:], rows[:, H * hd:])
    assert np.array_equal(f64(b.pool), f64(pool), equal_nan=True)
