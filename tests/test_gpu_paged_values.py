"""Values that the paged attention sees or must not see, against its float64
oracle, which holds infinities and NaN where the definition puts them."""
import numpy as np
import pytest
import torch

from tests.helpers import f64
from tests.test_gpu_paged import Batch

pytestmark = pytest.mark.gpu


def put(b, seq, row, channel, value):
    """A value at a cached row of a sequence (seq None: of the prefix); the
    channels are those of all key/value heads."""
    ids = b.head if seq is None else b.table[seq]
    b.pool[int(ids[row // b.page]), row % b.page, b.kv * b.hd + channel] = value


def check_values(b, causal, **kw):
    out, lse = b.run(causal, **kw)
    ref, rlse, size, mag = b.oracle(causal, **kw)
    got = f64(out)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(kind(got), kind(ref)), (kind.__name__, int(kind(got).sum()), int(kind(ref).sum()))
    b.compare(out, lse, ref, rlse, size, mag)
    return ref


TYPES = [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 16), ("f32", 64)]
# one row a sequence, short and in parts; pieces in several tiles; prompts; with
# prefixes that go before the rows and that are a job of their own
CALLS = [([1, 1], [40, 9], 0), ([1, 1], [1, 33], 0), ([1], [9000], 0), ([1] * 48, [30] * 48, 0),
         ([40, 3], [190, 64], 0), ([300, 1], [450, 20], 0), ([1, 1], [40, 9], 37), ([40, 3], [60, 64], 37),
         ([300, 1], [320, 20], 100), ([1, 20], [40, 50], 9000)]


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("new,lens,prefix", CALLS)
@pytest.mark.parametrize("causal", [True, False])
def test_infinite_values(dtype, hd, new, lens, prefix, causal):
    b = Batch(dtype, 4, 2, hd, 16, new, lens, prefix, seed=len(new) + prefix + new[0])
    inf, n = float("inf"), lens[0]
    put(b, 0, 0, 3, inf)                  # seen by all rows of the sequence
    put(b, 0, n // 2, hd + 5, -inf)       # the other head's
    put(b, 0, n - 1, 4, -inf)             # the last row's own: hidden from the others under the mask
    put(b, 0, 0, 7, inf)                  # opposite ones in a channel: NaN where both are seen
    put(b, 0, n - 1, 7, -inf)
    if len(new) > 1:
        put(b, 1, lens[1] - 1, 1, inf)
        put(b, 1, 0, hd + 1, float("nan"))
    if prefix:
        put(b, None, 0, 9, inf)
        put(b, None, prefix - 1, hd + 9, -inf)
    ref = check_values(b, causal)
    assert np.isposinf(ref[0, 3]) and np.isneginf(ref[new[0] - 1, 4])
    assert n == 1 or np.isnan(ref[new[0] - 1, 7])
    if prefix:
        assert np.isposinf(ref[:, 9]).all() and np.isneginf(ref[:, 3 * hd + 9]).all()
