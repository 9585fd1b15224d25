"""Values that the paged attention sees or must not see, against its float64
oracle, which holds infinities and NaN where the definition puts them."""
import numpy as np
import pytest
import torch

from tests.helpers import f64
from tests.test_gpu_paged import U32, Batch

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
MANY = [([300, 1], [450, 20], 0), ([300, 1], [320, 20], 100), ([1, 20], [40, 50], 9000), ([200], [3000], 0)]
FEW = [c for c in CALLS if len(c[0]) < 9 and max(c[0]) < 300 and c[2] < 9000]  # the few-row kernels'


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


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("new,lens,prefix", FEW)
def test_whole_channels_of_infinities(dtype, hd, new, lens, prefix):
    # Many infinities in one sum, whose probabilities' second numbers have any
    # sign; beside them channels of 2^110, finite in all sums.
    b = Batch(dtype, 4, 2, hd, 16, new, lens, prefix, seed=hd + new[0])
    values = b.pool[..., 2 * hd:]
    values[..., 2], values[..., hd + 6] = float("inf"), -float("inf")
    values[..., 3], values[..., 4] = 2.0 ** 110, -2.0 ** 110
    ref = check_values(b, True)
    assert np.isposinf(ref[0, 2]) and np.isneginf(ref[0, 3 * hd + 6]) and np.isfinite(ref[0, 3])


def margins(b, causal):
    """Of every row and head: how far its largest score is above the next."""
    pool, q, G, kvd = f64(b.pool), f64(b.q).reshape(b.cu[-1], b.H, b.hd), b.H // b.kv, b.kv * b.hd
    out = np.full((b.H, b.cu[-1]), np.inf)
    for s, n in enumerate(b.lens):
        own = b.cu[s + 1] - b.cu[s]
        rows = [pool[ids[r // b.page], r % b.page, :kvd] for ids, m in ((b.head, b.prefix), (b.table[s], n)) for r in range(m)]
        k = np.array(rows).reshape(-1, b.kv, b.hd)
        for r in range(own):
            seen = b.prefix + (n - own + r + 1 if causal else n)
            for h in range(b.H):
                x = np.sort(k[:seen, h // G] @ q[b.cu[s] + r, h])[::-1] * b.hd ** -0.5
                if len(x) > 1:
                    out[h, b.cu[s] + r] = x[0] - x[1]
    return out


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("new,lens,prefix", FEW + [([1, 1], [40, 50], 9000)] + MANY)
@pytest.mark.parametrize("power", [14, 22, 50])
@pytest.mark.parametrize("negative", [False, True])
def test_far_scores(dtype, hd, new, lens, prefix, power, negative):
    # Scores of 2^28, 2^44 and 2^100 times the ordinary ones, whose roundings are
    # many units of an exponential: every row takes the value of its first key.
    b = Batch(dtype, 4, 2, hd, 16, new, lens, prefix, seed=power + new[0])
    b.q.mul_(2.0 ** power)
    keys = b.pool[..., :2 * hd]
    if negative:  # all of them below zero
        b.q.abs_()
        keys.abs_().neg_()
    keys.mul_(2.0 ** power)
    out, lse = b.run(True)
    ref, rlse, _, mag = b.oracle(True)
    err = (hd + 8) * U32 * (mag + 1)  # of a score: hd products and their sum, its scale
    # the next key's probability is below 2^-140 whatever the roundings do: none is left of it in 32 bits
    clear = margins(b, True) > 4 * err + 100
    assert clear.mean() > 0.5, clear.mean()
    rows = clear.T[:, :, None].repeat(hd, 2).reshape(ref.shape)
    assert np.array_equal(f64(out)[rows], ref[rows])
    assert (np.abs(f64(lse) - rlse)[clear] <= (err + 4 * U32 * np.abs(rlse))[clear]).all()


def rounded(x):
    return torch.from_numpy(np.asarray(x)).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("length,far", [(2, False), (40, False), (40, True), (700, True), (9000, True)])
@pytest.mark.parametrize("prefix", [0, 20])
def test_probabilities_of_few_rows_have_16_bits(dtype, hd, length, far, prefix):
    # Two keys count, with probabilities in the ratio 1 to exp(-x), in one tile or
    # far apart; their values are 1 and the ratio in 8 bits, and of two signs, so
    # that the sum is what the ratio has beyond 8 bits.
    B, n = 24, 1
    b = Batch(dtype, 4, 2, hd, 16, [n] * B, [length] * B, prefix, seed=length)
    x = (1 + np.arange(B)) / 16.0
    last = length - 1 if far else 1
    one, ratio = torch.ones(()), torch.from_numpy(rounded(np.exp(-x)))
    for ids in (b.table.reshape(-1), b.head):
        b.pool[torch.from_numpy(ids.astype(np.int64)).to(b.pool.device)] = 0.0
    keys, values = b.pool[..., :2 * hd].view(*b.pool.shape[:2], 2, hd), b.pool[..., 2 * hd:]
    keys[..., 0] = -30000.0        # the others': nothing is left of them in 32 bits
    for s in range(B):
        for row, score, value in ((0, 0.0, -ratio[s]), (last, -x[s], one)):
            page, slot = int(b.table[s, row // 16]), row % 16
            keys[page, slot, :, 0] = score
            values[page, slot] = value.item()
    b.q.zero_()
    b.q.view(B, 4, hd)[..., 0] = hd ** 0.5 if hd in (16, 64) else 8.0
    scale = None if hd in (16, 64) else 0.125
    out, lse = b.run(True, scale=scale)
    ref, rlse, size, _ = b.oracle(True, scale=scale)
    # A score has one product, exact, and the scale's rounding and its own; an
    # exponential, the sums of two terms, a quotient: 12 roundings of 2^-24 (a
    # prefix's keys add zeros). Two bf16 numbers: half a step of a half step.
    p = 0.0 if dtype == "f32" or hd == 16 else 2.0 ** -16
    tol = ((2 * x.max() + 12) * U32 + p) * size + torch.finfo(b.dtype).eps / 2 * np.abs(ref)
    assert (np.abs(f64(out) - ref) <= tol).all(), (np.abs(f64(out) - ref) / tol).max()
    assert (np.abs(f64(lse) - rlse) <= 16 * U32).all()
    # with probabilities of 8 bits most rows would be beyond that
    assert (np.abs(ref) > 4 * tol).mean() > 0.7
