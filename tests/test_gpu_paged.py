"""The paged key/value cache on the GPU against its float64 oracle: appending
rows, the attention over them, and that attention behind a common prefix."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2509_01190_amd import zsa
from tests.helpers import dev, f64

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Batch:
    """A pool whose pages are dealt to the sequences in a shuffled order; what
    no sequence holds (other pages, the slots behind its last row) is NaN."""

    def __init__(self, dtype, H, kv, hd, page, new, lens, prefix=0, seed=0, layers=1, sharp=1.5):
        g = np.random.default_rng(seed)
        self.H, self.kv, self.hd, self.page, self.lens, self.prefix = H, kv, hd, page, lens, prefix
        self.dtype = TYPES[dtype]
        self.seqs = zsa.Seqs(new, dev())
        self.cu = [int(c) for c in self.seqs.host]
        kvd, need = kv * hd, [-(-max(n, 0) // page) for n in lens]
        first = -(-prefix // page)
        pages = first + sum(need) + 2
        order = g.permutation(pages).astype(np.int32)
        most = max(need + [1])
        self.table = g.choice(order, (len(lens), most)).astype(np.int32)
        self.head = order[:first].copy()
        pool = np.full((pages, page, 2 * kvd), np.nan, np.float32)
        at = first

        def fill(ids, n):
            for r in range(n):
                pool[ids[r // page], r % page] = g.standard_normal(2 * kvd)
                pool[ids[r // page], r % page, :kvd] *= sharp

        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            fill(self.table[b], max(lens[b], 0))
            at += n
        fill(self.head, prefix)
        # one layer of a pool for several: its pages lie apart
        store = torch.full((pages, layers, page, 2 * kvd), float("nan"), dtype=self.dtype, device=dev())
        store[:, layers - 1] = torch.from_numpy(pool).to(self.dtype).to(dev())
        self.pool = store[:, layers - 1]
        # the table's rows are wider than what is used
        wide = torch.full((len(lens), most + 3), -7, dtype=torch.int32, device=dev())
        wide[:, :most] = torch.from_numpy(self.table).to(dev())
        self.table_dev = wide[:, :most]
        self.kvc = zsa.PagedKV(self.pool, self.table_dev, kv)
        self.len_dev = torch.tensor(lens, dtype=torch.int32, device=dev())
        self.head_dev = torch.from_numpy(self.head).to(dev())
        q = g.standard_normal((self.cu[-1], H * hd)).astype(np.float32)
        # a slice of wider rows, as in a fused projection
        rows = torch.zeros((self.cu[-1], H * hd + 2 * kvd), dtype=self.dtype, device=dev())
        rows[:, :H * hd] = torch.from_numpy(q).to(self.dtype).to(dev())
        self.q = rows[:, :H * hd]

    def run(self, causal, **kw):
        out, lse = zsa.prefix_attention(self.q, self.kvc, self.H, self.seqs, self.len_dev, self.head_dev,
                                        self.prefix, causal=causal, want_lse=True, **kw)
        torch.cuda.synchronize()
        return out, lse

    def oracle(self, causal, **kw):
        return P.attention(f64(self.q), f64(self.pool), self.table, self.cu, self.lens, self.H, self.kv, causal,
                           prefix_pages=self.head, prefix_len=self.prefix, **kw)

    def check(self, causal, **kw):
        out, lse = self.run(causal, **kw)
        ref, rlse, size, mag = self.oracle(causal, **kw)
        self.compare(out, lse, ref, rlse, size, mag)
        return out, lse

    def compare(self, out, lse, ref, rlse, size, mag):
        got, glse = f64(out), f64(lse)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(np.isneginf(glse), np.isneginf(rlse))
        # A score is a sum of hd products (hd roundings at most, each of the
        # sum of magnitudes), times the scale, minus a maximum, through an
        # exponential (2 units more each): off by `ds`, so a probability by a
        # factor 1 + ds and a sum over the keys, added one by one, by one rounding each.
        keys = max([max(n, 0) for n in self.lens] + [0]) + self.prefix
        ds = (self.hd + 8) * U32 * (mag + 4.0)
        sums = (keys + 8) * U32
        # probabilities may be rounded to the storage type before they meet v
        p = half_step(self.dtype)
        with np.errstate(invalid="ignore"):
            per = (2 * ds + 2 * sums + p).T[:, :, None].repeat(self.hd, 2).reshape(ref.shape)
            tol = per * size + half_step(self.dtype) * np.abs(ref) * (1 + p)
            bad = np.abs(got - ref) > tol + 1e-30
            assert not bad.any(), (np.abs(got - ref) / (tol + 1e-30))[bad].max()
            fin = np.isfinite(rlse)
            assert (np.abs(glse - rlse)[fin] <= (ds + sums + 2 * U32 * np.abs(rlse))[fin]).all(), \
                np.abs(glse - rlse)[fin].max()


HEADS = [(12, 12, 64), (8, 2, 64), (4, 4, 128), (8, 1, 128), (6, 2, 128), (4, 4, 32), (6, 2, 16), (40, 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,hd", HEADS)
def test_one_new_row(dtype, H, kv, hd):
    # lengths of none, one, around tiles and pages
    lens = [1, 0, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 300, 2]
    Batch(dtype, H, kv, hd, 16, [1] * len(lens), lens, seed=H + hd).check(True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_pages(dtype, page, causal):
    lens = [700, 33, 257, 1]
    Batch(dtype, 4, 2, 64, page, [3, 1, 70, 1], lens, seed=page).check(causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,hd", [(4, 4, 64), (8, 2, 128), (3, 1, 128), (4, 4, 32), (2, 1, 16)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_new_rows(dtype, H, kv, hd, causal):
    # pieces whose earlier rows are cached, whole prompts, empty sequences
    # and, with fewer cached rows than new ones, rows that see no key
    new = [130, 1, 33, 0, 64, 5, 40, 9]
    lens = [300, 77, 33, 12, 64, 5, 25, 0]
    Batch(dtype, H, kv, hd, 32, new, lens, seed=3 * H + hd).check(causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,hd,prefix", [(12, 12, 64, 501), (8, 2, 128, 64), (8, 2, 128, 1), (4, 4, 64, 1300),
                                            (4, 2, 32, 77), (6, 2, 16, 130)])
@pytest.mark.parametrize("new", [[1] * 7, [1, 20, 0, 97, 3, 33, 5]])
def test_common_prefix(dtype, H, kv, hd, prefix, new):
    lens = [n + c for n, c in zip(new, [0, 40, 7, 0, 200, -9, 16])]
    Batch(dtype, H, kv, hd, 32, new, [max(n, 0) for n in lens], prefix, seed=prefix).check(True)


@pytest.mark.parametrize("dtype,H,kv,hd,prefix,batch,n", [
    ("bf16", 16, 8, 128, 521, 17, 1),    # one row a sequence, 34 packed rows a head over the prefix
    ("bf16", 8, 8, 128, 521, 17, 1),     # 17: few enough for the few-row kernel there too
    ("bf16", 8, 8, 128, 521, 17, 3),
    ("bf16", 16, 16, 64, 1100, 18, 40),
    ("f32", 8, 8, 128, 530, 9, 1),
    ("f32", 16, 8, 128, 530, 9, 3),
    ("f32", 16, 16, 64, 530, 9, 20),
])
def test_long_prefix_of_many_sequences(dtype, H, kv, hd, prefix, batch, n):
    # more than 32 MB if every sequence read it: rows of its own in the call's parts
    new = [n if b % 3 else 1 for b in range(batch)]
    lens = [m + (11 * b) % 70 for b, m in enumerate(new)]
    lens[4] = 0
    Batch(dtype, H, kv, hd, 16, new, lens, prefix, seed=prefix + n).check(True)


@pytest.mark.parametrize("dtype,H,kv,hd,prefix,batch,n", [
    ("bf16", 16, 16, 128, 1500, 17, 1),
    ("bf16", 32, 16, 128, 1500, 20, 1),   # 40 packed rows a head: three workgroups of the few-row kernel
    ("bf16", 32, 16, 128, 1500, 20, 9),   # up to 360: the many-row kernel's
    ("bf16", 16, 16, 64, 1500, 40, 3),    # up to 120 rows, in 16s
    ("f32", 16, 16, 64, 1500, 24, 1),     # in 16s as the sequences' own rows
    ("f32", 32, 16, 64, 1500, 24, 20),    # in 32s as those
    ("f32", 16, 2, 64, 6000, 60, 2),      # in 32s for the prefix's length
])
def test_longer_prefix_of_many_sequences(dtype, H, kv, hd, prefix, batch, n):
    # more than 160 MB if every sequence read it
    new = [n if b % 3 else 1 for b in range(batch)]
    lens = [m + (11 * b) % 70 for b, m in enumerate(new)]
    lens[4] = 0
    b = Batch(dtype, H, kv, hd, 64, new, lens, prefix, seed=prefix + n)
    assert batch * prefix * 2 * kv * hd * (2 if dtype == "bf16" else 4) > 160 << 20
    b.check(True)


@pytest.mark.parametrize("dtype,H,kv,hd,batch,most", [
    ("bf16", 8, 8, 64, 24, 2900), ("bf16", 16, 8, 128, 23, 2050), ("bf16", 8, 8, 32, 50, 1700), ("bf16", 4, 4, 64, 3, 1530),
    ("f32", 8, 8, 64, 24, 2100), ("f32", 8, 8, 128, 50, 1100), ("bf16", 8, 8, 16, 24, 1300),
])
@pytest.mark.parametrize("prefix", [0, 37])
def test_long_rows_in_one_split(dtype, H, kv, hd, batch, most, prefix):
    lens = [most - (61 * b) % 1000 if b % 2 else 1 + 13 * b for b in range(batch)]
    lens[0], lens[1] = most, 0
    Batch(dtype, H, kv, hd, 64, [1] * batch, lens, prefix, seed=most).check(True, max_kv_len=most)


@pytest.mark.parametrize("dtype,H,kv,hd,batch,n,most", [
    ("bf16", 8, 2, 128, 4, 30, 1500),     # up to 120 packed rows in 16s
    ("bf16", 8, 2, 128, 4, 30, 1600),     # the many-row kernel, a few of whose rows are there, in several splits
    ("bf16", 6, 2, 64, 5, 10, 2900),      # two workgroups of 16 each
    ("bf16", 6, 2, 64, 5, 10, 3200),
    ("bf16", 4, 1, 32, 3, 200, 2500),     # four tiles of 256, the last in part
    ("bf16", 4, 4, 128, 1, 300, 5000),
    ("f32", 6, 2, 64, 3, 30, 1600),
])
def test_pieces_of_long_sequences(dtype, H, kv, hd, batch, n, most):
    new = [n - 2 * b for b in range(batch)]
    lens = [most - 211 * b for b in range(batch)]
    Batch(dtype, H, kv, hd, 32, new, lens, seed=most + n).check(True, max_kv_len=most)


@pytest.mark.parametrize("dtype,H,kv,hd", [("bf16", 16, 16, 64), ("bf16", 16, 16, 128), ("bf16", 16, 16, 32),
                                           ("bf16", 16, 16, 16), ("f32", 16, 16, 64), ("f32", 16, 16, 128)])
@pytest.mark.parametrize("most,prefix", [(33, 0), (64, 0), (200, 0), (20, 13), (60, 100)])
def test_many_short_sequences(dtype, H, kv, hd, most, prefix):
    # more than two workgroups a CU
    new = [1 + (b % 5 == 0) for b in range(45)]
    lens = [(most * (b % 9)) // 8 for b in range(45)]
    Batch(dtype, H, kv, hd, 16, new, lens, prefix, seed=most + hd).check(True, max_kv_len=most)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_equals_the_same_rows_repeated(dtype):
    # the prefix cached once, against every sequence holding it as its own rows
    b = Batch(dtype, 8, 2, 64, 16, [1, 4, 1], [20, 30, 1], 64, seed=5)
    out, lse = b.check(True)
    table = np.concatenate([np.tile(b.head, (3, 1)), b.table], axis=1)
    kvc = zsa.PagedKV(b.pool, torch.from_numpy(table).to(dev()), 2)
    lens = b.len_dev + 64
    out2, lse2 = zsa.paged_attention(b.q, kvc, 8, b.seqs, lens, want_lse=True)
    b.compare(out2, lse2, *b.oracle(True))


@pytest.mark.parametrize("H,kv,hd", [(4, 2, 64), (4, 1, 128), (2, 2, 32)])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("prefix", [1, 31, 33, 64, 1100])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_behind_a_prefix(H, kv, hd, page, prefix, causal):
    # rows for the many-row kernel, which takes the prefix's with them; some that see no row of their own
    new = [300, 1, 0, 270, 150, 2]
    lens = [300, 40, 0, 333, 100, 0]
    Batch("bf16", H, kv, hd, page, new, lens, prefix, seed=prefix + hd).check(causal)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("n,prefix", [(1, 0), (40, 0), (300, 0), (1, 37), (40, 37), (300, 37)])
def test_values_that_are_not_finite(dtype, hd, n, prefix):
    # The last new row holds an infinity and the one before it a NaN: the
    # rows before them do not see them
    b = Batch(dtype, 4, 2, hd, 16, [n, 1], [n + 150, 9], prefix, seed=n)
    size, m = b.page, n + 150
    for row, value in ((m - 1, float("inf")), (m - 2, float("nan"))):
        if row >= 150:
            b.pool[int(b.table[0, row // size]), row % size, 2 * hd:] = value
    out, lse = b.run(True)
    ref, rlse, mags, mag = b.oracle(True)
    keep = np.isfinite(ref)
    assert np.array_equal(np.isfinite(f64(out)), keep)
    rows = keep.all(axis=1)
    assert rows.sum() >= n - 1
    got, p = f64(out), half_step(b.dtype)
    err = np.abs(got[rows] - ref[rows])
    ds = (2 * (hd + 8) * U32 * (mag.max() + 4) + 2 * (m + prefix + 8) * U32 + p)
    assert (err <= ds * mags[rows] + p * (1 + p) * np.abs(ref[rows]) + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_outside_the_pool_read_as_zeros(dtype):
    b = Batch(dtype, 4, 2, 64, 16, [1, 20], [90, 100], 40, seed=9)
    b.table[0, 2], b.table[1, 1], b.head[1] = -1, b.pool.shape[0], 2 ** 31 - 1
    b.table_dev.copy_(torch.from_numpy(b.table))
    b.head_dev.copy_(torch.from_numpy(b.head))
    b.check(True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layers_of_one_pool(dtype):
    b = Batch(dtype, 4, 2, 128, 16, [1, 30], [90, 100], 20, seed=2, layers=3)
    assert b.pool.stride(0) == 3 * 16 * 512
    b.check(True)


def test_longest_sequence_is_bounded_on_the_host():
    # rows from max_kv_len on are not read
    b = Batch("bf16", 4, 4, 64, 16, [1, 2], [90, 100], seed=4)
    b.check(False, max_kv_len=50)
    b.check(True, max_kv_len=100)


@pytest.mark.parametrize("dtype,H,kv,hd", [("bf16", 4, 2, 64), ("bf16", 8, 8, 128), ("f32", 4, 4, 64), ("f32", 4, 2, 128),
                                           ("bf16", 4, 4, 32), ("bf16", 2, 1, 16)])
@pytest.mark.parametrize("new,prefix", [([1, 1, 1], 0), ([1, 60, 1], 0), ([40, 90, 33], 0), ([1, 50, 1], 70)])
def test_wide_tables(dtype, H, kv, hd, new, prefix):
    # the bound is the table's width, far beyond the rows: many splits, most of
    # them empty, and rows read past the caches
    b = Batch(dtype, H, kv, hd, 32, new, [700, 260, 1], prefix, seed=hd + sum(new))
    wide = torch.randint(0, b.pool.shape[0], (3, 9000), dtype=torch.int32, device=dev())
    wide[:, :b.table.shape[1]] = b.table_dev
    b.kvc, b.table = zsa.PagedKV(b.pool, wide, kv), wide.cpu().numpy()
    b.check(True)
    b.check(False, max_kv_len=100000)


@pytest.mark.parametrize("dtype,H,kv,hd", [("bf16", 4, 1, 64), ("bf16", 2, 2, 128), ("f32", 2, 1, 32)])
def test_many_sequences(dtype, H, kv, hd):
    g = np.random.default_rng(hd)
    lens = [int(n) for n in g.integers(0, 40, 300)]
    new = [1 if b % 7 else int(g.integers(0, 30)) for b in range(300)]
    Batch(dtype, H, kv, hd, 16, new, lens, 37, seed=hd).check(True)


def test_lengths_beyond_the_bound_under_the_mask():
    b = Batch("bf16", 4, 2, 64, 16, [3, 40], [90, 100], seed=4)
    b.check(True, max_kv_len=70)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scores", [60.0, 3000.0])
def test_large_scores(dtype, scores):
    # keys whose scores tower over the others', early and late
    b = Batch(dtype, 4, 2, 64, 16, [1, 70], [700, 300], seed=8)
    for s, row in ((0, 3), (0, 650), (1, 5), (1, 200)):
        page = int(b.table[s, row // 16])
        q = f64(b.q)[b.cu[s], :64]
        b.pool[page, row % 16, :64] = torch.from_numpy(q / (q @ q) * 8 * scores).to(b.dtype).to(dev())
    b.check(True)


def test_pool_beyond_32_bit_offsets():
    # pages past 4 GiB of the pool
    kv, hd, page = 8, 128, 128
    pages = (5 << 30) // (page * 2 * kv * hd * 2)
    pool = torch.empty((pages, page, 2 * kv * hd), dtype=torch.bfloat16, device=dev())
    table = torch.tensor([[pages - 1, 1], [pages - 2, pages - 3]], dtype=torch.int32, device=dev())
    for p in table.flatten().tolist():
        pool[p].normal_(generator=torch.Generator(device=dev()).manual_seed(p))
    g = torch.Generator(device=dev()).manual_seed(1)
    n = [1, 150]
    seqs = zsa.Seqs(n, dev())
    lens = torch.tensor([200, 250], dtype=torch.int32, device=dev())
    T = sum(n)
    k = torch.randn(T, kv * hd, device=dev(), generator=g, dtype=torch.bfloat16)
    v = torch.randn(T, kv * hd, device=dev(), generator=g, dtype=torch.bfloat16)
    q = torch.randn(T, 4 * kv * hd, device=dev(), generator=g, dtype=torch.bfloat16)
    far = zsa.PagedKV(pool, table, kv)
    # the same cache in a small pool
    small = pool[table.flatten().long()].clone()
    near = zsa.PagedKV(small, torch.arange(4, dtype=torch.int32, device=dev()).view(2, 2), kv)
    for c in (far, near):
        assert zsa.paged_append(c, k, v, seqs, lens) is None
    assert torch.equal(pool[table.flatten().long()], small)
    a = zsa.paged_attention(q, far, 4 * kv, seqs, lens, want_lse=True)
    b = zsa.paged_attention(q, near, 4 * kv, seqs, lens, want_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,hd", [(12, 12, 64), (8, 2, 128), (4, 4, 32), (6, 2, 16)])
@pytest.mark.parametrize("new,lens", [([1] * 5, [1, 40, 16, 17, 300]),
                                      ([70, 0, 1, 33, 9], [100, 5, 1, 33, 4])])
@pytest.mark.parametrize("mode", ["plain", "keys", "queries"])
def test_append(dtype, H, kv, hd, new, lens, mode):
    b = Batch(dtype, H, kv, hd, 16, new, lens, seed=len(new) + hd)
    g = np.random.default_rng(1)
    T, kvd, theta = sum(new), kv * hd, 500000.0
    qkv = torch.from_numpy(g.standard_normal((T, (H + 2 * kv) * hd)).astype(np.float32)).to(b.dtype).to(dev())
    q, k, v = qkv[:, :H * hd], qkv[:, H * hd:H * hd + kvd], qkv[:, H * hd + kvd:]
    pos = g.integers(0, 200000, T).astype(np.int32)
    before = b.pool.clone()
    got = zsa.paged_append(b.kvc, k, v, b.seqs, b.len_dev,
                           pos=None if mode == "plain" else torch.from_numpy(pos).to(dev()), rope_theta=theta,
                           q=q if mode == "queries" else None, n_heads=H)
    torch.cuda.synchronize()
    rk = f64(k) if mode == "plain" else P.rotate(f64(k), pos, theta, hd)
    ref = P.append(f64(before), b.table, b.cu, lens, rk, f64(v))
    out = f64(b.pool)
    # untouched rows and the values: bit for bit
    touched = P.append(np.zeros(before.shape), b.table, b.cu, lens, np.ones((T, kvd)), np.ones((T, kvd))) != 0
    assert np.array_equal(np.where(touched, 0, np.nan_to_num(out)), np.where(touched, 0, np.nan_to_num(f64(before))))
    assert np.array_equal(out[..., kvd:][touched[..., kvd:]], ref[..., kvd:][touched[..., kvd:]])
    # a rotation: the cosine and sine off by 2 units of fp32 and the angle's
    # own rounding to fp32 (at most pi 2^-24), two products and a sum, and the storage's half step
    def close(x, y, size):
        tol = 12 * U32 * size + half_step(b.dtype) * np.abs(y) * (1 + 1e-3)
        assert (np.abs(x - y) <= tol).all(), (np.abs(x - y) / tol).max()

    def pair(x):
        z = np.abs(x).reshape(T, -1, 2, hd // 2)
        return np.broadcast_to(z.sum(axis=2, keepdims=True), z.shape).reshape(T, -1)

    where = touched[..., :kvd]
    if mode == "plain":
        assert got is None and np.array_equal(out[..., :kvd][where], ref[..., :kvd][where])
        return
    sizes = P.append(np.zeros(before.shape), b.table, b.cu, lens, pair(f64(k)), f64(v))[..., :kvd]
    close(out[..., :kvd][where], ref[..., :kvd][where], sizes[where])
    if mode == "keys":
        assert got is None
    else:
        close(f64(got), P.rotate(f64(q), pos, theta, hd), pair(f64(q)))


def test_append_rotates_as_the_projection_does():
    # the cache holds what the projection's rotary epilogue would have given
    b = Batch("bf16", 4, 2, 64, 16, [5, 9], [50, 9], seed=1)
    g = torch.Generator(device=dev()).manual_seed(0)
    x = torch.randn(14, 256, device=dev(), generator=g).to(torch.bfloat16)
    w = (torch.randn(512, 256, device=dev(), generator=g) / 16).to(torch.bfloat16)
    pos = torch.arange(14, dtype=torch.int32, device=dev()) * 37
    fused = f64(zsa.linear(x, w, epilogue=zsa.EPI_ROPE, pos=pos, head_dim=64, rope_cols=384))
    plain = zsa.linear(x, w)
    q = zsa.paged_append(b.kvc, plain[:, 256:384], plain[:, 384:], b.seqs, b.len_dev, pos=pos, q=plain[:, :256],
                         n_heads=4)
    rows = [P.rows(f64(b.pool), b.table[s], n)[n - m:] for s, (n, m) in enumerate(((50, 5), (9, 9)))]
    got = np.concatenate([f64(q), np.concatenate(rows)], axis=1)
    # the epilogue rotates before its one rounding, the append after the
    # product's: one half step of each half of a pair more, and its own
    z = np.abs(f64(plain))
    z[:, :384] = np.broadcast_to(z[:, :384].reshape(14, 6, 2, 32).sum(2, keepdims=True), (14, 6, 2, 32)).reshape(14, 384)
    assert (np.abs(got - fused) <= 3 * 2.0 ** -8 * z * 1.01).all()


def test_append_outside_the_pool_is_lost():
    b = Batch("bf16", 4, 2, 64, 16, [40, 3, 1], [40, 2, 16], seed=1)
    b.table[0, 1] = -5
    b.table[2, 0] = b.pool.shape[0]
    b.table_dev.copy_(torch.from_numpy(b.table))
    lens = [40, 2, 17]  # a row below 0 and one beyond the table: neither is stored
    lens[2] = b.table.shape[1] * 16 + 1
    k = torch.randn(44, 128, device=dev()).to(torch.bfloat16)
    before = f64(b.pool)
    zsa.paged_append(b.kvc, k, k, b.seqs, torch.tensor(lens, dtype=torch.int32, device=dev()))
    ref = P.append(before, b.table, b.cu, lens, f64(k), f64(k))
    assert np.array_equal(np.nan_to_num(f64(b.pool)), np.nan_to_num(ref))


# ---------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,H,kv,hd", [("bf16", 8, 2, 64), ("bf16", 4, 4, 128), ("f32", 4, 2, 32)])
def test_generation(dtype, H, kv, hd):
    """Prompts in pieces and then single rows, all through the cache, against
    the packed attention over everything at once and the oracle."""
    g = np.random.default_rng(7)
    plen, pieces, steps, page = [70, 33, 129], [[40, 33, 100], [30, 0, 29]], 3, 16
    full = [n + steps for n in plen]
    dt, kvd, B = TYPES[dtype], kv * hd, len(plen)
    qkv = [torch.from_numpy(g.standard_normal((n, (H + 2 * kv) * hd)).astype(np.float32)).to(dt).to(dev()) for n in full]
    pages = [-(-n // page) for n in full]
    order = torch.from_numpy(g.permutation(sum(pages)).astype(np.int32)).to(dev())
    table = torch.full((B, max(pages)), -1, dtype=torch.int32, device=dev())
    for b, p in enumerate(pages):
        table[b, :p] = order[sum(pages[:b]):sum(pages[:b]) + p]
    pool = torch.full((sum(pages), page, 2 * kvd), float("nan"), dtype=dt, device=dev())
    cache = zsa.PagedKV(pool, table, kv)
    done, outs, lses, qs = [0] * B, [[] for _ in full], [[] for _ in full], [[] for _ in full]
    for new in pieces + [[1] * B] * steps:
        seqs = zsa.Seqs(new, dev())
        rows = torch.cat([qkv[b][done[b]:done[b] + n] for b, n in enumerate(new)])
        pos = torch.cat([torch.arange(done[b], done[b] + n, dtype=torch.int32) for b, n in enumerate(new)]).to(dev())
        done = [d + n for d, n in zip(done, new)]
        lens = torch.tensor(done, dtype=torch.int32, device=dev())
        q = zsa.paged_append(cache, rows[:, H * hd:H * hd + kvd], rows[:, H * hd + kvd:], seqs, lens, pos=pos,
                             q=rows[:, :H * hd], n_heads=H)
        out, lse = zsa.paged_attention(q, cache, H, seqs, lens, max_kv_len=max(done), want_lse=True)
        for b, n in enumerate(new):
            lo = int(seqs.host[b])
            outs[b].append(out[lo:lo + n])
            lses[b].append(lse[:, lo:lo + n])
            qs[b].append(q[lo:lo + n])
    assert done == full
    q = torch.cat([x for b in qs for x in b])
    out = torch.cat([x for b in outs for x in b])
    lse = torch.cat([x for b in lses for x in b], dim=1)
    seqs = zsa.Seqs(full, dev())
    rows = [torch.from_numpy(P.rows(f64(pool), table[b].tolist(), n)).to(dt).to(dev()) for b, n in enumerate(full)]
    fused = torch.cat([q, torch.cat(rows)], dim=1)
    whole, wlse, _ = zsa.attention_with_scores(fused[:, :H * hd], fused[:, H * hd:H * hd + kvd],
                                               fused[:, H * hd + kvd:], H, seqs, True, want_scores=False, n_kv_heads=kv)
    ref, rlse, size, mag = P.attention(f64(q), f64(pool), table.cpu().numpy(), [int(c) for c in seqs.host], full, H,
                                       kv, True)
    check = Batch(dtype, H, kv, hd, page, [1], [max(full)])
    check.compare(out, lse, ref, rlse, size, mag)
    check.compare(whole, wlse, ref, rlse, size, mag)


def test_other_streams_and_two_calls_at_once():
    a = Batch("bf16", 8, 2, 128, 16, [1, 1, 60], [900, 30, 200], 300, seed=1)
    b = Batch("f32", 4, 4, 64, 16, [1, 50], [700, 300], seed=2)
    want = [a.run(True), b.run(True)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(zsa.prefix_attention(x.q, x.kvc, x.H, x.seqs, x.len_dev, x.head_dev, x.prefix,
                                                   want_lse=True))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])


def test_captured_calls_with_other_lengths():
    """Two captured graphs with eager calls between their replays; the
    lengths on the device grow from replay to replay."""
    b = Batch("bf16", 8, 2, 64, 16, [1, 1, 1], [300, 200, 100], 100, seed=6)
    k = torch.randn(3, 128, device=dev()).to(torch.bfloat16)
    start = torch.tensor([200, 120, 1], dtype=torch.int32, device=dev())
    lens = start.clone()

    def step():
        zsa.paged_append(b.kvc, k, k, b.seqs, lens)
        own = zsa.paged_attention(b.q, b.kvc, 8, b.seqs, lens, max_kv_len=300, want_lse=True)
        both = zsa.prefix_attention(b.q, b.kvc, 8, b.seqs, lens, b.head_dev, 100, max_kv_len=300, want_lse=True)
        return own + both

    before = b.pool.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step()
        graphs.append((g, outs))
    for i in range(4):
        lens.copy_(start + i)
        b.pool.copy_(before)
        want = [x.clone() for x in step()]
        torch.cuda.synchronize()
        for g, outs in graphs:
            for x in outs:
                x.fill_(7.0)
            b.pool.copy_(before)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(outs, want):
                assert torch.equal(x, y)
    b.lens = [int(n) for n in lens.tolist()]
    b.compare(want[2], want[3], *b.oracle(True))


def test_arguments_by_name():
    b = Batch("bf16", 4, 2, 64, 16, [1, 2], [30, 20], 20, seed=1)
    want = b.run(True)
    got = zsa.prefix_attention(q=b.q, kv=b.kvc, n_heads=4, seqs=zsa.Seqs.wrap(b.cu, b.seqs.dev), kv_len=b.len_dev,
                               prefix_pages=b.head_dev, prefix_len=20, want_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    k = torch.randn((3, 128), device=dev()).to(torch.bfloat16)
    assert zsa.paged_append(kv=b.kvc, k=k, v=k, seqs=b.seqs, kv_len=b.len_dev) is None
    out, lse = zsa.paged_attention(q=b.q, kv=b.kvc, n_heads=4, seqs=b.seqs, kv_len=b.len_dev)
    assert lse is None and out.shape == b.q.shape


def test_lengths_on_the_device_that_are_out_of_range():
    # negative: no rows; beyond the bound: the rows up to it
    b = Batch("bf16", 4, 2, 64, 16, [1, 2, 40], [30, 20, 60], 20, seed=1)
    for lens in ([-5, 1 << 30, 2 ** 31 - 1], [-2 ** 31, 45, 64]):
        b.len_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        b.lens = lens
        out, lse = b.run(False, max_kv_len=20)
        ref, rlse, size, mag = b.oracle(False, max_kv_len=20)
        b.lens = [20] * 3
        b.compare(out, lse, ref, rlse, size, mag)


def test_nothing_to_do():
    b = Batch("bf16", 4, 2, 64, 16, [0, 0], [30, 0], seed=1)
    out, lse = b.run(True)
    assert out.shape == (0, 256) and lse.shape == (4, 0)
    k = torch.zeros((0, 128), dtype=torch.bfloat16, device=dev())
    assert zsa.paged_append(b.kvc, k, k, b.seqs, b.len_dev) is None


def test_python_refusals():
    b = Batch("bf16", 4, 2, 64, 16, [1, 2], [30, 20], 20, seed=1)
    k = torch.zeros((3, 128), dtype=torch.bfloat16, device=dev())
    pos = torch.zeros(3, dtype=torch.int32, device=dev())
    ok = (b.kvc, k, k, b.seqs, b.len_dev)
    zsa.paged_append(*ok, pos=pos)
    for bad in [(b.kvc, k[:2], k, b.seqs, b.len_dev), (b.kvc, k, k.float(), b.seqs, b.len_dev),
                (b.kvc, k, k, zsa.Seqs([3], dev()), b.len_dev), (b.kvc, k, k, b.seqs, b.len_dev.long()),
                (b.kvc, k, k, b.seqs, b.len_dev.cpu()), (b.kvc, k[:, :64], k, b.seqs, b.len_dev)]:
        with pytest.raises(ValueError):
            zsa.paged_append(*bad)
    with pytest.raises(ValueError):
        zsa.paged_append(*ok, pos=pos.long())
    with pytest.raises(ValueError):
        zsa.paged_append(*ok, pos=pos, q=b.q, n_heads=3)
    with pytest.raises(zsa.ZsaError) as e:
        zsa.paged_append(*ok, q=b.q, n_heads=4)
    assert e.value.code == zsa.EINVAL
    with pytest.raises(ValueError):
        zsa.paged_attention(b.q, b.kvc, 8, b.seqs, b.len_dev)
    with pytest.raises(zsa.ZsaError) as e:
        zsa.paged_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, max_kv_len=b.table.shape[1] * 16 + 1)
    assert e.value.code == zsa.ESHAPE
    with pytest.raises(zsa.ZsaError) as e:
        zsa.paged_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, scale=0.0)
    assert e.value.code == zsa.EINVAL
    with pytest.raises(ValueError):
        zsa.prefix_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, b.head_dev[:1], 20)
    with pytest.raises(ValueError):
        zsa.prefix_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, None, 20)
    with pytest.raises(ValueError):
        zsa.PagedKV(b.pool, b.table_dev.long(), 2)
    with pytest.raises(ValueError):
        zsa.PagedKV(b.pool, b.table_dev, 3)
    with pytest.raises(ValueError):
        zsa.PagedKV(b.pool.transpose(0, 1), b.table_dev, 2)
    with pytest.raises(ValueError):
        zsa.paged_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, max_kv_len=(1 << 32) + 20)
    with pytest.raises(ValueError):
        zsa.prefix_attention(b.q, b.kvc, 4, b.seqs, b.len_dev, b.head_dev, (1 << 32) + 20)
    with pytest.raises(ValueError):
        zsa.Seqs.wrap([0, 1, 3], b.seqs.dev.long())
