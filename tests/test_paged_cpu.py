"""The paged cache's C entry points on the CPU: what they refuse before any
launch, and the oracle of the paged operators against plain forms."""
import ctypes

import numpy as np
import pytest

from oracle import paged as P
from paper_2509_01190_amd import zsa

PTR = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(12)]


def cache(**kw):
    c = dict(pool=0x100000, table=0x200000, page_stride=16 * 2 * 128, table_stride=4, n_pages=8, page_size=16,
             max_pages=4, n_kv_heads=2, head_dim=64, dtype=zsa.BF16)
    c.update(kw)
    return zsa.PagedKvStruct(*[c[n] for n, _ in zsa.PagedKvStruct._fields_])


def cu(*v):
    return np.array(v, dtype=np.int32)


def append(c=None, k=PTR[0], ks=128, v=PTR[1], vs=128, q=None, qs=0, H=0, qo=None, qos=0, pos=None, theta=1e4,
           offs=(0, 1, 3), dev=PTR[6], kv_len=PTR[5]):
    h = cu(*offs)
    c = cache() if c is None else c
    return zsa.lib().zsa_paged_append(None, ctypes.byref(c), k, ks, v, vs, q, qs, H, qo, qos, pos, theta,
                                      len(h) - 1, zsa._hp32(h), dev, kv_len)


def attend(c=None, q=PTR[0], qs=256, H=4, scale=0.125, offs=(0, 1, 3), dev=PTR[6], kv_len=PTR[5], most=64, pages=None,
           prefix=0, out=PTR[2], os=256, lse=None, ws=None, wsb=0):
    h = cu(*offs)
    c = cache() if c is None else c
    return zsa.lib().zsa_prefix_attention(None, ctypes.byref(c), q, qs, H, 1, scale, len(h) - 1, zsa._hp32(h), dev,
                                          kv_len, most, pages, prefix, out, os, lse, ws, wsb)


ODD = ctypes.c_void_p(0x1004)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), zsa.EINVAL), (dict(head_dim=48), zsa.EUNSUPPORTED), (dict(n_kv_heads=0), zsa.EINVAL),
    (dict(page_size=24), zsa.EUNSUPPORTED), (dict(page_size=8), zsa.EUNSUPPORTED), (dict(page_size=0), zsa.EUNSUPPORTED),
    (dict(n_pages=-1), zsa.ESHAPE), (dict(max_pages=-1), zsa.ESHAPE), (dict(table_stride=3), zsa.ESHAPE),
    (dict(pool=None), zsa.EINVAL), (dict(pool=0x100008), zsa.EALIGN), (dict(table=None), zsa.EINVAL),
    (dict(page_stride=16 * 2 * 128 - 8), zsa.ESHAPE), (dict(page_stride=16 * 2 * 128 + 4), zsa.EALIGN),
    (dict(page_size=1 << 20, page_stride=1 << 40, n_kv_heads=16), zsa.EUNSUPPORTED),
])
def test_caches_that_are_refused(kw, code):
    assert append(cache(**kw), ks=4096, vs=4096) == code
    assert attend(cache(**kw), H=16 if kw.get("n_kv_heads") == 16 else 4, qs=4096, os=4096) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), zsa.EINVAL), (dict(v=None), zsa.EINVAL), (dict(k=ODD), zsa.EALIGN), (dict(ks=64), zsa.ESHAPE),
    (dict(ks=129), zsa.EALIGN), (dict(vs=120), zsa.ESHAPE), (dict(kv_len=None), zsa.EINVAL), (dict(dev=None), zsa.EINVAL),
    (dict(offs=(0, 3, 1)), zsa.ESHAPE), (dict(offs=(1, 2, 3)), zsa.ESHAPE),
    (dict(pos=PTR[4], theta=0.0), zsa.EINVAL), (dict(pos=PTR[4], theta=float("nan")), zsa.EINVAL),
    (dict(q=PTR[2], qs=256, H=4, qo=PTR[3], qos=256), zsa.EINVAL),               # no positions
    (dict(q=PTR[2], qs=256, H=4, qo=None, qos=256, pos=PTR[4]), zsa.EINVAL),
    (dict(q=PTR[2], qs=256, H=3, qo=PTR[3], qos=256, pos=PTR[4]), zsa.ESHAPE),    # 2 does not divide 3
    (dict(q=PTR[2], qs=256, H=0, qo=PTR[3], qos=256, pos=PTR[4]), zsa.EINVAL),
    (dict(q=PTR[2], qs=248, H=4, qo=PTR[3], qos=256, pos=PTR[4]), zsa.ESHAPE),
    (dict(offs=(0, 1 << 24)), zsa.EUNSUPPORTED),
    (dict(q=PTR[2], qs=256, H=4, qo=ODD, qos=256, pos=PTR[4]), zsa.EALIGN),
])
def test_appends_that_are_refused(kw, code):
    assert append(**kw) == code
    assert zsa.lib().zsa_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), zsa.EINVAL), (dict(out=None), zsa.EINVAL), (dict(q=ODD), zsa.EALIGN), (dict(qs=128), zsa.ESHAPE),
    (dict(qs=260), zsa.EALIGN), (dict(os=128), zsa.ESHAPE), (dict(H=3), zsa.ESHAPE), (dict(H=0), zsa.EINVAL),
    (dict(scale=0.0), zsa.EINVAL), (dict(scale=float("nan")), zsa.EINVAL), (dict(kv_len=None), zsa.EINVAL),
    (dict(dev=None), zsa.EINVAL), (dict(offs=(0, 2, 1)), zsa.ESHAPE), (dict(most=-1), zsa.EINVAL),
    (dict(most=65), zsa.ESHAPE),                                                 # beyond the table
    (dict(prefix=-1), zsa.EINVAL), (dict(prefix=20), zsa.EINVAL),                # no prefix pages
    (dict(prefix=40000, pages=PTR[7]), zsa.EWORKSPACE),
    (dict(prefix=40000, pages=PTR[7], wsb=1 << 40), zsa.EINVAL),                              # parts, and no workspace
    (dict(prefix=40000, pages=PTR[7], ws=PTR[8], wsb=64), zsa.EWORKSPACE),
    (dict(prefix=40000, pages=PTR[7], ws=ODD, wsb=1 << 30), zsa.EALIGN),
    (dict(prefix=(1 << 30) + 1, pages=PTR[7]), zsa.EUNSUPPORTED),
    (dict(offs=(0, 1 << 30), H=2, qs=128, os=128, lse=PTR[3]), zsa.EUNSUPPORTED),
])
def test_attentions_that_are_refused(kw, code):
    assert attend(**kw) == code
    assert zsa.lib().zsa_last_error()


def test_no_rows_need_no_pointers():
    c = cache(pool=None, table=None, n_pages=0, max_pages=0, table_stride=0)
    assert append(c, k=None, v=None, kv_len=None, offs=(0, 0, 0)) == zsa.OK
    assert attend(c, q=None, out=None, kv_len=None, offs=(0, 0, 0), most=0) == zsa.OK


def test_workspace_is_that_of_the_parts():
    c = cache()
    h = cu(0, 1, 3)
    size = zsa.lib().zsa_paged_attention_workspace_size
    assert size(ctypes.byref(c), 4, 2, zsa._hp32(h), 64, 0) == 0                 # one part: written at once
    assert size(ctypes.byref(c), 4, 2, zsa._hp32(h), 64, 20) == 0                # a short prefix is read with the rows' own
    two = size(ctypes.byref(c), 4, 2, zsa._hp32(h), 64, 40000)
    assert two >= 2 * 3 * 4 * (2 + 64) * 4                                       # the prefix's part and the rows' own
    assert size(None, 4, 2, zsa._hp32(h), 64, 40000) == 0
    assert size(ctypes.byref(c), 4, 2, zsa._hp32(cu(0, 0, 0)), 64, 40000) == 0


@pytest.mark.parametrize("kw,most,prefix", [
    (dict(head_dim=0), 4096, 40000), (dict(head_dim=-16), 4096, 0), (dict(head_dim=48), 4096, 40000),
    (dict(dtype=7), 4096, 40000), (dict(), (1 << 31) - 1, 0), (dict(), 64, (1 << 31) - 1),
])
def test_calls_that_are_refused_need_no_workspace(kw, most, prefix):
    c, h = cache(max_pages=1 << 27, table_stride=1 << 27, **kw), cu(0, 1, 3)
    assert zsa.lib().zsa_paged_attention_workspace_size(ctypes.byref(c), 4, 2, zsa._hp32(h), most, prefix) == 0
    assert attend(c, qs=4096, os=4096, most=most, pages=PTR[7], prefix=prefix) in (zsa.EINVAL, zsa.EUNSUPPORTED, zsa.ESHAPE)


@pytest.mark.parametrize("most,prefix", [(1 << 30, 0), (64, 1 << 30), (1 << 30, 1 << 30)])
def test_workspace_of_the_longest(most, prefix):
    c = cache(max_pages=1 << 26, table_stride=1 << 26)
    h = np.arange(5001, dtype=np.int32)
    size = zsa.lib().zsa_paged_attention_workspace_size
    assert 5000 * 4 * 66 * 4 < size(ctypes.byref(c), 4, 5000, zsa._hp32(h), most, prefix) < 1 << 36


# ---------------------------------------------------------------------------- the oracle
def test_oracle_against_plain_softmax():
    g = np.random.default_rng(0)
    pool = g.standard_normal((6, 16, 2 * 2 * 8))
    table = np.array([[3, 1], [0, 5]])
    q = g.standard_normal((5, 4 * 8))
    out, lse, size, mag = P.attention(q, pool, table, [0, 2, 5], [20, 3], 4, 2, True, prefix_pages=[4], prefix_len=7)
    for b, (lo, hi, m) in enumerate([(0, 2, 20), (2, 5, 3)]):
        rows = np.concatenate([pool[4, :7], pool[table[b, 0]], pool[table[b, 1]]])[:7 + m]
        for h in range(4):
            k, v = rows[:, (h // 2) * 8:(h // 2 + 1) * 8], rows[:, 16 + (h // 2) * 8:16 + (h // 2 + 1) * 8]
            s = q[lo:hi, h * 8:(h + 1) * 8] @ k.T / np.sqrt(8)
            i, j = np.indices(s.shape)
            s[j > len(rows) - (hi - lo) + i] = -np.inf
            p = np.exp(s)
            assert np.allclose(out[lo:hi, h * 8:(h + 1) * 8], p @ v / p.sum(1, keepdims=True))
            assert np.allclose(lse[h, lo:hi], np.log(p.sum(1)))


def test_oracle_rows_without_keys_and_missing_pages():
    g = np.random.default_rng(1)
    pool = g.standard_normal((2, 16, 16))
    table = np.array([[1], [9]])
    q = g.standard_normal((4, 8))
    out, lse, _, _ = P.attention(q, pool, table, [0, 3, 4], [2, 5], 1, 1, True)
    assert np.isneginf(lse[0, 0]) and not out[0].any()
    assert np.allclose(out[1], pool[1, 0, 8:])          # one key: its value
    assert not out[3].any() and np.isclose(lse[0, 3], np.log(5))  # five rows of zeros
    stored = P.append(pool, table, [0, 3, 4], [2, 5], np.ones((4, 8)), 2 * np.ones((4, 8)))
    assert (stored[1, :2, :8] == 1).all() and (stored[1, :2, 8:] == 2).all()
    assert np.array_equal(stored[1, 2:], pool[1, 2:]) and np.array_equal(stored[0], pool[0])


def test_oracle_rotation_is_the_stack_oracles():
    from oracle import zsa_oracle as O
    g = np.random.default_rng(2)
    x, pos = g.standard_normal((6, 2 * 16)), g.integers(0, 5000, 6)
    y = P.rotate(x, pos, 1e4, 16)
    # lengths of pairs stay, position 0 changes nothing, angles add up; as the stack's oracle has it
    z, w = x.reshape(6, 2, 2, 8), y.reshape(6, 2, 2, 8)
    assert np.allclose((z ** 2).sum(2), (w ** 2).sum(2))
    assert np.allclose(P.rotate(x, np.zeros(6), 1e4, 16), x)
    assert np.allclose(P.rotate(P.rotate(x, pos, 1e4, 16), 3 * pos, 1e4, 16), P.rotate(x, 4 * pos, 1e4, 16))
    assert np.allclose(P.rotate(x, pos, 1e4, 16), O.rope(x, pos, 2, 1e4))
