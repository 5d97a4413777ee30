"""The C ABI of the rotary positions, the 8-bit K/V cache and the attention over
it, as far as it needs no GPU: refusals before any launch with the documented
status, the rotary table against angles in 64 bits, and the plain 64-bit forms
themselves against hand-worked values."""
import ctypes
import math

import numpy as np
import pytest

import paper_2605_31057_amd as L
from oracle import cache as OC

ref = ctypes.byref
PTR = 0x100000


def _tensor(heads=2, n=10, d=128, data=PTR, sh=None, st=None):
    return L._Tensor(data, heads, n, d, n * d if sh is None else sh, d if st is None else st)


def _rope(frames=3, height=4, width=5, pairs=(22, 21, 21), layout=0, table=PTR):
    return L._Rope(frames, height, width, (ctypes.c_int32 * 3)(*pairs), layout, table)


def _cache(heads=2, capacity=256, block=128, n_tokens=100, k=PTR, v=2 * PTR, ks=3 * PTR,
           vs=4 * PTR):
    return L._KvCache(heads, capacity, block, n_tokens, k, v, ks, vs)


BAD_ROPES = [
    (dict(frames=0), L.EINVAL), (dict(height=0), L.EINVAL), (dict(width=-1), L.EINVAL),
    (dict(frames=1 << 20, height=1 << 10, width=2), L.EINVAL),
    (dict(pairs=(22, 21, 22)), L.EINVAL), (dict(pairs=(0, 0, 0)), L.EINVAL),
    (dict(pairs=(-1, 2, 3)), L.EINVAL), (dict(layout=2), L.EINVAL),
    (dict(table=None), L.EINVAL), (dict(table=PTR + 4), L.EUNSUPPORTED),
]


@pytest.mark.parametrize("fn", ["lvsa_rope_forward", "lvsa_rope_backward"])
def test_rope_refusals(fn):
    f = getattr(L.lib(), fn)
    x, y, r = _tensor(), _tensor(data=5 * PTR), _rope()
    assert f(None, 0, 0, ref(r), ref(y), None) == L.EINVAL
    assert f(ref(x), 0, 0, None, ref(y), None) == L.EINVAL
    assert f(ref(x), 0, 0, ref(r), None, None) == L.EINVAL
    assert f(ref(x), 3, 0, ref(r), ref(y), None) == L.EINVAL
    assert f(ref(x), 0, -1, ref(r), ref(y), None) == L.EINVAL
    assert f(ref(x), 0, 2 ** 31 - 5, ref(r), ref(y), None) == L.EINVAL
    for t, st in ((_tensor(n=0), L.EINVAL), (_tensor(heads=0), L.EINVAL),
                  (_tensor(data=None), L.EINVAL), (_tensor(d=64), L.EUNSUPPORTED),
                  (_tensor(data=PTR + 8), L.EUNSUPPORTED), (_tensor(st=132), L.EUNSUPPORTED),
                  (_tensor(sh=-128), L.EUNSUPPORTED)):
        assert f(ref(t), 0, 0, ref(r), ref(y), None) == st
    for t, st in ((_tensor(n=9, data=5 * PTR), L.EINVAL), (_tensor(heads=1, data=5 * PTR), L.EINVAL),
                  (_tensor(data=5 * PTR, st=64), L.EINVAL), (_tensor(data=5 * PTR, sh=0), L.EINVAL),
                  (_tensor(data=PTR, st=256), L.EINVAL)):   # in place: the same strides
        assert f(ref(x), 0, 0, ref(r), ref(t), None) == st
    for kw, st in BAD_ROPES:
        assert f(ref(x), 0, 0, ref(_rope(**kw)), ref(y), None) == st, kw


BAD_CACHES = [
    (dict(k=None), L.EINVAL), (dict(v=None), L.EINVAL), (dict(ks=None), L.EINVAL),
    (dict(vs=None), L.EINVAL), (dict(heads=0), L.EINVAL), (dict(n_tokens=-1), L.EINVAL),
    (dict(n_tokens=257), L.EINVAL), (dict(block=32), L.EUNSUPPORTED),
    (dict(capacity=192), L.EUNSUPPORTED), (dict(capacity=(1 << 24) + 128), L.EUNSUPPORTED),
    (dict(heads=65536), L.EUNSUPPORTED), (dict(k=PTR + 8), L.EUNSUPPORTED),
    (dict(v=PTR + 4), L.EUNSUPPORTED), (dict(ks=PTR + 2), L.EUNSUPPORTED),
]


def test_kv_write_refusals():
    f = L.lib().lvsa_kv_write
    x, c = _tensor(), _cache()
    for kw, st in BAD_CACHES:
        k = _tensor(heads=kw.get("heads", 2) or 2)
        assert f(ref(_cache(**kw)), ref(k), ref(k), 0, 0, None, None) == st, kw
    assert f(None, ref(x), ref(x), 0, 0, None, None) == L.EINVAL
    assert f(ref(c), None, ref(x), 0, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(x), None, 0, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(x), ref(x), -1, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(x), ref(x), 0, -1, None, None) == L.EINVAL
    assert f(ref(c), ref(x), ref(x), 0, 101, None, None) == L.EINVAL      # a hole
    assert f(ref(c), ref(_tensor(n=157)), ref(_tensor(n=157)), 0, 100, None, None) == L.EINVAL
    assert f(ref(c), ref(_tensor(n=0)), ref(_tensor(n=0)), 0, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(_tensor(heads=1)), ref(_tensor(heads=1)), 0, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(x), ref(_tensor(n=9)), 0, 0, None, None) == L.EINVAL
    assert f(ref(c), ref(x), ref(_tensor(d=64)), 0, 0, None, None) == L.EUNSUPPORTED
    for kw, st in BAD_ROPES:
        assert f(ref(c), ref(x), ref(x), 0, 0, ref(_rope(**kw)), None) == st, kw
    assert c.n_tokens == 100


def test_kv_read_refusals():
    f = L.lib().lvsa_kv_read
    x, y, c = _tensor(), _tensor(data=5 * PTR), _cache()
    for kw, st in BAD_CACHES:
        if kw.get("heads") != 65536:
            assert f(ref(_cache(**kw)), 0, ref(x), ref(y), 0, None) == st, kw
    assert f(None, 0, ref(x), ref(y), 0, None) == L.EINVAL
    assert f(ref(c), 0, None, None, 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(x), ref(y), 7, None) == L.EINVAL
    assert f(ref(c), -1, ref(x), ref(y), 0, None) == L.EINVAL
    assert f(ref(c), 91, ref(x), ref(y), 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(x), ref(x), 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(_tensor(n=0)), None, 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(x), ref(_tensor(n=9, data=5 * PTR)), 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(_tensor(heads=1)), None, 0, None) == L.EINVAL
    assert f(ref(c), 0, ref(_tensor(st=64)), None, 0, None) == L.EINVAL
    assert f(ref(c), 0, None, ref(_tensor(d=64)), 0, None) == L.EUNSUPPORTED


def test_attention_cache_refusals():
    lib = L.lib()

    def f(q, start, c, mask, out, need=None):
        m = None if mask is None else ref(mask)
        st = lib.lvsa_attention_cache(q and ref(q), start, c and ref(c), m, out and ref(out), None,
                                      0, None)
        nbytes = ctypes.c_int64()
        ws = lib.lvsa_attention_cache_workspace(q and ref(q), start, c and ref(c), m,
                                                ref(nbytes))
        if need is None:
            assert ws == st      # the same arguments are refused by both
        return st

    q, o, c = _tensor(heads=4), _tensor(heads=4, data=5 * PTR), _cache()
    mask = L.BlockMask(100, 64, 2, 2, PTR, PTR)
    for kw, st in BAD_CACHES:
        if kw.get("heads") != 65536:
            assert f(q, 0, _cache(**kw), None, o) == st, kw
    assert f(None, 0, c, None, o) == L.EINVAL
    assert f(q, 0, None, None, o) == L.EINVAL
    assert f(q, -1, c, None, o) == L.EINVAL
    assert f(_tensor(heads=3), 0, c, None, o) == L.EINVAL
    assert f(_tensor(heads=1), 0, c, None, o) == L.EINVAL
    assert f(_tensor(heads=4, n=0), 0, c, None, o) == L.EINVAL
    assert f(_tensor(heads=4, d=64), 0, c, None, o) == L.EUNSUPPORTED
    assert f(_tensor(heads=4, n=1 << 26, sh=128, st=128), 0, c, None, o) == L.EUNSUPPORTED
    assert f(q, 91, c, mask, o) == L.EINVAL
    for bad, st in (((99, 64, 2, 2, PTR, PTR), L.EINVAL), ((100, 64, 1, 2, PTR, PTR), L.EINVAL),
                    ((100, 64, 2, 3, PTR, PTR), L.EINVAL), ((100, 64, 2, 2, None, PTR), L.EINVAL),
                    ((100, 64, 2, 2, PTR, None), L.EINVAL),
                    ((100, 32, 4, 4, PTR, PTR), L.EUNSUPPORTED)):
        assert f(q, 0, c, L.BlockMask(*bad), o) == st, bad
    n = 8001 * 64
    big = _cache(capacity=8064 * 64, n_tokens=n)
    assert f(q, 0, big, L.BlockMask(n, 64, 8001, 8001, PTR, PTR), o) == L.EUNSUPPORTED
    for out, st in ((None, L.EINVAL), (_tensor(heads=4, n=9, data=5 * PTR), L.EINVAL),
                    (_tensor(heads=2, data=5 * PTR), L.EINVAL), (_tensor(heads=4), L.EINVAL),
                    (_tensor(heads=4, data=5 * PTR, st=64), L.EINVAL),
                    (_tensor(heads=4, data=5 * PTR + 8), L.EUNSUPPORTED)):
        assert f(q, 0, c, None, out, need=False) == st


def test_rope_table():
    grid, pairs = (121, 30, 52), (22, 21, 21)
    r = _rope(*grid, pairs)
    n = ctypes.c_int64()
    assert L.lib().lvsa_rope_table_size(ref(r), ref(n)) == L.OK
    assert n.value == 121 * 22 + 30 * 21 + 52 * 21
    buf = np.full((n.value + 1, 2), 7.0, dtype=np.float32)
    at = buf.ctypes.data_as(ctypes.c_void_p)
    assert L.lib().lvsa_rope_table(ref(r), 10000.0, at, n.value) == L.OK
    want = np.concatenate([np.stack([np.cos(a), np.sin(a)], -1).reshape(-1, 2)
                           for a in OC.rope_table(grid, pairs)])
    # one rounding to fp32 (2^-25 of a value below 1) over 64-bit angles up to 120
    assert np.abs(buf[:-1] - want).max() <= 2.0 ** -25 + 1e-12
    assert (buf[-1] == 7.0).all()
    for theta, cap, st in ((0.0, n.value, L.EINVAL), (-1.0, n.value, L.EINVAL),
                           (math.inf, n.value, L.EINVAL), (math.nan, n.value, L.EINVAL),
                           (10000.0, n.value - 1, L.EINVAL)):
        assert L.lib().lvsa_rope_table(ref(r), theta, at, cap) == st
    assert L.lib().lvsa_rope_table(ref(r), 1e4, None, n.value) == L.EINVAL
    assert L.lib().lvsa_rope_table(None, 1e4, at, n.value) == L.EINVAL
    assert L.lib().lvsa_rope_table_size(ref(r), None) == L.EINVAL


def test_plain_forms_against_hand_values():
    # e4m3: steps of 1/8 in [1, 2), of 32 in [256, 448], of 2^-9 below 2^-6
    x = np.array([1.0, 1.0625, 1.1875, 1.06, 300.0, 432.0, 448.0, 2.0 ** -10, 1.5 * 2.0 ** -9,
                  -0.3])
    assert OC.e4m3(x).tolist() == [1.0, 1.0, 1.25, 1.0, 288.0, 448.0, 448.0, 0.0, 2.0 ** -8,
                                   -0.3125]
    assert OC.block_scale(np.array([448.0, -3.0])) == 1.0
    assert OC.block_scale(np.array([448.5])) == 2.0
    assert OC.block_scale(np.array([224.0, np.nan, np.inf])) == 0.5
    assert OC.block_scale(np.zeros(3)) == 2.0 ** -117
    # one pair turned by a quarter: (a, b) -> (-b, a)
    x = np.zeros((1, 1, 128))
    x[0, 0, :2] = 3.0, 4.0
    cos, sin = np.ones((1, 64)), np.zeros((1, 64))
    cos[0, 0], sin[0, 0] = 0.0, 1.0
    assert OC.rotate(x, cos, sin, False)[0, 0, :2].tolist() == [-4.0, 3.0]
    y = OC.rotate(np.roll(x, 0), cos, sin, True)
    assert y[0, 0, 0] == 0.0 and y[0, 0, 64] == 3.0 and y[0, 0, 1] == 4.0
    # two keys whose scores differ by ln 3: weights 1/4 and 3/4
    q, k, v = np.zeros((1, 1, 128)), np.zeros((1, 2, 128)), np.zeros((1, 2, 128))
    q[0, 0, 0], k[0, 1, 0] = np.sqrt(128), np.log(3)
    v[0, 0, 0], v[0, 1, 1] = 4.0, 4.0
    out = OC.attend(q, k, v)[0]
    assert np.allclose(out[0, 0, :2], [1.0, 3.0])


def test_python_refusals():
    import torch
    with pytest.raises(L.LvsaError):
        L.Rope(0, 4, 5, device="cpu")
    with pytest.raises(ValueError):
        L.Rope(3, 4, 5, table=torch.zeros(7, 2), device="cpu")
    with pytest.raises(ValueError):
        L.KvCache(2, 256, n_tokens=257, device="cpu")
    for bad in (dict(frames=2 ** 32 + 3), dict(pairs=(2 ** 32, 21, 21)), dict(height=-1)):
        with pytest.raises(L.LvsaError):
            L.Rope(**{**dict(frames=3, height=4, width=5, device="cpu"), **bad})
    for bad in ((2, 256, 32), (2, 0, 64), (2, (1 << 24) + 1, 64), (0, 128, 64), (65536, 128, 64)):
        with pytest.raises(L.LvsaError):
            L.KvCache(*bad, device="cpu")
    for at in (-1, 2 ** 31, 2 ** 32):      # ctypes would take 2^32 for 0
        with pytest.raises(L.LvsaError):
            L._place(at)
    c = L.KvCache(2, 200, 64, device="cpu")
    assert (c.heads, c.capacity, c.block, c.n_tokens) == (2, 256, 64, 0)
    with pytest.raises(ValueError):
        c.n_tokens = -1
    with pytest.raises(ValueError):
        L.KvCache(2, 256, buffers=(c.k, c.v, c.k_scale, c.v_scale))   # block 128: other scales
    with pytest.raises((ValueError, RuntimeError)):
        L.kv_read(c, out=(torch.zeros(2, 4, 128), torch.zeros(2, 4, 128)))   # not on a device
