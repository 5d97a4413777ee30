"""Tensors that the rotary, cache and cache-attention calls write: layouts in which two
rows share elements are refused, every other one is accepted."""
import ctypes
import random

import pytest

import paper_2605_31057_amd as L

ref = ctypes.byref
PTR = 0x100000


def _tensor(heads, n, sh, st, data=PTR):
    return L._Tensor(data, heads, n, 128, sh, st)


def _rope(table):
    return L._Rope(3, 4, 5, (ctypes.c_int32 * 3)(22, 21, 21), 0, table)


def _status(heads, n, sh, st):
    """Of a rotation whose table is refused after its tensors: nothing is launched."""
    x, y = _tensor(heads, n, n * 128, 128), _tensor(heads, n, sh, st, 5 * PTR)
    return L.lib().lvsa_rope_forward(ref(x), 0, 0, ref(_rope(PTR + 4)), ref(y), None)


def _shared(heads, n, sh, st):
    rows = sorted(h * sh + t * st for h in range(heads) for t in range(n))
    return any(b - a < 128 for a, b in zip(rows, rows[1:]))


@pytest.mark.parametrize("heads,n,sh,st", [
    (2, 10, 128, 128), (2, 2, 128, 128), (3, 4, 256, 128), (2, 3, 128, 192), (4, 4, 384, 256),
    (2, 10, 128 * 9, 128), (40, 1560, 128 * 1559, 128), (1000, 7, 128, 128 * 999),
    (2, 3, 128 * 3 + 8, 128 * 2)])
def test_rows_that_share_elements_are_refused(heads, n, sh, st):
    assert _shared(heads, n, sh, st)
    assert _status(heads, n, sh, st) == L.EINVAL
    x, bad = _tensor(heads, n, n * 128, 128), _tensor(heads, n, sh, st, 5 * PTR)
    c = L._KvCache(heads, 2048, 128, 2000, PTR, 2 * PTR, 3 * PTR, 4 * PTR)
    lib = L.lib()
    assert lib.lvsa_kv_read(ref(c), 0, ref(bad), None, 0, None) == L.EINVAL
    assert lib.lvsa_kv_read(ref(c), 0, None, ref(bad), 0, None) == L.EINVAL
    assert lib.lvsa_attention_cache(ref(x), 0, ref(c), None, ref(bad), None, 0, None) == L.EINVAL
    r = _rope(PTR)
    same = _tensor(heads, n, sh, st)
    assert lib.lvsa_rope_backward(ref(same), 0, 0, ref(r), ref(same), None) == L.EINVAL   # in place


@pytest.mark.parametrize("heads,n,sh,st", [
    (2, 10, 1280, 128), (2, 10, 128, 256), (2, 10, 136, 264), (1, 10, 0, 128), (2, 1, 128, 8),
    (2, 3, 128 * 3, 128 * 2), (3, 3, 128, 384), (2, 2, 384, 256), (65535, 1 << 27, 128, 128 * 65535),
    (40, 1 << 20, 1 << 40, 128), (2, 1 << 27, 1 << 62, 1 << 30)])
def test_rows_apart_are_accepted(heads, n, sh, st):
    assert _status(heads, n, sh, st) == L.EUNSUPPORTED       # the table


def test_rows_against_their_elements():
    rng = random.Random(1)
    seen = set()
    for _ in range(4000):
        heads, n = rng.randint(1, 6), rng.randint(1, 6)
        sh, st = (8 * rng.randint(16, 110) for _ in range(2))
        shared = _shared(heads, n, sh, st)
        seen.add(shared)
        assert (_status(heads, n, sh, st) == L.EINVAL) == shared, (heads, n, sh, st)
    assert seen == {False, True}
