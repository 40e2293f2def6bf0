"""What the long-context operators answer before they touch a device.  No GPU needed."""
import ctypes as C

import numpy as np
import pytest

import long_context as L
from paper_2501_08090_amd import binding as B

INVALID, SHAPE = -1, -2
FAKE = 1 << 20  # an aligned address that is never read: every call here is refused first


def refused(rc, want):
    assert rc == want and B.last_error() != ""


def test_null_handles():
    lib = B.load()
    assert lib.chiron_kv8_pool_bytes(None, 5) == 0 and lib.chiron_kv8_pool_destroy(None) == 0
    out = C.c_void_p(5)
    refused(lib.chiron_kv8_pool_create(None, C.c_void_p(FAKE), C.c_uint64(1 << 30), 4, B.CHIRON_INT8, C.byref(out)), INVALID)
    assert not out.value
    refused(lib.chiron_kv8_pool_create(None, C.c_void_p(FAKE), C.c_uint64(1 << 30), 4, B.CHIRON_INT8, None), INVALID)
    refused(lib.chiron_kv8_append_rope(None, 0, FAKE, FAKE, 1, FAKE, FAKE, 1, 1, None), INVALID)
    refused(lib.chiron_kv8_gather(None, 0, FAKE, 1, FAKE, FAKE, 1, FAKE, FAKE, None), INVALID)
    refused(lib.chiron_op_row_attention(None, 0, FAKE, FAKE, None), INVALID)
    refused(lib.chiron_op_row_attention8(None, 0, FAKE, FAKE, None), INVALID)
    refused(lib.chiron_kv_grant_pages(None, FAKE, 4, FAKE, FAKE, 1, 1, FAKE, FAKE, None), INVALID)
    refused(lib.chiron_kv_release_pages(None, FAKE, 4, FAKE, None, 1, FAKE, None), INVALID)


def page_list(pages=FAKE, count=FAKE, capacity=10):
    return B.PageListArgs(pages, count, capacity)


def maps(row_starts=FAKE):
    return B.RowMapArgs(row_starts, None, None, None, None)


@pytest.mark.parametrize("lst,bt,width,seq,new,batch,rows,out,work,want", (
    (dict(count=None), FAKE, 4, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    (dict(pages=None), FAKE, 4, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    (dict(capacity=-1), FAKE, 4, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    (dict(capacity=(1 << 30) + 1), FAKE, 4, FAKE, FAKE, 1, 1, {}, FAKE, SHAPE),
    ({}, None, 4, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    ({}, FAKE, 0, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    ({}, FAKE, (1 << 26) + 1, FAKE, FAKE, 1, 1, {}, FAKE, INVALID),
    ({}, FAKE, 4, None, FAKE, 1, 1, {}, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, None, 1, 1, {}, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, FAKE, -1, 1, {}, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, FAKE, 1, -1, {}, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, FAKE, 1, (1 << 30) + 1, {}, FAKE, SHAPE),
    ({}, FAKE, 4, FAKE, FAKE, 1, 1, dict(row_starts=None), FAKE, INVALID),
    ({}, FAKE, 4, FAKE, FAKE, 1, 1, {}, None, INVALID),
    ({}, FAKE, 4, FAKE, FAKE, 1, 1, {}, FAKE + 8, INVALID),
))
def test_grant_refusals(lst, bt, width, seq, new, batch, rows, out, work, want):
    a, m = page_list(**lst), maps(**out)
    refused(B.load().chiron_kv_grant_pages(C.addressof(a), bt, width, seq, new, batch, rows, C.addressof(m), work, None), want)


@pytest.mark.parametrize("lst,bt,width,first,batch,work,want", (
    (dict(count=None), FAKE, 4, FAKE, 1, FAKE, INVALID),
    ({}, None, 4, FAKE, 1, FAKE, INVALID),
    ({}, FAKE, 0, FAKE, 1, FAKE, INVALID),
    ({}, FAKE, 4, None, 1, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, -1, FAKE, INVALID),
    ({}, FAKE, 4, FAKE, 1, None, INVALID),
    ({}, FAKE, 4, FAKE, 1, FAKE + 4, INVALID),
))
def test_release_refusals(lst, bt, width, first, batch, work, want):
    a = page_list(**lst)
    refused(B.load().chiron_kv_release_pages(C.addressof(a), bt, width, first, None, batch, work, None), want)
    assert B.load().chiron_kv_release_pages(C.addressof(page_list()), None, 4, None, None, 0, FAKE, None) == 0  # nobody: nothing to do


def test_workspaces():
    pages, rows = B.load().chiron_kv_pages_workspace_bytes, B.load().chiron_row_attention_workspace_bytes
    assert pages(-1) == 0 and 0 < pages(0) < pages(1000) and pages(999) % 16 == 0
    assert rows(32, 8, 128, 64, 64, 1) % 16 == 0 and 0 < rows(32, 8, 128, 64, 64, 1) < rows(32, 8, 128, 1024, 1024, 1)
    assert rows(32, 8, 128, 1, 100, 100) > rows(32, 8, 128, 1, 5, 5) > 0
    assert rows(32, 8, 128, 3, 5, 1 << 30) == rows(32, 8, 128, 3, 5, 5) and rows(16, 16, 64, 1, 40, 40) > 0  # fewer rows than a tile has
    for bad in ((0, 8, 128, 1, 1, 1), (32, 0, 128, 1, 1, 1), (33, 8, 128, 1, 1, 1), (136, 8, 128, 1, 1, 1), (32, 8, 96, 1, 1, 1), (32, 8, 128, 0, 1, 1),
                (32, 8, 128, 1, 0, 1), (32, 8, 128, 1, 1, 0), (32, 8, 128, -1, -1, -1)):
        assert rows(*bad) == 0


def test_format_names():
    with pytest.raises(ValueError):
        B.KVPool8(None, 4, "e5m2")


@pytest.mark.parametrize("fmt", ("int8", "e4m3"))
def test_definition_of_the_8_bit_page(fmt):
    """the power of two is the smallest that holds the page, values are off by at most half a step, and by a whole one where an old value
    was rounded twice"""
    rng = np.random.default_rng(3)
    for scale in (1e-40, 1e-3, 1.0, 5e4, 1e38):
        x = rng.standard_normal((9, 64)) * scale
        got, e = L.store(np.zeros((0, 64)), 99, x, fmt)
        amax = abs(L.bounded(x)).max()
        assert e == L.MIN_EXP or L.TOP[fmt] * 2.0 ** (e - 1) < amax <= L.TOP[fmt] * 2.0 ** e
        step = 2.0 ** e if fmt == "int8" else np.maximum(abs(L.bounded(x)) * 2.0 ** -3, 2.0 ** (e - 9))
        assert (abs(got - L.bounded(x)) <= 0.5 * step).all()
        both, e2 = L.store(got, e, x[:3] * 5, fmt)
        assert e2 >= e and (abs(both[:9] - L.bounded(x)) <= (2.0 ** e2 if fmt == "int8" else np.maximum(step, 2.0 ** (e2 - 9)))).all()
    got, e = L.store(np.zeros((0, 2)), 0, np.array([[np.nan, 0.0]]), fmt)
    assert e == L.MIN_EXP and (got == 0).all()
    got, e = L.store(np.zeros((0, 2)), 0, np.array([[np.inf, -1e39]]), fmt)
    assert np.array_equal(got, [[2.0 ** 100, -(2.0 ** 100)]])


def test_definition_of_grants_and_releases():
    """pages are conserved, a grant repeated on its own result changes nothing, and a release undoes it"""
    rng = np.random.default_rng(4)
    bt = np.full((5, 6), -1, np.int32)
    old, new = np.array([0, 16, 5, 40, 90]), np.array([3, 1, 0, 30, 7])
    for i, o in enumerate(old):
        bt[i, :-(-o // 16)] = rng.permutation(100)[:-(-o // 16)] + 100 * i
    before = bt.copy()
    left, starts, seq, pos, slots, granted = L.grant(bt, [900, 901, 902, 903, 904, 905], old, new, 50)
    assert granted.tolist() == [3, 1, 0, 30, 0] and starts.tolist() == [0, 3, 4, 4, 34, 34] and left == [900, 901]  # 97 tokens do not fit 96
    assert bt[0, 0] == 902 and bt[1, 1] == 903 and bt[3, 3:5].tolist() == [904, 905] and seq[34] == -1 and slots[0] == 902 * 16
    again = bt.copy()
    assert L.grant(again, left, old, new, 50)[0] == left and np.array_equal(again, bt)
    assert L.release(bt, left, old) == [900, 901, 902, 903, 904, 905] and np.array_equal(bt, before)
