"""What the binding of a pool's pages takes and refuses, before anything of it goes to a device (host only)."""
import ctypes as C

import numpy as np
import pytest

import paper_2602_21548_amd as K
from paper_2602_21548_amd import pages as P


class NoPools:
    """Pools that no call may come to."""

    @property
    def handle(self):
        raise AssertionError("the copies were taken")


@pytest.mark.parametrize("copies", [np.array([[-2 ** 63, 5]]), np.array([[2 ** 63, 5]], dtype=np.uint64), np.array([[5, 2 ** 64 - 1]], dtype=np.uint64), np.array([[5, -2 ** 31 - 1]]),
                                    np.array([[2 ** 31, 5]]), np.array([[2 ** 32, 5]]), [[-2 ** 63, 5]], [[5, 2 ** 63]], [[5, 2 ** 70]]])
def test_copies_of_blocks_that_32_bits_do_not_hold(copies):
    with pytest.raises(ValueError):
        K.kvl_copy_blocks(NoPools(), copies)


def held(tables):
    """Bytes that tables keep, by the arrays that they are parts of."""
    bases = {}
    for t in tables:
        while t.base is not None:
            t = t.base
        bases[id(t)] = t.nbytes
    return sum(bases.values())


def test_short_tables_after_a_long_one_do_not_keep_its_room():
    pages = K.kvl_pages(16, 300000)
    long, short, none = K.kvl_pages_adopt(pages, [np.arange(250000), np.array([299999, 7, 250001]), np.array([], dtype=np.int32)], [16 * 250000, 37, 0])
    for _ in range(3):
        t = K.kvl_pages_tables(pages, [long])
        assert held(t) <= 4 * 4 * 250000 and np.array_equal(t[0], np.arange(250000))
        t = K.kvl_pages_tables(pages, [short, none, short])
        assert [x.tolist() for x in t] == [[299999, 7, 250001], [], [299999, 7, 250001]] and all(x.dtype == np.int32 for x in t)
        assert held(t) <= 4 * 4 * 6
        assert held(K.kvl_pages_tables(pages, [none])) == 0 and K.kvl_pages_tables(pages, []) == []
    # (and each call's are its own)
    a, b = K.kvl_pages_tables(pages, [short]), K.kvl_pages_tables(pages, [short])
    a[0][:] = 1
    assert b[0].tolist() == [299999, 7, 250001]


@pytest.mark.parametrize("table", [np.array([2 ** 32 + 1, 2]), np.array([2, -2 ** 32]), np.array([2 ** 63, 2], dtype=np.uint64), np.array([2 ** 32 - 1, 2], dtype=np.uint32)])
def test_tables_of_blocks_that_32_bits_do_not_hold(table):
    """Adopted, or of a plan: as other blocks outside the pool."""
    pages = K.kvl_pages(16, 8)
    layout, attn = K.make_layout(1, 16, [64], 8), K.make_attn_layout(16, 2, 1, 64, 8)
    for call in (lambda: K.kvl_pages_adopt(pages, [np.array([0, 1]), table], [20, 20]), lambda: K.kvl_plan(layout, [20], [5], [table], K.KVL_GATHER | K.KVL_HOST_ONLY),
                 lambda: K.kvl_attn_plan(attn, [20], [5], [table], K.KVL_GATHER | K.KVL_HOST_ONLY)):
        with pytest.raises(K.KvlError) as e:
            call()
        assert e.value.code == K.KVL_ERANGE
    assert K.kvl_pages_stats(pages)["sequences"] == 0
    for hit, app in ((np.array([2 ** 32]), [5]), ([20], np.array([2 ** 32 + 5])), (np.array([-2 ** 32]), [5])):
        with pytest.raises(K.KvlError) as e:
            K.kvl_attn_plan(attn, hit, app, [np.array([1, 2])], K.KVL_GATHER | K.KVL_HOST_ONLY)
        assert e.value.code == K.KVL_ERANGE
    assert K.kvl_pages_adopt(pages, [np.array([5, 2]), [6, 1]], np.array([20, 20])).size == 2      # (other types hold what is in the pool)


@pytest.mark.parametrize("size,blocks", [((1 << 32) + 1, 1), (1 << 63, 1), (16, 1 << 31), (16, 1 << 63)])
def test_pools_of_more_than_a_plane_takes(size, blocks):
    layout = P.kvl_page_layout_t(1, 1, (C.c_uint64 * len(P.kvl_page_layout_t().block_bytes))(size), blocks)
    out = C.c_void_p()
    assert P._lib.kvl_page_pools(C.byref(layout), (C.c_void_p * 1)(4096), K.KVL_NO_POINTER_CHECKS, C.byref(out)) == K.KVL_ERANGE
    assert not out.value
