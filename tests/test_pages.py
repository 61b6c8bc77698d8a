"""Whose the blocks of a cache are: the library against a plain model of it, and what it refuses (host only)."""
import ctypes as C
import random
import subprocess

import numpy as np
import pytest

import paper_2602_21548_amd as K
from paper_2602_21548_amd import pages as P


class Model:
    """Sets and lists: the lowest free block first, counted by looking at every table."""

    def __init__(self, bs, blocks):
        self.bs, self.blocks, self.tables, self.tokens, self.next = bs, blocks, {}, {}, 0

    def users(self, b):
        return sum(b in t for t in self.tables.values())

    def free(self):
        used = {b for t in self.tables.values() for b in t}
        return [b for b in range(self.blocks) if b not in used]

    def put(self, table, tokens):
        self.next += 1
        self.tables[self.next], self.tokens[self.next] = list(table), tokens
        return self.next

    def extend(self, names, tokens):
        """The copies, or None where blocks do not suffice (and nothing changes)."""
        before = {k: list(t) for k, t in self.tables.items()}, dict(self.tokens)
        copies = []
        for s, n in zip(names, tokens):
            t = self.tables[s]
            want = -(-(self.tokens[s] + n) // self.bs)
            shared = n and self.tokens[s] % self.bs and self.users(t[-1]) > 1
            free = self.free()
            if len(free) < want - len(t) + bool(shared):
                self.tables, self.tokens = before
                return None
            if shared:
                copies.append([t[-1], free[0]])
                t[-1] = free.pop(0)
            t += free[:want - len(t)]
            self.tokens[s] += n
        return copies

    def keep(self, s, n):
        self.tokens[s] = n
        del self.tables[s][-(-n // self.bs):]

    def compact(self, most):
        copies = []
        while len(copies) < most:
            used = sorted({b for t in self.tables.values() for b in t})
            free = self.free()
            if not used or not free or free[0] > used[-1]:
                break
            a, b = used[-1], free[0]
            copies.append([a, b])
            for t in self.tables.values():
                t[:] = [b if x == a else x for x in t]
        return copies


@pytest.mark.parametrize("seed", range(20))
def test_against_the_model(seed):
    rng = random.Random(seed)
    bs, blocks = rng.choice([1, 2, 5, 16]), rng.choice([1, 7, 63, 64, 65, 130, 300])
    pages, model, name = K.kvl_pages(bs, blocks), Model(bs, blocks), {}
    some = lambda: rng.sample(sorted(name), rng.randint(0, len(name)))  # noqa: E731
    refused = 0
    for _ in range(120):
        what = rng.choice(["new", "adopt", "fork", "extend", "extend", "extend", "truncate", "free", "compact"])
        if what == "new":
            for x in K.kvl_pages_adopt(pages, [np.zeros(0, np.int32)] * 2, 0):
                name[int(x)] = model.put([], 0)
        elif what == "adopt":
            n = rng.randint(0, blocks * bs)
            table = rng.sample(range(blocks), -(-n // bs)) + [blocks + 5] * rng.randint(0, 2)
            x = K.kvl_pages_adopt(pages, [np.array(table, dtype=np.int32)], [n])
            name[int(x[0])] = model.put(table[:-(-n // bs)], n)
        elif what == "fork" and name:
            s = [rng.choice(sorted(name)) for _ in range(rng.randint(0, 3))]
            for a, x in zip(s, K.kvl_pages_fork(pages, s)):
                name[int(x)] = model.put(model.tables[name[a]], model.tokens[name[a]])
        elif what == "extend":
            s = some()
            tokens = [rng.choice([0, 1, 1, 2, bs, 3 * bs]) for _ in s]
            want = model.extend([name[a] for a in s], tokens)
            if want is None:
                refused += 1
                with pytest.raises(K.KvlError) as e:
                    K.kvl_pages_extend(pages, s, tokens)
                assert e.value.code == K.KVL_ESPACE
            else:
                assert K.kvl_pages_extend(pages, s, tokens).tolist() == want
        elif what == "truncate":
            s = some()
            tokens = [rng.randint(0, model.tokens[name[a]]) for a in s]
            K.kvl_pages_truncate(pages, s, tokens)
            for a, n in zip(s, tokens):
                model.keep(name[a], n)
        elif what == "free":
            s = some()[:3]
            K.kvl_pages_free(pages, s)
            for a in s:
                model.tables.pop(name[a])
                model.tokens.pop(name.pop(a))
        elif what == "compact":
            most = rng.choice([None, 0, 1, 3, 1000])
            assert K.kvl_pages_compact(pages, most).tolist() == model.compact(10 ** 9 if most is None else most)
        s = sorted(name)
        assert [t.tolist() for t in K.kvl_pages_tables(pages, s)] == [model.tables[name[a]] for a in s]
        assert K.kvl_pages_tokens(pages, s).tolist() == [model.tokens[name[a]] for a in s]
        free, used = model.free(), {b for t in model.tables.values() for b in t}
        assert K.kvl_pages_stats(pages) == dict(free_blocks=len(free), used_blocks=len(used), shared_blocks=sum(model.users(b) > 1 for b in used),
                                                moves=sum(b >= len(used) for b in used), sequences=len(name))


def test_forks_that_grow_together_leave_one_the_block():
    pages = K.kvl_pages(16, 8)
    s = K.kvl_pages_adopt(pages, [np.array([3], dtype=np.int32)], [10])
    f = K.kvl_pages_fork(pages, [s[0], s[0]])
    assert K.kvl_pages_extend(pages, [*f, s[0]], 1).tolist() == [[3, 0], [3, 1]]        # the last one keeps it
    assert [t.tolist() for t in K.kvl_pages_tables(pages, [*s, *f])] == [[3], [0], [1]]
    # a full block stays shared
    t = K.kvl_pages_adopt(pages, [np.array([5], dtype=np.int32)], [16])
    g = K.kvl_pages_fork(pages, t)
    assert K.kvl_pages_extend(pages, g, 1).size == 0
    assert K.kvl_pages_tables(pages, g)[0].tolist() == [5, 2]


def test_numbers_are_not_used_again():
    pages = K.kvl_pages(16, 8)
    seen = set()
    for _ in range(100):
        s = K.kvl_pages_adopt(pages, [np.array([1], dtype=np.int32)], 16)
        assert int(s[0]) not in seen
        seen.add(int(s[0]))
        K.kvl_pages_free(pages, s)
        for call in (lambda: K.kvl_pages_free(pages, s), lambda: K.kvl_pages_fork(pages, s), lambda: K.kvl_pages_extend(pages, s, 1),
                     lambda: K.kvl_pages_truncate(pages, s, 0), lambda: K.kvl_pages_tables(pages, s), lambda: K.kvl_pages_tokens(pages, s)):
            with pytest.raises(K.KvlError) as e:
                call()
            assert e.value.code == K.KVL_EINVAL


def test_refusals_change_nothing():
    pages = K.kvl_pages(16, 8)
    s = K.kvl_pages_adopt(pages, [np.array([1, 2], dtype=np.int32), np.array([4], dtype=np.int32)], [20, 3])
    before = [t.tolist() for t in K.kvl_pages_tables(pages, s)], K.kvl_pages_stats(pages)
    i32 = lambda *x: np.array(x, dtype=np.int32)  # noqa: E731
    for code, call in [
        (K.KVL_EINVAL, lambda: K.kvl_pages_extend(pages, [s[0], s[1], s[0]], 1)), (K.KVL_EINVAL, lambda: K.kvl_pages_free(pages, [s[1], s[1]])),
        (K.KVL_EINVAL, lambda: K.kvl_pages_truncate(pages, [s[1], s[1]], 0)), (K.KVL_EINVAL, lambda: K.kvl_pages_free(pages, [s[0], 0])),
        (K.KVL_EINVAL, lambda: K.kvl_pages_fork(pages, [s[0], (1 << 64) - 1])), (K.KVL_EINVAL, lambda: K.kvl_pages_tables(pages, [s[0], 77])),
        (K.KVL_ERANGE, lambda: K.kvl_pages_truncate(pages, s, [0, 4])), (K.KVL_ERANGE, lambda: K.kvl_pages_extend(pages, s, [1, (1 << 31) - 3])),
        (K.KVL_ESPACE, lambda: K.kvl_pages_extend(pages, s, [1, 14 + 16 * 5])), (K.KVL_ESPACE, lambda: K.kvl_pages_extend(pages, s, [(1 << 31) - 21, 0])),
        (K.KVL_ERANGE, lambda: K.kvl_pages_adopt(pages, [i32(0), i32(8)], [1, 1])), (K.KVL_ERANGE, lambda: K.kvl_pages_adopt(pages, [i32(0), i32(-1)], [1, 1])),
        (K.KVL_ERANGE, lambda: K.kvl_pages_adopt(pages, [i32(0), i32(3)], [1, 17])), (K.KVL_EALIAS, lambda: K.kvl_pages_adopt(pages, [i32(0), i32(3, 3)], [1, 17])),
        (K.KVL_ERANGE, lambda: K.kvl_pages_adopt(pages, [i32(0)], [1 << 31])),
    ]:
        with pytest.raises(K.KvlError) as e:
            call()
        assert e.value.code == code
        assert ([t.tolist() for t in K.kvl_pages_tables(pages, s)], K.kvl_pages_stats(pages)) == before
    for call in (lambda: K.kvl_pages_extend(pages, s, [1]), lambda: K.kvl_pages_extend(pages, s, -1), lambda: K.kvl_pages_extend(pages, [0.5], 1),
                 lambda: K.kvl_pages_extend(pages, s, 1 << 32), lambda: K.kvl_pages_fork(pages, [-1]), lambda: K.kvl_pages_compact(pages, -1), lambda: K.kvl_pages(-1, 8),
                 lambda: K.kvl_pages(1 << 32, 8)):
        with pytest.raises(ValueError):
            call()
    for bs, n, code in ((0, 8, K.KVL_EINVAL), (16, 0, K.KVL_EINVAL), (16, 1 << 31, K.KVL_ERANGE)):
        with pytest.raises(K.KvlError) as e:
            K.kvl_pages(bs, n)
        assert e.value.code == code
    assert K.kvl_pages_tables(pages, []) == [] and K.kvl_pages_extend(pages, [], []).shape == (0, 2)
    pages.destroy()
    pages.destroy()
    with pytest.raises(ValueError):
        K.kvl_pages_stats(pages)


def test_too_few_free_blocks_for_copies_alone():
    """All blocks in use, a shared one among them: a token that would need a copy is refused, one that fits its own block is not."""
    pages = K.kvl_pages(4, 2)
    s = K.kvl_pages_adopt(pages, [np.array([0], dtype=np.int32), np.array([1], dtype=np.int32)], [2, 2])
    f = K.kvl_pages_fork(pages, [s[0]])
    with pytest.raises(K.KvlError) as e:
        K.kvl_pages_extend(pages, f, 1)
    assert e.value.code == K.KVL_ESPACE
    assert K.kvl_pages_extend(pages, [s[1]], 2).size == 0
    assert K.kvl_pages_extend(pages, f, 0).size == 0
    K.kvl_pages_free(pages, [s[0]])
    assert K.kvl_pages_extend(pages, f, 2).size == 0            # (it is the block's last user now)


def test_a_large_pool():
    """Three levels of words, the last ones not full."""
    n = 64 * 64 * 3 + 65
    pages = K.kvl_pages(1, n)
    s = K.kvl_pages_adopt(pages, [np.zeros(0, np.int32)] * 2, 0)
    K.kvl_pages_extend(pages, s, [n - 1, 1])
    a, b = K.kvl_pages_tables(pages, s)
    assert np.array_equal(a, np.arange(n - 1)) and b.tolist() == [n - 1]
    with pytest.raises(K.KvlError):
        K.kvl_pages_extend(pages, s[1:], 1)
    K.kvl_pages_truncate(pages, s[:1], 5000)
    K.kvl_pages_extend(pages, s[1:], 2)
    assert K.kvl_pages_tables(pages, s[1:])[0].tolist() == [n - 1, 5000, 5001]
    assert K.kvl_pages_compact(pages).tolist() == [[n - 1, 5002]]


def test_binding_and_header_agree(tmp_path):
    from test_abi import declared_functions
    lib = C.CDLL(K.LIB_PATH)
    for name in declared_functions("kvl_pages.h"):
        assert hasattr(lib, name)
    assert sorted(P.SIGNATURES) == declared_functions("kvl_pages.h")
    assert C.sizeof(P.kvl_block_copy_t) == 8 and C.sizeof(P.kvl_page_layout_t) == 48 and C.sizeof(P.kvl_pages_stats_t) == 40
    src = tmp_path / "c.c"
    src.write_text('#include "kvl_pages.h"\nint main(void) { kvl_block_copy_t c = {0, 1}; return c.from; }\n')
    import os
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(K.__file__))), "include")
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I" + include, str(src), "-o", str(tmp_path / "c")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("dtype", [np.int64, np.uint64, np.int32, np.uint16, ">i8"])
def test_numbers_of_any_integer_type(dtype):
    """And at any stride; what does not fit is refused, whichever form it has."""
    pages = K.kvl_pages(4, 64)
    s = K.kvl_pages_adopt(pages, [np.zeros(0, np.int32)] * 6, 0)
    some = np.zeros(6, dtype=dtype)
    some[::2] = s[:3]
    K.kvl_pages_extend(pages, some[::2], np.array([5, 0, 9], dtype=dtype))
    assert K.kvl_pages_tokens(pages, s.astype(dtype)).tolist() == [5, 0, 9, 0, 0, 0]
    K.kvl_pages_truncate(pages, some[::2], np.array([1, 0, 8], dtype=dtype))
    assert K.kvl_pages_tokens(pages, s[:3]).tolist() == [1, 0, 8]
    for bad in (np.array([-1], dtype=np.int64), np.array([1 << 32], dtype=np.uint64), np.array([[1]]), np.array([1.0])):
        with pytest.raises(ValueError):
            K.kvl_pages_extend(pages, s[:1], bad)


def test_a_long_pool_of_which_little_moves():
    n = 100_000
    pages = K.kvl_pages(1, n)
    s = K.kvl_pages_adopt(pages, [np.array([n - 1, 3, n - 7], dtype=np.int32)], [3])
    assert K.kvl_pages_compact(pages, 1).tolist() == [[n - 1, 0]]
    copies = K.kvl_pages_compact(pages)
    assert copies.tolist() == [[n - 7, 1], [3, 2]] and copies.base is None
    assert K.kvl_pages_tables(pages, s)[0].tolist() == [0, 2, 1]
    assert K.kvl_pages_compact(pages).shape == (0, 2) and K.kvl_pages_compact(K.kvl_pages(1, 1)).shape == (0, 2)
