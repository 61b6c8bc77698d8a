"""Plans with prefixes and documents, on the host: the tokens that their pieces of work name, and what they refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from oracle import attn_oracle as O
from paper_2602_21548_amd import attn as A


def plan(hit, app, bs=16, heads=(8, 2), flags=K.KVL_GATHER | K.KVL_TOKENS_ALL, window=0, sinks=0, **masks):
    need = [(h + a + bs - 1) // bs for h, a in zip(hit, app)]
    at = np.cumsum([0] + need)
    tables = [np.arange(a, b, dtype=np.int32) for a, b in zip(at[:-1], at[1:])]
    layout = K.make_attn_layout(bs, *heads, 64, int(at[-1]) + 1, torch.bfloat16, window=window, sinks=sinks)
    return K.kvl_attn_plan(layout, hit, app, tables, flags | K.KVL_HOST_ONLY, **masks)


def tokens_of(items, request, row):
    """The tokens that the pieces with this row of a request name."""
    out = []
    for r, first, n, begin, end, sinks, gap, _ in items.tolist():
        if r == request and first <= row < first + n:
            out += [v if v < sinks else v + gap for v in range(begin, end)]
    return out


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("keys", ["all", "hit", "append"])
def test_pieces_name_what_their_rows_see(seed, keys):
    g = np.random.default_rng(seed)
    n = int(g.integers(1, 5))
    hit, app = g.integers(0, 300, size=n), g.integers(0, 90, size=n)
    total = hit + app
    prefix = [int(g.integers(0, t + 9)) for t in total] if seed % 3 else None
    documents = [np.unique(g.integers(0, t + 9, size=int(g.integers(0, 6)))) for t in total] if seed % 4 else None
    window, sinks = (int(g.integers(1, 80)), int(g.integers(0, 9))) if seed % 2 else (0, int(g.integers(0, 9)))
    group = 4
    p = plan(hit, app, bs=int(g.integers(1, 40)), window=window, sinks=sinks, prefix=prefix, documents=documents,
             flags=K.KVL_GATHER | {"all": K.KVL_TOKENS_ALL, "hit": 0, "append": K.KVL_TOKENS_APPEND}[keys])
    items = p.items()
    for r in range(n):
        h, a = int(hit[r]), int(app[r])
        first, last = {"all": (0, h + a), "hit": (0, h), "append": (h, h + a)}[keys]
        mask = dict(window=window, sinks=sinks, prefix=0 if prefix is None else prefix[r], starts=() if documents is None else documents[r].tolist())
        for i in range(a):
            named = tokens_of(items, r, i * group)
            assert len(set(named)) == len(named)
            assert {t for t in range(first, last) if O.sees(h + i, t, **mask)} <= set(named) <= set(range(first, last))


def test_one_document_or_prefix_of_nothing_changes_no_list():
    hit, app = [100, 5], [20, 70]
    a, b = plan(hit, app), plan(hit, app, prefix=[0, 0], documents=[[], [0]])
    assert np.array_equal(a.items(), b.items()) and a.workspace_bytes == b.workspace_bytes


def test_documents_leave_out_what_is_before_them():
    """The last of three documents: its query's pieces name its own tokens (and the prefix's)."""
    p = plan([1000], [1], prefix=[10], documents=[[50, 300, 900]])
    assert sorted(tokens_of(p.items(), 0, 0)) == [*range(10), *range(900, 1001)]
    p = plan([1000], [1], documents=[[1000]])
    assert tokens_of(p.items(), 0, 0) == [1000]
    p = plan([1000], [1], documents=[[1001, 4000000000]])
    assert tokens_of(p.items(), 0, 0) == list(range(1001))


def test_a_prefix_beyond_the_batch_is_all_of_it():
    p = plan([3], [40], prefix=[(1 << 32) - 1])
    for row in range(160):
        assert sorted(tokens_of(p.items(), 0, row)) == list(range(43))


@pytest.mark.parametrize("starts", [[5, 5], [9, 3], [0, 7, 7]])
def test_starts_that_do_not_ascend_are_refused(starts):
    with pytest.raises(K.KvlError) as e:
        plan([20], [3], documents=[starts])
    assert e.value.code == K.KVL_EINVAL


def test_arguments_that_are_no_masks():
    for bad in (dict(prefix=[1]), dict(prefix=[1, -1]), dict(prefix=[1, 1 << 32]), dict(prefix=[0.5, 1.0]), dict(prefix=3), dict(documents=[[0]]),
                dict(documents=[[0], [-1]]), dict(documents=[[0], [[1]]]), dict(documents=[[0], [0.5]])):
        with pytest.raises(ValueError):
            plan([20, 4], [3, 4], **bad)


def test_the_librarys_own_refusals():
    layout = K.make_attn_layout(16, 4, 2, 64, 8, torch.bfloat16)
    table = np.arange(2, dtype=np.int32)
    req = (A._b.kvl_request_t * 1)()
    req[0].hit_tokens, req[0].append_tokens, req[0].n_blocks = 20, 2, 2
    req[0].block_table = table.ctypes.data_as(C.POINTER(C.c_int32))
    mask, out = (A.kvl_attn_mask_t * 1)(), C.c_void_p()
    mask[0].n_documents = 1                     # (and no array)
    flags = K.KVL_GATHER | K.KVL_HOST_ONLY
    assert A._lib.kvl_attn_plan_masked(C.byref(layout), req, mask, 1, flags, C.byref(out)) == K.KVL_EINVAL and not out.value
    assert A._lib.kvl_attn_plan_masked(C.byref(layout), req, None, 1, flags, C.byref(out)) == K.KVL_OK and out.value
    A._lib.kvl_attn_plan_destroy(out)
    assert A._lib.kvl_attn_plan_masked(C.byref(layout), None, mask, 1, flags, C.byref(out)) == K.KVL_EINVAL


def test_struct_sizes_match_the_header():
    assert C.sizeof(A.kvl_attn_mask_t) == 16 and C.sizeof(A.kvl_attn_scores_t) == 16 and C.sizeof(A.kvl_attn_join_t) == 56
