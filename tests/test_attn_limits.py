"""What the attention operators' plans refuse for its size, and what they take (host only)."""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K

HOST = K.KVL_HOST_ONLY


def plan(hit, app, tables, flags, **kw):
    return K.kvl_attn_plan(K.make_attn_layout(**{**dict(q_heads=16, kv_heads=16, head_dim=64), **kw}), hit, app, tables, flags | HOST)


def refused(*args, **kw):
    with pytest.raises(K.KvlError) as e:
        plan(*args, **kw)
    assert e.value.code == K.KVL_ERANGE


def test_receiving_blocks():
    """One workgroup for each of them and head over an 8-bit cache; 16-bit caches know no such limit."""
    n = (1 << 19) + 1                           # times 16 heads: just above 2^23
    table = [np.arange(n, dtype=np.int32)]
    kw = dict(block_tokens=1, pool_blocks=n)
    assert plan([0], [n], table, K.KVL_SCATTER, **kw).tokens == n
    refused([0], [n], table, K.KVL_SCATTER, cache_dtype=torch.float8_e4m3fn, **kw)
    plan([1], [n - 1], table, K.KVL_SCATTER, cache_dtype=torch.float8_e4m3fn, **kw)
    with pytest.raises(K.KvlError) as e:        # (blocks named twice are found without the list, too)
        plan([0], [n], [np.concatenate([table[0][:-1], table[0][:1]])], K.KVL_SCATTER, **kw)
    assert e.value.code == K.KVL_EALIAS


def test_pieces_of_attention():
    """2^24 pieces times heads: a request of one new token each, its table an empty prefix's one block."""
    n = 1 << 20
    one = np.zeros(1, dtype=np.int32)
    kw = dict(block_tokens=1, pool_blocks=1)
    refused([0] * n, [1] * n, [one] * n, K.KVL_GATHER | K.KVL_TOKENS_ALL, **kw)
    assert plan([0] * (n - 1), [1] * (n - 1), [one] * (n - 1), K.KVL_GATHER | K.KVL_TOKENS_ALL, **kw).tokens == n - 1


def test_rows_of_an_8_bit_block():
    """The kernel numbers a block's pieces of rows, up to eight each, in 32 bits."""
    kw = dict(block_tokens=1 << 30, pool_blocks=3, kv_heads=1, q_heads=1, head_dim=128)
    table = [np.array([2], dtype=np.int32)]
    e4m3 = dict(cache_dtype=torch.float8_e4m3fn)
    assert plan([(1 << 28) - 2], [2], table, K.KVL_SCATTER, **kw, **e4m3).tokens == 2
    refused([(1 << 28) - 1], [2], table, K.KVL_SCATTER, **kw, **e4m3)
    refused([(1 << 29) + 7], [1], table, K.KVL_SCATTER, **kw, **e4m3)
    assert plan([(1 << 29) + 7], [1], table, K.KVL_SCATTER, **kw).tokens == 1
    assert plan([(1 << 29) + 7], [1], table, K.KVL_GATHER | K.KVL_TOKENS_ALL, **kw, **e4m3).tokens == 1
