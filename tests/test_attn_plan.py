"""Plans of the attention operators, on the host: what the pieces of work cover, and what is refused."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from paper_2602_21548_amd import attn as A
from oracle import attn_oracle as O

from test_abi import declared_functions

HOST = K.KVL_HOST_ONLY


def layout(**kw):
    base = dict(block_tokens=16, q_heads=8, kv_heads=2, head_dim=128, pool_blocks=4096)
    base.update(kw)
    return K.make_attn_layout(**base)


def tables_for(hit, app, bs, start=0):
    out, at = [], start
    for h, a in zip(hit, app):
        n = (h + a + bs - 1) // bs
        out.append(np.arange(at, at + n, dtype=np.int32))
        at += n
    return out


def plan(hit, app, flags=K.KVL_GATHER | K.KVL_TOKENS_ALL, tables=None, **kw):
    lay = layout(**kw)
    return K.kvl_attn_plan(lay, hit, app, tables_for(hit, app, lay.block_tokens) if tables is None else tables, flags | HOST)


def test_library_exports_what_the_header_declares():
    lib = ctypes.CDLL(K.LIB_PATH)
    for name in declared_functions("kvl_attn.h"):
        assert hasattr(lib, name)
    assert sorted(A.SIGNATURES) == declared_functions("kvl_attn.h")


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(A.kvl_attn_layout_t) == 48
    assert ctypes.sizeof(A.kvl_attn_item_t) == 32
    assert ctypes.sizeof(A.kvl_append_t) == 80
    assert ctypes.sizeof(A.kvl_attn_t) == 64


def test_header_is_plain_c(tmp_path):
    import subprocess
    src = tmp_path / "a.c"
    src.write_text('#include "kvl_attn.h"\nint main(void) { kvl_attn_layout_t l; l.window = 0; return (int)l.window; }\n')
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I" + os.path.join(root, "include"), "-c", str(src),
                        "-o", str(tmp_path / "a.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


# every (row, visible key) is in exactly one piece, and no piece holds a key that none of its rows sees at either end
@pytest.mark.parametrize("keys", ["hit", "append", "all"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 0), (40, 5), (1, 0), (7, 300), (5000, 3)])
@pytest.mark.parametrize("heads,dim,cache", [((8, 2), 128, None), ((7, 1), 64, torch.float8_e4m3fn)])
def test_pieces_cover_each_visible_key_once(keys, window, sinks, heads, dim, cache):
    hit = [0, 1, 37, 500, 2000, 0, 9000]
    app = [1, 0, 3, 70, 1, 300, 2]
    flag = {"hit": 0, "append": K.KVL_TOKENS_APPEND, "all": K.KVL_TOKENS_ALL}[keys]
    p = plan(hit, app, K.KVL_GATHER | flag, q_heads=heads[0], kv_heads=heads[1], head_dim=dim, window=window, sinks=sinks, cache_dtype=cache)
    group = heads[0] // heads[1]
    got = {}
    rows_seen = {}
    for r, row0, rows, begin, end, s, gap, pieces in p.items().tolist():
        assert 1 <= rows <= 128 and begin <= end
        places = np.arange(begin, end)
        tokens = np.where(places < s, places, places + gap)
        got.setdefault((r, row0, rows, pieces), []).append(tokens)
    for (r, row0, rows, pieces), spans in got.items():
        assert len(spans) == pieces
        rows_seen.setdefault(r, []).extend(range(row0, row0 + rows))
        tokens = np.concatenate(spans)
        assert np.unique(tokens).size == tokens.size
        tokens = set(tokens.tolist())
        first, last = {"hit": (0, hit[r]), "append": (hit[r], hit[r] + app[r]), "all": (0, hit[r] + app[r])}[keys]
        want = set()
        for row in range(row0, row0 + rows):
            q = hit[r] + row // group
            want |= {t for t in range(first, min(last, q + 1)) if not window or q - t < window or t < sinks}
        assert want <= tokens
        assert tokens - want == set(), "a key that nobody sees would be read"
    for r, n in enumerate(app):
        assert sorted(rows_seen.get(r, [])) == list(range(n * group))


def test_pieces_of_one_long_request_are_alike_and_many():
    p = plan([131000], [1], q_heads=32, kv_heads=8, block_tokens=64, pool_blocks=4096, cache_dtype=torch.float8_e4m3fn)
    items = p.items()
    n = items[:, 4] - items[:, 3]
    assert items.shape[0] * 8 >= 512 and n[:-1].min() == n.max()
    assert p.workspace_bytes == items.shape[0] * 8 * 16 * 130 * 4


def test_one_piece_wants_no_workspace():
    assert plan([100], [1]).workspace_bytes == 0
    assert plan([], []).workspace_bytes == 0 and plan([], []).tokens == 0


@pytest.mark.parametrize("change", [
    dict(block_tokens=0), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=9), dict(head_dim=96), dict(head_dim=0), dict(rope_dim=24),
    dict(rope_dim=144), dict(rope_pairs=2), dict(q_heads=131072, kv_heads=2)])
def test_layouts_refused(change):
    with pytest.raises(K.KvlError) as e:
        plan([10], [1], tables=[np.arange(64, dtype=np.int32)], **change)
    assert e.value.code == K.KVL_EINVAL


def test_types_refused():
    with pytest.raises(ValueError):
        layout(dtype=torch.float32)
    with pytest.raises(K.KvlError) as e:        # a cache of the other 16-bit type
        plan([10], [1], dtype=torch.bfloat16, cache_dtype=torch.float16)
    assert e.value.code == K.KVL_EINVAL
    with pytest.raises(K.KvlError):             # queries of 8 bits
        plan([10], [1], dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        layout(window=-1)


@pytest.mark.parametrize("flags", [0, K.KVL_TOKENS_ALL, K.KVL_GATHER | K.KVL_TOKENS_ALL | K.KVL_TOKENS_APPEND, K.KVL_GATHER | K.KVL_NO_MERGE, 1 << 20])
def test_flags_refused(flags):
    with pytest.raises(K.KvlError) as e:
        plan([10], [1], flags)
    assert e.value.code == K.KVL_EINVAL


def code_of(*args, **kw):
    with pytest.raises(K.KvlError) as e:
        plan(*args, **kw)
    return e.value.code


def test_tables_refused():
    both = K.KVL_GATHER | K.KVL_SCATTER | K.KVL_TOKENS_ALL
    assert code_of([30], [3], both, tables=[np.array([0, 1], dtype=np.int32)]) == K.KVL_ERANGE           # too short
    assert code_of([30], [3], both, tables=[np.array([0, 1, 4096], dtype=np.int32)]) == K.KVL_ERANGE
    assert code_of([30], [3], both, tables=[np.array([0, -1, 2], dtype=np.int32)]) == K.KVL_ERANGE
    assert code_of([10], [1], both, pool_blocks=1 << 30) == K.KVL_ERANGE
    assert code_of([2 ** 31 - 1], [1], both, tables=[np.zeros(4, dtype=np.int32)]) == K.KVL_ERANGE
    # two requests receive rows in one block; one request's tail names a block twice
    assert code_of([30, 31], [3, 1], both, tables=[np.array([0, 1, 2], dtype=np.int32), np.array([5, 1], dtype=np.int32)]) == K.KVL_EALIAS
    assert code_of([16], [32], both, tables=[np.array([0, 3, 3], dtype=np.int32)]) == K.KVL_EALIAS
    # blocks that are only read may be shared, and plans without KVL_SCATTER receive nothing
    plan([32, 32], [3, 3], both, tables=[np.array([0, 1, 2], dtype=np.int32), np.array([0, 1, 3], dtype=np.int32)])
    plan([30, 31], [3, 1], K.KVL_GATHER | K.KVL_TOKENS_ALL, tables=[np.array([0, 1, 2], dtype=np.int32), np.array([5, 1], dtype=np.int32)])


def test_host_plans_do_not_run():
    p = plan([10], [1], K.KVL_GATHER | K.KVL_SCATTER | K.KVL_TOKENS_ALL)
    none = (ctypes.c_void_p * 4)()
    a, b = A.kvl_append_t(), A.kvl_attn_t(scale=1.0)
    assert A._lib.kvl_append_layer(p.handle, ctypes.byref(a), none, None) == K.KVL_EINVAL
    assert A._lib.kvl_attn_layer(p.handle, ctypes.byref(b), none, None) == K.KVL_EINVAL
    assert A._lib.kvl_attn_layer(None, ctypes.byref(b), none, None) == K.KVL_EINVAL
    assert A._lib.kvl_append_layer(p.handle, None, none, None) == K.KVL_EINVAL
    p.destroy()
    with pytest.raises(ValueError):
        p.items()
    A._lib.kvl_attn_plan_destroy(None)


def test_wrapper_refuses_host_tensors_and_wrong_shapes():
    p = plan([10], [1], K.KVL_GATHER | K.KVL_SCATTER | K.KVL_TOKENS_ALL)
    x = torch.zeros(1, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        K.kvl_attn_layer(p, x, [x, x], x)
    with pytest.raises(ValueError):
        K.kvl_attn_layer(p, x, [x], x)
    with pytest.raises(TypeError):
        A._rows(p, x, p._q_shape, "q")


# the oracle's own pieces, against torch's conversions
def test_oracle_codes():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_values(codes.numpy()), want, equal_nan=True)
    x = torch.cat([torch.randn(2000, generator=torch.Generator().manual_seed(1)) * 10 ** e for e in range(-4, 3)]).double().clamp(-448, 448)
    mid = torch.from_numpy((O.E4M3[1:] + O.E4M3[:-1]) / 2)
    x = torch.cat([x, mid, -mid])
    want = x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    exact = x.double() == x.float().double()
    got = np.array([O.e4m3_code(v) for v in x.tolist()])
    assert np.array_equal(got[exact.numpy()], want[exact.numpy()]) and int(exact.sum()) > 250
    assert O.e4m3_code(float("inf")) == 127 and O.e4m3_code(1e9) == 126 and O.e4m3_code(-1e9) == 254


def test_oracle_scales():
    assert O.least_scale(0.0) == 2.0 ** -32 and O.least_scale(448.0) == 1.0 and O.least_scale(np.nextafter(448.0, 500)) == 2.0
    assert O.least_scale(1e300) == 2.0 ** 63


def test_oracle_attention_is_softmax():
    g = np.random.default_rng(3)
    k, v, q = g.standard_normal((4, 8, 1, 16)), g.standard_normal((4, 8, 1, 16)), g.standard_normal((5, 2, 16))
    table = np.array([2, 0, 3], dtype=np.int32)
    out, lse, _, _ = O.attend([13], [5], [table], 8, q, k, v, 0.3)
    kk, vv = k[table].reshape(24, 16)[:18], v[table].reshape(24, 16)[:18]
    s = torch.from_numpy(0.3 * np.einsum("thd,sd->hts", q, kk))
    mask = torch.arange(18)[None, :] > 13 + torch.arange(5)[:, None]
    s = s.masked_fill(mask, -float("inf"))
    want = (torch.softmax(s, -1) @ torch.from_numpy(vv)).permute(1, 0, 2).numpy()
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, torch.logsumexp(s, -1).T.numpy(), atol=1e-12)
