"""Copies of a cache's blocks on the GPU, bit for bit, and forks that are appended to and attended over."""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K

pytestmark = pytest.mark.gpu


def pool(layers, blocks, sizes, seed=0, shift=0):
    """[layers][planes] of uint8, each plane `shift` bytes behind an allocation's begin."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [[torch.randint(0, 256, (blocks * b + shift,), dtype=torch.uint8, device="cuda", generator=g)[shift:] for b in sizes] for _ in range(layers)]


def check(layers, blocks, sizes, copies, shift=0, **kw):
    planes = pool(layers, blocks, sizes, shift=shift)
    want = [[t.clone().view(blocks, -1) for t in layer] for layer in planes]
    for layer in want:
        for t in layer:
            if len(copies):
                c = torch.from_numpy(np.asarray(copies, dtype=np.int64)).cuda()
                t[c[:, 1]] = t[c[:, 0]]
    torch.cuda.synchronize()
    K.kvl_copy_blocks(K.kvl_page_pools(sizes, blocks, planes), copies, **kw)
    torch.cuda.synchronize()
    for a, b in zip(planes, want):
        for x, y in zip(a, b):
            assert torch.equal(x.view(blocks, -1), y)


@pytest.mark.parametrize("sizes", [[16], [1], [3], [4, 32], [4096, 4096, 32, 32], [4112], [656 * 64], [73728], [8192 + 16, 4, 5, 12]])
@pytest.mark.parametrize("layers", [1, 3])
def test_sizes(sizes, layers):
    check(layers, 9, sizes, [[0, 8], [0, 1], [5, 2]])


@pytest.mark.parametrize("shift", [1, 4, 8, 16])
@pytest.mark.parametrize("size", [4096, 36, 7])
def test_planes_that_begin_anywhere(size, shift):
    check(2, 6, [size, 64], [[1, 0], [4, 5]], shift=shift)


@pytest.mark.parametrize("n", [0, 1, 23, 24, 25, 319, 320, 321, 1000])
def test_numbers_of_copies(n):
    """Around what one launch takes."""
    order = np.random.default_rng(n).permutation(2100)
    check(2, 2100, [144, 4], np.stack([order[:n], order[1000:1000 + n]], 1).astype(np.int32))


@pytest.mark.parametrize("sizes,layers", [([65536, 65536, 32, 32], 2), ([1040], 1), ([9 << 20, 12, 5], 1)])
def test_one_block_to_many(sizes, layers):
    """More and fewer than share a workgroup, in lists that one launch does not take, of little and of much."""
    order = np.random.default_rng(4).permutation(500)
    blocks = 500 if max(sizes) < 1 << 20 else 40
    order = order[order < blocks] if blocks < 500 else order
    ways = [1, 8, 9, 7, 2] if blocks < 500 else [200, 1, 1, 7, 8, 9, 17, 40, 2]
    frm = np.repeat(order[:len(ways)], ways)
    check(layers, blocks, sizes, np.stack([frm, order[len(ways):len(ways) + len(frm)]], 1).astype(np.int32))


def test_more_than_the_caches_hold():
    check(3, 300, [1 << 20], np.stack([np.repeat(np.arange(50), 2), np.arange(100, 200)], 1).astype(np.int32))


def test_one_block_to_many_and_lists_of_numbers():
    check(2, 50, [528], [[7, b] for b in range(50) if b != 7])
    check(1, 50, [528], np.array([[7, 3]], dtype=np.int64))


def test_blocks_beyond_32_bits():
    """A pool of more than 4 GB."""
    blocks, size = 70000, 65536
    plane = torch.zeros(blocks * size, dtype=torch.uint8, device="cuda")
    rows = plane.view(blocks, size)
    rows[69999] = torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda")
    rows[3] = 9
    K.kvl_copy_blocks(K.kvl_page_pools([size], blocks, [[plane]]), [[69999, 66000], [3, 69998]])
    assert torch.equal(rows[66000], rows[69999]) and bool((rows[69998] == 9).all()) and not rows[65999].any() and not rows[66001].any()


def test_other_streams_and_a_handle_dropped_at_once():
    planes = pool(4, 64, [65536])
    want = [[t.clone().view(64, -1) for t in layer] for layer in planes]
    for layer in want:
        layer[0][32:] = layer[0][:32]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        pools = K.kvl_page_pools([65536], 64, planes)
        K.kvl_copy_blocks(pools, [[b, b + 32] for b in range(32)], stream=stream)
        pools.destroy()
    side.synchronize()
    for a, b in zip(planes, want):
        assert torch.equal(a[0].view(64, -1), b[0])


def test_captured_and_replayed():
    planes = pool(3, 40, [4096, 32])
    pools = K.kvl_page_pools([4096, 32], 40, planes)
    K.kvl_copy_blocks(pools, [[0, 39]])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.kvl_copy_blocks(pools, [[0, 20], [1, 21]])
    for k in range(4):
        for layer in planes:
            for t in layer:
                t.random_(0, 256)
        want = [[t.clone() for t in layer] for layer in planes]
        for layer in want:
            for t in layer:
                t.view(40, -1)[20:22] = t.view(40, -1)[:2]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(planes, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    del graph


def test_refusals():
    planes = pool(2, 10, [64, 32])
    pools = K.kvl_page_pools([64, 32], 10, planes)
    before = [[t.clone() for t in layer] for layer in planes]
    for copies, code in [([[0, 10]], K.KVL_ERANGE), ([[10, 0]], K.KVL_ERANGE), ([[-1, 0]], K.KVL_ERANGE), ([[0, -1]], K.KVL_ERANGE), ([[0, 1], [2, 1]], K.KVL_EALIAS),
                         ([[0, 1], [1, 2]], K.KVL_EALIAS), ([[1, 2], [0, 1]], K.KVL_EALIAS), ([[4, 4]], K.KVL_EALIAS)]:
        with pytest.raises(K.KvlError) as e:
            K.kvl_copy_blocks(pools, copies)
        assert e.value.code == code
    for copies in ([1, 2], [[1, 2, 3]], [[0.5, 1]], [[0, 1 << 31]]):
        with pytest.raises(ValueError):
            K.kvl_copy_blocks(pools, copies)
    for args in (([64], 10, planes), ([64, 33], 10, planes), ([64, 32], 11, planes), ([64, 32], 10, [planes[0], planes[1][:1]]), ([], 10, []), ([64, -1], 10, planes)):
        with pytest.raises(ValueError):
            K.kvl_page_pools(*args)
    with pytest.raises(TypeError):
        K.kvl_page_pools([64, 32], 10, [planes[0], [t.cpu() for t in planes[1]]])
    for sizes, n, code in (([0, 32], 10, K.KVL_EINVAL), ([64, 32], 0, K.KVL_EINVAL)):
        with pytest.raises(K.KvlError) as e:
            K.kvl_page_pools(sizes, n, planes)
        assert e.value.code == code
    with pytest.raises(K.KvlError):
        K.kvl_page_pools([64], 10, [])
    with pytest.raises(K.KvlError):
        K.kvl_page_pools([64], 10, [[planes[0][0]]], flags=K.KVL_GATHER)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(planes, before) for x, y in zip(a, b))
    pools.destroy()
    with pytest.raises(ValueError):
        K.kvl_copy_blocks(pools, [[0, 1]])


@pytest.mark.parametrize("e4m3", [False, True])
def test_forks_are_sequences_of_their_own(e4m3):
    """A prompt is loaded, forked, each fork is appended to and attended over, then the pool is compacted: every result is that of a cache that each
    sequence has for itself."""
    bs, q_heads, kv, d, blocks, layers, hit, forks, steps = 16, 4, 2, 64, 40, 2, 37, 3, 12
    dtype = torch.bfloat16
    layout = K.make_attn_layout(bs, q_heads, kv, d, blocks, dtype, torch.float8_e4m3fn if e4m3 else dtype)
    sizes = [bs * kv * d, bs * kv * d, 4 * kv, 4 * kv] if e4m3 else [2 * bs * kv * d] * 2

    def planes():
        if e4m3:
            return [torch.zeros(blocks, bs, kv, d, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros(blocks, kv, device="cuda") for _ in range(2)]
        return [torch.zeros(blocks, bs, kv, d, dtype=dtype, device="cuda") for _ in range(2)]

    def step(pool, tables, before, n, x):
        """x: [sequences * n, heads, d] of each layer; what attention gives."""
        plan = K.kvl_attn_plan(layout, before, [n] * len(tables), tables, K.KVL_SCATTER | K.KVL_GATHER | K.KVL_TOKENS_ALL)
        ws = torch.empty(max(256, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
        outs = []
        for layer in range(layers):
            q, k, v = x[layer].split([q_heads, kv, kv], dim=1)
            K.kvl_append_layer(plan, k, v, pool[layer])
            out = torch.zeros(x[layer].shape[0], q_heads, d, dtype=dtype, device="cuda")
            K.kvl_attn_layer(plan, q, pool[layer], out, ws)
            outs.append(out)
        return outs

    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    new = lambda n: [torch.randn(n, q_heads + 2 * kv, d, device="cuda", generator=g).to(dtype) for _ in range(layers)]  # noqa: E731
    shared = [planes() for _ in range(layers)]
    own = [[planes() for _ in range(layers)] for _ in range(forks + 1)]
    own_table = np.arange(8, dtype=np.int32)
    pools, pages = K.kvl_page_pools(sizes, blocks, shared), K.kvl_pages(bs, blocks)
    s = K.kvl_pages_adopt(pages, [np.array([30, 4, 17], dtype=np.int32)], [hit])
    prompt = new(hit)
    step(shared, K.kvl_pages_tables(pages, s), [0], hit, prompt)
    for mine in own:
        step(mine, [own_table], [0], hit, prompt)
    s = np.concatenate([s, K.kvl_pages_fork(pages, np.repeat(s, forks))])
    assert K.kvl_pages_stats(pages)["used_blocks"] == 3
    for i in range(steps):
        before = K.kvl_pages_tokens(pages, s)
        K.kvl_copy_blocks(pools, K.kvl_pages_extend(pages, s, 1))
        if i == 7:
            K.kvl_copy_blocks(pools, K.kvl_pages_compact(pages))
            assert K.kvl_pages_stats(pages)["moves"] == 0
        x = new(forks + 1)
        got = step(shared, K.kvl_pages_tables(pages, s), before, 1, x)
        for f, mine in enumerate(own):
            want = step(mine, [own_table], [before[f]], 1, [t[f:f + 1] for t in x])
            for a, b in zip(got, want):
                assert torch.equal(a[f:f + 1], b)
    assert K.kvl_pages_stats(pages)["used_blocks"] == 2 + (forks + 1) * 2      # (two full blocks in common)
    K.kvl_pages_free(pages, s)
    assert K.kvl_pages_stats(pages)["free_blocks"] == blocks
