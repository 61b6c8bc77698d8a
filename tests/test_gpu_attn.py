"""The attention operators on the GPU against the oracle's 64 bits.

Whatever no query may see is NaN in every test: blocks of the pool that no table names, rows behind a request's last token,
keys outside the plan's range, and the scales of unnamed blocks.

Tolerances.  A rounding to the type T moves a value by at most u = eps(T) / 2 of it.  Outputs: the softmax weights are rounded to T
(u * sum p |V|) and the result once more (u * |out|).  Scores are sums of head_dim exact products in 32 bits, their argument of
the exponential a few operations more: off by at most ds = (head_dim + 16) * 2^-24 * scale * max sum |q K|, with the exponential's own 2^-20;
weights and their sum by twice that each.  Sums over n keys in 32 bits add n * 2^-24.
"""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from oracle import attn_oracle as O

pytestmark = pytest.mark.gpu

NAN = float("nan")


def unit(dtype):
    return torch.finfo(dtype).eps / 2


class Batch:
    """A batch with its pool on both sides: doubles (or codes and scales) for the oracle, device planes for the library."""

    def __init__(self, hit, app, bs, heads, dim, dtype=torch.bfloat16, e4m3=False, keys="all", seed=1, window=0, sinks=0, rope_dim=0, pairs="halves",
                 powers=True, spread=1.0, extra=3, tables=None, flags=0, hold=None):
        g = self.g = np.random.default_rng(seed)
        self.hit, self.app, self.bs, self.keys = hit, app, bs, keys
        self.q_heads, self.kv_heads = heads
        self.dim, self.dtype, self.e4m3 = dim, dtype, e4m3
        self.window, self.sinks, self.pairs, self.rope_dim = window, sinks, pairs, rope_dim
        need = [(h + a + bs - 1) // bs for h, a in zip(hit, app)]
        self.blocks = sum(need) + extra
        order = g.permutation(self.blocks).astype(np.int32)
        at = np.cumsum([0] + need)
        self.tables = [order[a:b].copy() for a, b in zip(at[:-1], at[1:])] if tables is None else tables
        self.tokens = sum(app)
        shape = (self.blocks, bs, self.kv_heads, dim)
        # what the cache holds: `hold` says which tokens, [0, hit) where the new ones are still to be appended
        self.pools, self.scales = [], []
        held = np.zeros((self.blocks, bs), dtype=bool)
        for h, a, t in zip(hit, app, self.tables):
            first, last = {"hit": (0, h), "append": (h, h + a), "all": (0, h + a)}[hold or keys]
            for x in range(first, last):
                held[t[x // bs], x % bs] = True
        self.held = held
        for x in range(2):
            values = g.standard_normal(shape) * spread
            if e4m3:
                scale = np.full((self.blocks, self.kv_heads), NAN, dtype=np.float32)
                codes = np.full(shape, 0x7F, dtype=np.uint8)
                used = np.nonzero(held.any(1))[0]
                for b in used:
                    for h in range(self.kv_heads):
                        scale[b, h] = 2.0 ** int(g.integers(-12, 4)) if powers else float(np.exp(g.uniform(-5, 2)))
                some = torch.from_numpy(values * 60).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
                codes[held] = some[held]
                self.pools.append(codes)
                self.scales.append(scale)
            else:
                v = torch.from_numpy(values).to(dtype).double().numpy()
                v[~held] = NAN
                self.pools.append(v)
        make = lambda heads: torch.from_numpy(g.standard_normal((self.tokens, heads, dim))).to(dtype)  # noqa: E731
        self.q, self.k, self.v = make(self.q_heads), make(self.kv_heads), make(self.kv_heads)
        self.scale = dim ** -0.5
        self.rope = None
        if rope_dim:
            n = max([h + a for h, a in zip(hit, app)]) + 2
            angle = np.arange(n)[:, None] * 10000.0 ** (-2 * np.arange(rope_dim // 2) / rope_dim)
            self.rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1)).float()
        self.layout = K.make_attn_layout(bs, self.q_heads, self.kv_heads, dim, self.blocks, dtype, torch.float8_e4m3fn if e4m3 else dtype,
                                         window, sinks, rope_dim, K.KVL_ROPE_HALVES if pairs == "halves" else K.KVL_ROPE_NEIGHBOURS)
        self.flags = flags

    def plan(self, flags=K.KVL_GATHER):
        keys = {"all": K.KVL_TOKENS_ALL, "hit": 0, "append": K.KVL_TOKENS_APPEND}[self.keys]
        return K.kvl_attn_plan(self.layout, self.hit, self.app, self.tables, flags | keys | self.flags)

    def planes(self):
        if self.e4m3:
            return [torch.from_numpy(x.copy()).cuda() for x in self.pools + self.scales]
        return [torch.from_numpy(x).to(self.dtype).cuda() for x in self.pools]

    def values(self):
        if not self.e4m3:
            return self.pools
        return [O.e4m3_values(c) * s.astype(np.float64)[:, None, :, None] for c, s in zip(self.pools, self.scales)]

    def want(self):
        return O.attend(self.hit, self.app, self.tables, self.bs, self.q.double().numpy(), *self.values(), self.scale, self.keys, self.window, self.sinks)


def attend(b, plan=None, q=None, out=None, lse=True, stream=None, planes=None):
    p = plan or b.plan()
    q = b.q.cuda() if q is None else q
    out = torch.full((b.tokens, b.q_heads, b.dim), NAN, dtype=b.dtype, device="cuda") if out is None else out
    l = torch.full((b.tokens, b.q_heads), NAN, device="cuda") if lse else None
    ws = torch.full((p.workspace_bytes // 4,), NAN, device="cuda") if p.workspace_bytes else None
    K.kvl_attn_layer(p, q, planes or b.planes(), out, ws, scale=b.scale, lse=l, stream=stream)
    return out, l


def close(b, out, lse, want, foreign=False):
    """`foreign`: scales that are no powers of two, which the kernel for many rows multiplies in T: keys and values with a rounding of their own."""
    w_out, w_lse, weight, reach = want
    u = unit(b.dtype)
    n = max([h + a for h, a in zip(b.hit, b.app)] + [1])
    ds = (b.dim + 16) * 2.0 ** -24 * reach + 2.0 ** -20 + (u * reach if foreign else 0)
    rel = 4 * ds[..., None] + n * 2.0 ** -24 + u + (u if foreign else 0)
    # (fp16: weights below 2^-22 of the largest are off by up to 2^-33 of it)
    floor = n * 2.0 ** -33 * (np.nanmax(np.abs(b.values()[1])) if b.tokens else 0) if b.dtype == torch.float16 else 1e-30
    bound = rel * weight + u * np.abs(w_out) * 1.01 + floor + (2.0 ** -24 if b.dtype == torch.float16 else 0)
    got = out.double().cpu().numpy()
    far = np.abs(got - w_out) - bound
    assert np.all(np.isfinite(got)), f"{np.sum(~np.isfinite(got))} outputs are not finite"
    assert far.max(initial=-1) <= 0, f"off by {np.abs(got - w_out).flat[far.argmax()]:.3g}, bound {bound.flat[far.argmax()]:.3g} at {np.unravel_index(far.argmax(), far.shape)}"
    if lse is not None:
        l = lse.double().cpu().numpy()
        empty = np.isneginf(w_lse)
        assert np.array_equal(np.isneginf(l), empty)
        e = np.abs(l[~empty] - w_lse[~empty]) - (2 * ds + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(w_lse) + reach))[~empty]
        assert e.max(initial=-1) <= 0


CASES = [
    # hit, app, block, heads, dim
    ([5], [1], 16, (1, 1), 128),                                    # one head of one token
    ([0, 1, 15, 16, 17, 63, 64, 65], [1] * 8, 16, (8, 2), 128),     # first tokens and tile edges
    ([33, 700, 0, 129, 300], [1] * 5, 24, (16, 1), 64),             # pages that end inside a tile
    ([400, 0, 90, 513], [2, 3, 1, 4], 1, (14, 2), 128),             # a group of seven, pages of one token
    ([250, 10, 0], [5, 16, 9], 7, (12, 4), 64),                     # odd pages
    ([1000, 300], [8, 1], 100, (8, 1), 128),                        # 64 rows and 8
    ([0, 31, 200], [200, 65, 33], 16, (8, 4), 128),                 # whole prompts
    ([130, 0], [150, 301], 24, (6, 2), 64),
    ([77, 500, 40, 0], [129, 1, 7, 40], 64, (9, 3), 128),           # every kernel in one batch
    ([2500], [1], 64, (4, 2), 128),                                 # keys cut into pieces
    ([1900], [70], 32, (2, 1), 64),
]


@pytest.mark.parametrize("hit,app,bs,heads,dim", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("e4m3", [False, True])
def test_whole_prompt(hit, app, bs, heads, dim, dtype, e4m3):
    b = Batch(hit, app, bs, heads, dim, dtype, e4m3)
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, b.want())


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (64, 0), (100, 4), (100, 70), (300, 2000), (10000, 3)])
@pytest.mark.parametrize("keys", ["all", "hit", "append"])
@pytest.mark.parametrize("e4m3", [False, True])
def test_windows_and_first_tokens(window, sinks, keys, e4m3):
    b = Batch([0, 3, 260, 700, 90, 0], [1, 1, 4, 40, 120, 70], 24, (8, 2), 64, torch.bfloat16, e4m3, keys, window=window, sinks=sinks)
    out, lse = attend(b)
    torch.cuda.synchronize()
    want = b.want()
    if keys == "hit":
        assert np.isneginf(want[1]).any()       # rows that see nothing are among them
    close(b, out, lse, want)
    assert np.all(out.cpu().float().numpy()[np.isneginf(want[1])] == 0)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scales_that_are_no_powers_of_two(dim, dtype):
    b = Batch([90, 700, 300], [1, 40, 3], 16, (8, 2), dim, dtype, True, powers=False, spread=0.2)
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, b.want(), foreign=True)


# scores far apart: the running maximum rises late, and most weights vanish
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("app", [1, 40])
def test_scores_far_apart(e4m3, app):
    b = Batch([900], [app], 16, (4, 2), 128, torch.bfloat16, e4m3, spread=3.0)
    b.scale = 1.0 if not e4m3 else 0.05
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, b.want())


# a token that holds NaN or infinities spoils the rows that see it and no others
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("what", ["k", "v", "v-inf"])
@pytest.mark.parametrize("app,heads", [(6, (4, 2)), (90, (4, 2)), (10, (6, 1))])
def test_spoilt_tokens_reach_only_rows_that_see_them(e4m3, what, app, heads):
    if e4m3 and what == "v-inf":
        what = "v"                                  # (e4m3 has no infinities)
    b = Batch([70], [app], 16, heads, 64, torch.float16, e4m3, window=60, sinks=2)
    at = 70 + app // 2
    pool = b.pools[0 if what == "k" else 1]
    block, row = b.tables[0][at // 16], at % 16
    if e4m3:
        pool[block, row, :, 5] = 0xFF
    else:
        pool[block, row, :, 5] = np.inf if what == "v-inf" else NAN
    out, lse = attend(b)
    torch.cuda.synchronize()
    clean = [i for i in range(app) if 70 + i < at or 70 + i - at >= 60]
    spoilt = [i for i in range(app) if i not in clean]
    assert clean and spoilt
    got = out.cpu().float().numpy()
    with np.errstate(invalid="ignore"):
        w_out, w_lse, weight, reach = b.want()
    assert np.all(np.isfinite(got[clean]))
    u = unit(b.dtype)
    bound = (4 * ((b.dim + 16) * 2.0 ** -24 * reach[clean][..., None] + 2.0 ** -20) + 2 * u) * weight[clean] + u * np.abs(w_out[clean]) + 1e-5
    assert np.all(np.abs(got[clean] - w_out[clean]) <= bound)
    if what == "k":
        assert np.all(np.isnan(got[spoilt]))
    else:
        assert not np.any(np.isfinite(got[spoilt][:, :, 5]))
        others = np.delete(np.arange(64), 5)
        assert np.all(np.isfinite(got[spoilt][:, :, others]))
        if what == "v-inf":
            assert np.all(np.isposinf(got[spoilt][:, :, 5]))


def test_strides_and_orders():
    b = Batch([100, 40], [1, 20], 16, (8, 2), 128, torch.bfloat16)
    fused = torch.full((b.tokens, 8 + 4, 128), NAN, dtype=b.dtype, device="cuda")
    fused[:, 2:10] = b.q.cuda()
    wide = torch.zeros(b.tokens, 16, 128, dtype=b.dtype, device="cuda")
    out, lse = attend(b, q=fused[:, 2:10], out=wide[:, 4:12])
    torch.cuda.synchronize()
    close(b, out, lse, b.want())
    assert not wide[:, :4].any() and not wide[:, 12:].any()


def test_blocks_shared_by_requests():
    bs = 16
    tables = [np.array([4, 2, 7, 1], dtype=np.int32), np.array([4, 2, 0], dtype=np.int32)]
    b = Batch([50, 33], [1, 1], bs, (4, 1), 128, torch.bfloat16, extra=1, tables=tables)
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, b.want())


def test_streams():
    b = Batch([2500, 300], [1, 2], 16, (8, 2), 128, torch.bfloat16, True)
    p, side = b.plan(), torch.cuda.Stream()
    planes = b.planes()
    with torch.cuda.stream(side):
        q = torch.zeros(b.tokens, 8, 128, dtype=b.dtype, device="cuda")
        torch.cuda._sleep(2_000_000)
        q.copy_(b.q)
        out, lse = attend(b, p, q=q, planes=planes)             # torch's current stream
    torch.cuda.synchronize()
    close(b, out, lse, b.want())
    out, lse = attend(b, p, planes=planes, stream=side)         # one that is named
    side.synchronize()
    torch.cuda.synchronize()


def test_plans_dropped_before_their_work_ends():
    results = []
    torch.cuda._sleep(20_000_000)
    for seed in range(6):
        b = Batch([1500, 10 * seed], [1, 3], 16, (8, 2), 64, torch.bfloat16, seed=seed)
        p = b.plan()
        results.append((b, *attend(b, p)))
        p.destroy()
    torch.cuda.synchronize()
    for b, out, lse in results:
        close(b, out, lse, b.want())


def test_graph_replays():
    b = Batch([2100, 70], [1, 1], 16, (8, 2), 128, torch.bfloat16, True, hold="hit", rope_dim=64)
    p = b.plan(K.KVL_GATHER | K.KVL_SCATTER)
    planes, rope = b.planes(), b.rope.cuda()
    q, k, v = (torch.zeros_like(x, device="cuda") for x in (b.q, b.k, b.v))
    out = torch.zeros_like(q)
    ws = torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda")
    q2 = torch.zeros_like(q)

    def step(stream=None):
        K.kvl_append_layer(p, k, v, planes, rope, q, q2, stream=stream)
        K.kvl_attn_layer(p, q2, planes, out, ws, stream=stream)

    start = [t.clone() for t in planes]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for seed in range(4):
        gen = torch.Generator().manual_seed(seed)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen))
        for t, s in zip(planes, start):
            t.copy_(s)
        graph.replay()
        got = [out.clone()] + [t.clone() for t in planes]
        for t, s in zip(planes, start):
            t.copy_(s)
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, [out] + planes):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    torch.cuda.synchronize()
    del graph


def test_same_result_each_time():
    b = Batch([3000, 500, 100], [1, 40, 3], 16, (8, 2), 128, torch.bfloat16, True)
    p, planes = b.plan(), b.planes()
    first, _ = attend(b, p, planes=planes)
    for _ in range(3):
        again, _ = attend(b, p, planes=planes)
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_pool_beyond_32_bit_offsets():
    """A block whose bytes begin above 4 GiB, in both operators."""
    bs, heads, dim = 64, (8, 8), 128
    blocks = 36_000                                     # 128 KiB each
    table = np.array([35_999, 3, 35_000], dtype=np.int32)
    lay = K.make_attn_layout(bs, *heads, dim, blocks, torch.bfloat16)
    p = K.kvl_attn_plan(lay, [130], [2], [table], K.KVL_GATHER | K.KVL_SCATTER | K.KVL_TOKENS_ALL)
    gen = torch.Generator(device="cuda").manual_seed(5)
    planes = [torch.empty(blocks, bs, 8, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert planes[0].nbytes > 1 << 32
    for t in planes:
        t[table.tolist()] = torch.randn(3, bs, 8, dim, device="cuda", generator=gen).bfloat16()
    q, k, v = (torch.randn(2, 8, dim, device="cuda", generator=gen).bfloat16() for _ in range(3))
    K.kvl_append_layer(p, k, v, planes)
    out, ws = torch.empty_like(q), torch.empty(max(1, p.workspace_bytes), dtype=torch.uint8, device="cuda")
    K.kvl_attn_layer(p, q, planes, out, ws)
    torch.cuda.synchronize()
    small = [t[table.tolist()].double().cpu().numpy() for t in planes]
    assert np.array_equal(small[0][2, 2:4], k.double().cpu().numpy()) and np.array_equal(small[1][2, 2:4], v.double().cpu().numpy())
    b = Batch([130], [2], bs, heads, dim, extra=0, tables=[np.arange(3, dtype=np.int32)])
    b.q, b.pools = q.cpu(), small
    w = O.attend([130], [2], [np.arange(3)], bs, q.double().cpu().numpy(), *small, dim ** -0.5)
    close(b, out, None, w)


# append ---------------------------------------------------------------------------------------------------------------------------

def appended(b, q=True, strided=False, stream=None):
    p = b.plan(K.KVL_SCATTER)
    planes = b.planes()
    rope = None if b.rope is None else b.rope.cuda()
    dq, dk, dv = b.q.cuda(), b.k.cuda(), b.v.cuda()
    if strided:
        fused = torch.cat([dq, dk, dv], 1)
        dq, dk, dv = fused[:, :b.q_heads], fused[:, b.q_heads:b.q_heads + b.kv_heads], fused[:, b.q_heads + b.kv_heads:]
    out = torch.full((b.tokens, b.q_heads, b.dim), NAN, dtype=b.dtype, device="cuda") if q else None
    K.kvl_append_layer(p, dk, dv, planes, rope, dq if q else None, out, stream=stream)
    torch.cuda.synchronize()
    return out, planes


def turned(b, x):
    table = None if b.rope is None else b.rope.double().numpy()
    y = np.zeros(x.shape)
    i = 0
    for h, n in zip(b.hit, b.app):
        for t in range(h, h + n):
            for head in range(x.shape[1]):
                y[i, head] = O.rotate(x[i, head].double().numpy(), table, t, b.pairs)
            i += 1
    return y


def near_turned(got, want, x, dtype):
    """Rounded once to the type; the rotation is two products and a sum in 32 bits, at most 3 * 2^-24 of |a| + |b| off."""
    size = np.abs(x.double().numpy()).max(initial=0)
    bound = unit(dtype) * np.abs(want) * 1.0001 + 6 * 2.0 ** -24 * size + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)


APPENDS = [
    ([5], [1], 16, (1, 1), 128),
    ([0, 16, 15, 33], [1, 1, 1, 1], 16, (8, 2), 128),
    ([0, 7, 100, 64, 3], [3, 0, 40, 64, 130], 24, (6, 3), 64),
    ([10, 0], [5, 21], 1, (4, 4), 64),
    ([100, 190], [260, 11], 100, (4, 1), 128),
]


@pytest.mark.parametrize("hit,app,bs,heads,dim", APPENDS)
@pytest.mark.parametrize("rope,pairs", [(0, "halves"), (16, "halves"), (64, "halves"), (64, "neighbours"), (48, "neighbours")])
@pytest.mark.parametrize("dtype,strided", [(torch.bfloat16, False), (torch.float16, True)])
def test_append_16_bits(hit, app, bs, heads, dim, rope, pairs, dtype, strided):
    b = Batch(hit, app, bs, heads, dim, dtype, hold="hit", rope_dim=rope, pairs=pairs)
    out, planes = appended(b, strided=strided)
    near_turned(out, turned(b, b.q), b.q, dtype)
    k = turned(b, b.k)
    pool = [x.copy() for x in b.pools]
    O.append(hit, app, b.tables, bs, k, pool[0])
    O.append(hit, app, b.tables, bs, b.v.double().numpy(), pool[1])
    got = [t.double().cpu().numpy() for t in planes]
    assert np.array_equal(got[1], pool[1], equal_nan=True)
    new = ~np.isnan(pool[0]) & ~b.held[..., None, None]
    assert np.array_equal(got[0][~new], pool[0][~new], equal_nan=True)      # every other row keeps its bytes
    size = np.abs(b.k.double().numpy()).max(initial=0)
    assert np.all(np.abs(got[0] - pool[0])[new] <= (unit(dtype) * 1.0001 * np.abs(pool[0]) + 6 * 2.0 ** -24 * size + 2.0 ** -25)[new])
    if not rope:
        assert np.array_equal(got[0], pool[0], equal_nan=True) and torch.equal(out.cpu(), b.q)


@pytest.mark.parametrize("hit,app,bs,heads,dim", APPENDS)
@pytest.mark.parametrize("rope,pairs", [(0, "halves"), (64, "halves"), (32, "neighbours")])
@pytest.mark.parametrize("dtype,powers", [(torch.bfloat16, True), (torch.float16, True), (torch.bfloat16, False)])
@pytest.mark.parametrize("spread", [1e-4, 1.0, 300.0])
def test_append_8_bits(hit, app, bs, heads, dim, rope, pairs, dtype, powers, spread):
    """Codes and scales are the oracle's, bit for bit."""
    b = Batch(hit, app, bs, heads, dim, dtype, True, hold="hit", rope_dim=rope, pairs=pairs, powers=powers)
    b.k, b.v = (b.k * spread).to(dtype), (b.v * spread).to(dtype)
    out, planes = appended(b, strided=True)
    near_turned(out, turned(b, b.q), b.q, dtype)
    for x, new in ((0, turned(b, b.k)), (1, b.v.double().numpy())):
        pool, scales = b.pools[x].copy(), b.scales[x].astype(np.float64)
        O.append(hit, app, b.tables, bs, new, pool, scales)
        assert np.array_equal(planes[2 + x].double().cpu().numpy(), scales, equal_nan=True)
        same = planes[x].cpu().numpy() == pool
        zero = (planes[x].cpu().numpy() & 0x7F == 0) & (pool & 0x7F == 0)   # (either sign of zero)
        assert np.all(same | zero), f"{np.sum(~(same | zero))} codes of {pool.size}"


def test_append_8_bits_odd_values():
    b = Batch([3], [4], 16, (2, 2), 64, torch.bfloat16, True, hold="hit")
    b.k[0, 0, 3], b.k[1, 0, 9], b.k[2, 0, 60] = NAN, float("inf"), -float("inf")
    b.v[:, 1] = 0
    b.v[0, 0, 0] = 3e38
    out, planes = appended(b)
    assert torch.isfinite(planes[2][b.tables[0][0]]).all()
    for x, new in ((0, b.k.double().numpy()), (1, b.v.double().numpy())):
        pool, scales = b.pools[x].copy(), b.scales[x].astype(np.float64)
        O.append(b.hit, b.app, b.tables, 16, new, pool, scales)
        assert np.array_equal(planes[2 + x].double().cpu().numpy(), scales, equal_nan=True)
        assert np.array_equal(O.e4m3_values(planes[x].cpu().numpy()), O.e4m3_values(pool), equal_nan=True)


def test_append_without_queries_and_in_place():
    b = Batch([30, 2], [1, 9], 16, (8, 2), 128, torch.bfloat16, True, hold="hit", rope_dim=128)
    _, with_q = appended(b)
    _, without = appended(b, q=False)
    for x, y in zip(with_q, without):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    p, q = b.plan(K.KVL_SCATTER), b.q.cuda()
    K.kvl_append_layer(p, b.k.cuda(), b.v.cuda(), b.planes(), b.rope.cuda(), q)
    torch.cuda.synchronize()
    near_turned(q, turned(b, b.q), b.q, b.dtype)


def test_append_then_attend():
    """Both, as a layer makes them, the keys' codes as the append left them."""
    b = Batch([70, 0, 300], [1, 90, 4], 16, (8, 2), 128, torch.bfloat16, True, hold="hit", rope_dim=128)
    p = b.plan(K.KVL_GATHER | K.KVL_SCATTER)
    planes, q = b.planes(), b.q.cuda()
    K.kvl_append_layer(p, b.k.cuda(), b.v.cuda(), planes, b.rope.cuda(), q)
    out, lse = attend(b, p, q=q, planes=planes)
    torch.cuda.synchronize()
    b.q = q.cpu()
    b.pools, b.scales = [t.cpu().numpy() for t in planes[:2]], [t.cpu().numpy() for t in planes[2:]]
    close(b, out, lse, b.want())


def test_nothing_to_do():
    b = Batch([30, 2], [0, 0], 16, (8, 2), 128, torch.bfloat16)
    p = b.plan(K.KVL_GATHER | K.KVL_SCATTER)
    q = torch.empty(0, 8, 128, dtype=b.dtype, device="cuda")
    k = torch.empty(0, 2, 128, dtype=b.dtype, device="cuda")
    planes = b.planes()
    K.kvl_append_layer(p, k, k, planes, q=q)
    K.kvl_attn_layer(p, q, planes, q.clone())
    torch.cuda.synchronize()


def test_refusals():
    """Each comes back as an error before anything is launched."""
    b = Batch([2500], [2], 16, (8, 2), 128, torch.bfloat16, True, rope_dim=64)
    p = b.plan(K.KVL_GATHER | K.KVL_SCATTER)
    assert p.workspace_bytes
    planes, rope = b.planes(), b.rope.cuda()
    q, k, v = b.q.cuda(), b.k.cuda(), b.v.cuda()
    out = torch.empty_like(q)
    ws = torch.empty(p.workspace_bytes, dtype=torch.uint8, device="cuda")

    def refused(code, call, *args, **kw):
        with pytest.raises(K.KvlError) as e:
            call(*args, **kw)
        assert e.value.code == code, e.value

    refused(K.KVL_EINVAL, K.kvl_attn_layer, p, q, planes, out)                              # no workspace
    refused(K.KVL_ESPACE, K.kvl_attn_layer, p, q, planes, out, ws[:-256])
    refused(K.KVL_EINVAL, K.kvl_attn_layer, p, q, planes, out, torch.empty(p.workspace_bytes + 64, dtype=torch.uint8, device="cuda")[64:])
    for scale in (0.0, -1.0, NAN, float("inf")):
        refused(K.KVL_EINVAL, K.kvl_attn_layer, p, q, planes, out, ws, scale=scale)
    refused(K.KVL_ESPACE, K.kvl_append_layer, p, k, v, planes, rope[:2501], q)              # a table too short
    refused(K.KVL_EINVAL, K.kvl_append_layer, b.plan(K.KVL_GATHER), k, v, planes, rope, q)
    refused(K.KVL_EINVAL, K.kvl_attn_layer, b.plan(K.KVL_SCATTER), q, planes, out, ws)
    for bad in (q.float(), q.cpu()):
        with pytest.raises(TypeError):
            K.kvl_attn_layer(p, bad, planes, out, ws)
    for bad in (q[:1], q.transpose(0, 1).contiguous().transpose(0, 1), torch.empty(2 * 1024 + 4, dtype=b.dtype, device="cuda")[4:].view(2, 8, 128),
                torch.empty(2, 1028, dtype=b.dtype, device="cuda")[:, :1024].unflatten(1, (8, 128))):
        with pytest.raises(ValueError):
            K.kvl_attn_layer(p, bad, planes, out, ws)
    with pytest.raises(ValueError):
        K.kvl_attn_layer(p, q, planes[:2], out, ws)
    with pytest.raises(ValueError):
        K.kvl_attn_layer(p, q, [planes[0][:-1], *planes[1:]], out, ws)
    with pytest.raises(ValueError):
        K.kvl_attn_layer(p, q, planes, out, ws, lse=torch.empty(2, 7, device="cuda"))
    with pytest.raises(ValueError):
        K.kvl_append_layer(p, k, v, planes, None, q)
    with pytest.raises(ValueError):
        K.kvl_append_layer(p, k, v, planes, rope[:, :16], q)
    with pytest.raises(ValueError):
        K.kvl_append_layer(p, k, v, planes, rope, None, q)
    torch.cuda.synchronize()
