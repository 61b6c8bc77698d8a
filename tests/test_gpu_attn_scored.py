"""Attention with capped scores, a bias by distance, prefixes and documents on the GPU against the oracle's 64 bits, and joins of results.

Tolerances are those of the plain operator (test_gpu_attn.py), with what the scores add to their error: a capped score is computed as
cap (1 - 2 / (1 + 2^x)), whose sum, reciprocal, exponential and last step are off by at most (2 (1 + 2 + 2) + 1) 2^-24 < 2^-20 of the cap (a tanh's slope is
at most 1, so what the argument is off by comes through as it is); a bias is a slope times log2(e), times a distance, in parts that are
added to the score one after the other: six roundings of at most 2^-24 of the largest bias.
"""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from oracle import attn_oracle as O
from test_gpu_attn import NAN, Batch, unit

pytestmark = pytest.mark.gpu


class Scored(Batch):
    def __init__(self, *args, cap=0.0, slopes=False, prefix=None, documents=None, loud=1.0, **kw):
        super().__init__(*args, **kw)
        self.cap, self.prefix, self.documents = cap, prefix, documents
        # (the first head's slope is 0, the last one's negative: it favours what is far)
        self.slopes = None
        if slopes:
            self.slopes = torch.exp2(-8 * torch.arange(1, self.q_heads + 1) / self.q_heads)
            self.slopes[0] = 0
            self.slopes[-1] *= -0.05 if self.q_heads > 1 else 1
        self.q = (self.q.float() * loud).to(self.dtype)

    def plan(self, flags=K.KVL_GATHER):
        keys = {"all": K.KVL_TOKENS_ALL, "hit": 0, "append": K.KVL_TOKENS_APPEND}[self.keys]
        return K.kvl_attn_plan(self.layout, self.hit, self.app, self.tables, flags | keys | self.flags, self.prefix, self.documents)

    def want(self):
        return O.attend(self.hit, self.app, self.tables, self.bs, self.q.double().numpy(), *self.values(), self.scale, self.keys, self.window, self.sinks,
                        self.cap, None if self.slopes is None else self.slopes.double().numpy(), self.prefix, self.documents)


def attend(b, plan=None, planes=None, out=None, workspace=None, stream=None):
    p = plan or b.plan()
    out = torch.full((b.tokens, b.q_heads, b.dim), NAN, dtype=b.dtype, device="cuda") if out is None else out
    lse = torch.full((b.tokens, b.q_heads), NAN, device="cuda")
    if workspace is None:
        workspace = torch.full((p.workspace_bytes // 4,), NAN, device="cuda") if p.workspace_bytes else None
    K.kvl_attn_layer(p, b.q.cuda(), planes or b.planes(), out, workspace, scale=b.scale, lse=lse, stream=stream, cap=b.cap or None,
                     slopes=None if b.slopes is None else b.slopes.cuda())
    return out, lse


def close(b, out, lse, want, foreign=False):
    w_out, w_lse, weight, reach = want
    u, n = unit(b.dtype), max([h + a for h, a in zip(b.hit, b.app)] + [1])
    far = 0 if b.slopes is None else float(b.slopes.abs().max()) * n
    ds = (b.dim + 16) * 2.0 ** -24 * reach + 2.0 ** -20 + 2.0 ** -20 * b.cap + 6 * 2.0 ** -24 * far + (u * reach if foreign else 0)
    rel = 4 * ds[..., None] + n * 2.0 ** -24 + u + (u if foreign else 0)
    floor = n * 2.0 ** -33 * np.nanmax(np.abs(b.values()[1])) if b.dtype == torch.float16 else 1e-30
    bound = rel * weight + u * np.abs(w_out) * 1.01 + floor + (2.0 ** -24 if b.dtype == torch.float16 else 0)
    got = out.double().cpu().numpy()
    assert np.all(np.isfinite(got)), f"{np.sum(~np.isfinite(got))} outputs are not finite"
    over = np.abs(got - w_out) - bound
    assert over.max(initial=-1) <= 0, f"off by {np.abs(got - w_out).flat[over.argmax()]:.3g}, bound {bound.flat[over.argmax()]:.3g} at {np.unravel_index(over.argmax(), over.shape)}"
    l = lse.double().cpu().numpy()
    empty = np.isneginf(w_lse)
    assert np.array_equal(np.isneginf(l), empty)
    assert np.all(got[empty] == 0)
    e = np.abs(l[~empty] - w_lse[~empty]) - (2 * ds + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(w_lse) + reach))[~empty]
    assert e.max(initial=-1) <= 0


BATCHES = [
    # hit, app, block, heads, dim
    ([0, 1, 15, 16, 17, 63, 64, 65], [1] * 8, 16, (8, 2), 128),     # first tokens and tile edges
    ([33, 700, 0, 129, 300], [1] * 5, 24, (16, 1), 64),             # pages that end inside a tile
    ([400, 0, 90, 513], [2, 3, 1, 4], 1, (14, 2), 128),             # a group of seven, pages of one token
    ([250, 10, 0], [5, 16, 9], 7, (12, 4), 64),                     # odd pages
    ([1000, 300], [8, 1], 100, (8, 1), 128),                        # 64 rows and 8
    ([0, 31, 200], [200, 65, 33], 16, (8, 4), 128),                 # whole prompts
    ([130, 0], [150, 301], 24, (6, 2), 64),
]
FORMS = {
    "cap": dict(cap=5.0, loud=6.0),
    "large_cap": dict(cap=1000.0, loud=3.0),
    "least_cap": dict(cap=2.0 ** -10),
    "slopes": dict(slopes=True),
    "both_window": dict(cap=20.0, slopes=True, loud=4.0, window=37, sinks=3),
    "slopes_hit": dict(slopes=True, keys="hit"),
    "cap_append": dict(cap=7.0, keys="append"),
}


TYPES = [(torch.bfloat16, False), (torch.float16, True), (torch.bfloat16, True), (torch.float16, False)]


@pytest.mark.parametrize("at,form,dtype,e4m3", [(at, form, dtype, e4m3) for at in range(len(BATCHES)) for i, form in enumerate(FORMS)
                                                for dtype, e4m3 in (TYPES[:2] if (at + i) % 2 else TYPES[2:])])
def test_scores(at, form, dtype, e4m3):
    b = Scored(*BATCHES[at], dtype=dtype, e4m3=e4m3, seed=at, **FORMS[form])
    close(b, *attend(b), b.want())


def some_masks(b_hit, b_app, seed, prefix, documents):
    g = np.random.default_rng(seed)
    total = [h + a for h, a in zip(b_hit, b_app)]
    p = [int(g.integers(0, t + 3)) for t in total] if prefix else None
    d = [np.unique(g.integers(0, t + 4, size=int(g.integers(0, 7)))) for t in total] if documents else None
    return dict(prefix=p, documents=d)


@pytest.mark.parametrize("at", range(len(BATCHES)))
@pytest.mark.parametrize("what", ["prefix", "documents", "prefix_documents", "all", "hit", "append"])
@pytest.mark.parametrize("dtype,e4m3", [(torch.bfloat16, False), (torch.float16, True)])
def test_masks(at, what, dtype, e4m3):
    hit, app = BATCHES[at][:2]
    masks = some_masks(hit, app, 17 * at + len(what), what != "documents", what != "prefix")
    kw = dict(all=dict(window=29, sinks=5, slopes=True, cap=9.0), hit=dict(keys="hit", sinks=2), append=dict(keys="append", window=50)).get(what, {})
    b = Scored(*BATCHES[at], dtype=dtype, e4m3=e4m3, seed=at, **masks, **kw)
    close(b, *attend(b), b.want())


def test_a_mask_of_nothing_is_no_mask():
    """No prefix and one document: bit for bit what the plan without a mask gives; and a cap of 0 is none."""
    b = Scored(*BATCHES[5], window=64, sinks=4, prefix=[0, 0, 0], documents=[[], [0], [0]])
    plain = Scored(*BATCHES[5], window=64, sinks=4)
    got, want = attend(b), attend(plain)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    out = torch.zeros_like(got[0])
    lse = torch.zeros_like(got[1])
    p = plain.plan()
    K.kvl_attn_layer(p, b.q.cuda(), b.planes(), out, torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda"), scale=b.scale, lse=lse, cap=0.0)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("app", [3, 150])
def test_other_documents_do_not_reach_a_query_whatever_they_hold(app, e4m3):
    """One document's keys and values are NaN and infinite: the queries of the others are as they were."""
    kw = dict(hit=[90], app=[app], bs=16, heads=(8, 2), dim=64, e4m3=e4m3, documents=[[0, 40, 70, 91]], cap=8.0, slopes=True)
    b = Scored(**kw)
    want = b.want()
    planes = b.planes()
    for t in range(40, 70):
        block, row = b.tables[0][t // 16], t % 16
        for x in range(2):
            if e4m3:
                planes[x][block, row] = 0x7F if t % 2 else 0xFF
            else:
                planes[x][block, row] = [NAN, float("inf"), -float("inf")][t % 3]
    close(b, *attend(b, planes=planes), want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_infinite_values_reach_the_rows_that_see_them(e4m3):
    """With a prefix that ends inside the tail: an infinite value in a key that only some rows see."""
    b = Scored([20], [60], 16, (4, 2), 64, e4m3=e4m3, prefix=[30], documents=[[0, 50]])
    want = b.want()
    planes = b.planes()
    planes[1][b.tables[0][45 // 16], 45 % 16, 1, 7] = 0x7F if e4m3 else float("inf")      # (token 45: seen by queries at 45 to 49)
    out, lse = attend(b, planes=planes)
    got = out.float().cpu().numpy()
    hurt = np.zeros(got.shape, dtype=bool)
    hurt[25:30, 2:4, 7] = True
    assert np.all(~np.isfinite(got[hurt])) and np.all(np.isfinite(got[~hurt]))
    out[torch.from_numpy(hurt).cuda()] = torch.from_numpy(want[0][hurt]).to(out)
    close(b, out, lse, want)


@pytest.mark.parametrize("dim", [64, 128])
def test_long_keys_in_pieces(dim):
    """Keys cut into pieces: the join of them takes capped scores and biases as it takes others."""
    b = Scored([9000, 4000], [1, 1], 64, (8, 2), dim, cap=10.0, slopes=True, prefix=[50, 0], documents=[[100, 8000], [3000]])
    assert b.plan().workspace_bytes > 0
    close(b, *attend(b), b.want())


def test_a_bias_over_far_keys():
    """Queries far behind the only keys (the cached prefix): what a bias loses in 32 bits."""
    b = Scored([100], [500], 16, (2, 1), 64, slopes=True, keys="hit")
    close(b, *attend(b), b.want())


@pytest.mark.parametrize("blocks", [(1 << 19) - 1, 1 << 19, (1 << 19) + 9])
@pytest.mark.parametrize("slopes", [False, True])
def test_planes_around_4_gib(blocks, slopes):
    """The last blocks of planes of 2^32 bytes, one block less and some more: what a small pool gives, bit for bit (addresses in 32 and 64 bits)."""
    b = Scored([70, 0, 5], [90, 200, 1], 64, (2, 1), 64, slopes=slopes)
    want = attend(b)
    small = b.planes()
    first = blocks - small[0].shape[0]
    planes = [torch.empty(blocks, *x.shape[1:], dtype=x.dtype, device="cuda") for x in small]
    for x, y in zip(planes, small):
        x[first:] = y
    layout = K.make_attn_layout(64, 2, 1, 64, blocks, b.dtype)
    p = K.kvl_attn_plan(layout, b.hit, b.app, [t + np.int32(first) for t in b.tables], K.KVL_GATHER | K.KVL_TOKENS_ALL)
    got = attend(b, p, planes=planes)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_one_output_twice_and_on_another_stream():
    """Two plans' calls on two streams at once, each with a workspace of its own."""
    b = Scored([3000, 100], [2, 40], 16, (8, 2), 128, cap=6.0, prefix=[10, 120])
    p1, p2 = b.plan(), b.plan()
    want = attend(b, p1)
    planes, streams = b.planes(), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s, p in zip(streams, (p1, p2)):
        with torch.cuda.stream(s):
            for _ in range(3):
                got.append(attend(b, p, planes=planes))
    torch.cuda.synchronize()
    for out, lse in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_captured_and_replayed():
    b = Scored([3000, 100], [2, 40], 16, (8, 2), 128, cap=6.0, slopes=True, documents=[[5, 2000], [30]])
    p = b.plan()
    planes, q, slopes = b.planes(), b.q.cuda(), b.slopes.cuda()
    out, lse = torch.zeros(b.tokens, 8, 128, dtype=b.dtype, device="cuda"), torch.zeros(b.tokens, 8, device="cuda")
    ws = torch.zeros(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda")
    joined = torch.zeros_like(out)

    def step():
        K.kvl_attn_layer(p, q, planes, out, ws, scale=b.scale, lse=lse, cap=6.0, slopes=slopes)
        K.kvl_attn_join(p, [out, out], [lse, lse], joined)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        q.copy_((b.q.float() * (1 + k)).to(b.dtype))
        step()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone(), joined.clone()
        for x in (out, lse, joined):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse, joined), want):
            assert torch.equal(x, y)
        assert bool(out.float().abs().max() > 0)
        _ = torch.randn(1 << 20, device="cuda").sum().item()
    del graph


def test_refusals():
    b = Scored([20, 0], [3, 17], 16, (4, 2), 64, slopes=True)
    p, planes, q = b.plan(), b.planes(), b.q.cuda()
    out, ws = torch.zeros_like(q), torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda")
    for cap in (-1.0, 2.0 ** -11, 2.0 ** 11, float("nan"), float("inf"), -0.5):
        with pytest.raises(K.KvlError) as e:
            K.kvl_attn_layer(p, q, planes, out, ws, cap=cap)
        assert e.value.code == K.KVL_EINVAL
    for scale in (2.0 ** -65, 2.0 ** 65):
        with pytest.raises(K.KvlError) as e:
            K.kvl_attn_layer(p, q, planes, out, ws, scale=scale, slopes=b.slopes.cuda())
        assert e.value.code == K.KVL_EINVAL
    for slopes in (torch.zeros(4), torch.zeros(5, device="cuda"), torch.zeros(4, device="cuda").double(), torch.zeros(2, 2, device="cuda"), [0.1] * 4,
                   torch.zeros(8, device="cuda")[::2]):
        with pytest.raises((ValueError, TypeError)):
            K.kvl_attn_layer(p, q, planes, out, ws, slopes=slopes)
    torch.cuda.synchronize()
    assert not out.any()


# Joins ------------------------------------------------------------------------------------------------------------------------------------
#
# Of a part's weight: the exponential's argument, a difference of lses, is off by 2^-24 of its terms times log2(e) and once more; the exponential by 2^-23:
# below 2^-22 (1 + |lse|); sums of n terms n 2^-24; the result is rounded once.

def join_plan(tokens, heads, dim, dtype, **kw):
    lay = K.make_attn_layout(16, heads, heads, dim, tokens // 16 + 1, dtype)
    return K.kvl_attn_plan(lay, [0], [tokens], [np.arange(tokens // 16 + 1, dtype=np.int32)], K.KVL_GATHER, **kw)


def some_parts(n, tokens, heads, dim, dtype, seed=1):
    g = np.random.default_rng(seed)
    lses = [torch.from_numpy(g.standard_normal((tokens, heads)) * 4).float() for _ in range(n)]
    parts = [torch.from_numpy(g.standard_normal((tokens, heads, dim))).to(dtype) for _ in range(n)]
    for x, l in zip(parts, lses):
        none = torch.from_numpy(g.random((tokens, heads)) < 0.2)
        l[none] = -float("inf")
        x[none] = NAN                       # (what has no share may hold anything)
    if tokens > 2:
        for l in lses:
            l[2] = -float("inf")            # a token that sees nothing
    return parts, lses


def joined_right(parts, lses, out, lse, dtype):
    w_out, w_lse = O.join([x.double().numpy() for x in parts], [l.double().numpy() for l in lses])
    scale = np.abs(np.nan_to_num(np.stack([x.double().numpy() for x in parts]))).max(0)
    most = max(float(l[l > -float("inf")].abs().max()) if bool((l > -float("inf")).any()) else 0 for l in lses)
    rel = 2 * 2.0 ** -22 * (1 + most) + 2 * len(parts) * 2.0 ** -24
    bound = rel * scale + unit(dtype) * np.abs(w_out) * 1.01 + 2.0 ** -24
    assert np.all(np.abs(out.double().cpu().numpy() - w_out) <= bound)
    if lse is not None:
        l = lse.double().cpu().numpy()
        assert np.array_equal(np.isneginf(l), np.isneginf(w_lse))
        some = ~np.isneginf(w_lse)
        assert np.all(np.abs(l[some] - w_lse[some]) <= rel + 2.0 ** -23 * (1 + np.abs(w_lse[some])))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 16])
@pytest.mark.parametrize("tokens,heads,dim", [(1, 1, 64), (1, 32, 128), (37, 7, 128), (300, 12, 64), (3, 64, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_join(n, tokens, heads, dim, dtype):
    p = join_plan(tokens, heads, dim, dtype)
    parts, lses = some_parts(n, tokens, heads, dim, dtype, seed=n)
    out, lse = torch.full((tokens, heads, dim), NAN, dtype=dtype, device="cuda"), torch.full((tokens, heads), NAN, device="cuda")
    K.kvl_attn_join(p, [x.cuda() for x in parts], [l.cuda() for l in lses], out, lse)
    joined_right(parts, lses, out, lse, dtype)
    again = torch.zeros_like(out)
    K.kvl_attn_join(p, tuple(x.cuda() for x in parts), tuple(l.cuda() for l in lses), again)        # (the general path, without an lse)
    assert torch.equal(out, again)


def test_a_large_join():
    """More than the caches hold: 3 parts of 700 tokens of 128 heads, of which the rows of some tokens are looked at."""
    n, h, d, dtype = 700, 128, 128, torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    parts = [torch.randn(n, h, d, device="cuda", generator=g).to(dtype) for _ in range(5)]
    lses = [torch.randn(n, h, device="cuda", generator=g) for _ in range(5)]
    assert 6 * n * h * d * 2 > 128 << 20
    out, lse = torch.full((n, h, d), NAN, dtype=dtype, device="cuda"), torch.full((n, h), NAN, device="cuda")
    K.kvl_attn_join(join_plan(n, h, d, dtype), parts, lses, out, lse)
    at = [0, 1, 255, 256, 699]
    joined_right([x[at].cpu() for x in parts], [l[at].cpu() for l in lses], out[at], lse[at], dtype)
    w = torch.softmax(torch.stack(lses).double(), 0)
    near = sum(x.double() * y[..., None] for x, y in zip(parts, w))
    assert float((out.double() - near).abs().max()) < 2.0 ** -8 * float(near.abs().max()) + 2.0 ** -18


def test_join_in_place_and_at_strides():
    p = join_plan(40, 6, 64, torch.bfloat16)
    parts, lses = some_parts(3, 40, 6, 64, torch.bfloat16)
    wide = torch.zeros(40, 20 * 64, dtype=torch.bfloat16, device="cuda")
    views = [wide[:, 6 * 64 * i:6 * 64 * (i + 1)].unflatten(1, (6, 64)) for i in range(3)]
    for v, x in zip(views, parts):
        v.copy_(x)
    wide[:, 18 * 64:] = 7
    mine = [l.cuda() for l in lses]
    K.kvl_attn_join(p, views, mine, views[1], mine[2])
    joined_right(parts, lses, views[1], mine[2], torch.bfloat16)
    assert torch.equal(views[0].isnan().cpu(), parts[0].isnan()) and bool((wide[:, 18 * 64:] == 7).all())


@pytest.mark.parametrize("e4m3", [False, True])
def test_prefix_and_tail_apart_are_both_at_once(e4m3):
    """Attention over the cached prefix, over the tail, and their join: what one plan over all keys gives (with other scores, too)."""
    kw = dict(hit=[100, 0, 33], app=[40, 9, 1], bs=16, heads=(8, 2), dim=64, e4m3=e4m3, cap=12.0, slopes=True, prefix=[120, 3, 10], window=70, hold="all")
    parts = [attend(Scored(keys=keys, **kw)) for keys in ("hit", "append")]
    b = Scored(keys="all", **kw)
    out, lse = torch.zeros_like(parts[0][0]), torch.zeros_like(parts[0][1])
    K.kvl_attn_join(b.plan(), [x for x, _ in parts], [l for _, l in parts], out, lse)
    want = b.want()
    # (each part's outputs were rounded already)
    w_out, w_lse, weight, reach = want
    close(b, out, lse, (w_out, w_lse, weight * 2, reach + 1))


def test_join_refusals():
    p = join_plan(20, 4, 64, torch.bfloat16)
    parts, lses = some_parts(2, 20, 4, 64, torch.bfloat16)
    parts, lses, out = [x.cuda() for x in parts], [l.cuda() for l in lses], torch.zeros(20, 4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(parts=[]), dict(parts=parts[:1]), dict(parts=[parts[0], parts[1].half()]), dict(parts=[parts[0], parts[1][:-1]]), dict(parts=[parts[0].cpu(), parts[1]]),
                dict(lses=[lses[0], lses[1].double()]), dict(lses=[lses[0], lses[1][:, :2]]), dict(lses=lses * 2), dict(out=out.float()), dict(out=out[1:]), dict(lse=lses[0][1:]),
                dict(parts=parts * 9, lses=lses * 9)):
        with pytest.raises((ValueError, TypeError)):
            K.kvl_attn_join(p, **{**dict(parts=parts, lses=lses, out=out), **bad})
    wide = torch.zeros(20, 512, dtype=torch.bfloat16, device="cuda")[:, :256].unflatten(1, (4, 64))
    with pytest.raises(K.KvlError):             # the same place at another stride
        K.kvl_attn_join(p, [wide, parts[1]], lses, torch.as_strided(wide, (20, 4, 64), (256, 64, 1)))
    scatter = K.kvl_attn_plan(p.layout, [0], [20], [np.arange(2, dtype=np.int32)], K.KVL_SCATTER)
    with pytest.raises(K.KvlError):
        K.kvl_attn_join(scatter, parts, lses, out)
    torch.cuda.synchronize()
    assert not out.any()
