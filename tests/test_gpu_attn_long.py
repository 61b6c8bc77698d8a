"""The attention operators' forms for much work: hundreds of pieces to join, queries in launches of their own."""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from test_gpu_attn import Batch, attend, unit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dim,e4m3", [((1, 1), 128, True), ((4, 1), 64, True), ((2, 1), 64, False)])
def test_more_than_256_pieces(heads, dim, e4m3):
    """The join takes up to 256 pieces in a round.  Half of each row's weight is on five keys far apart, and what they have is seen in the output;
    the sum of all, to which a piece adds a thousandth, in lse.  Sums: no more than a piece's keys and the pieces one after the other, 768 terms."""
    b = Batch([131_000], [1], 64, heads, dim, torch.bfloat16, e4m3, spread=1.0)
    if e4m3:
        b.scales = [np.where(np.isnan(s), np.nan, np.float32(2.0 ** -6)) for s in b.scales]
    b.q[0, 1:] = b.q[0, :1]                     # (one row's keys would not do for another)
    p = b.plan()
    assert p.items()[0, 7] > 256
    q = b.q[0, 0].double().numpy()
    size = 11.5 / (b.scale * np.abs(q).sum())
    for t in (5, 65_000, 66_000, 90_123, 131_000):
        at = b.tables[0][t // 64], t % 64, 0
        key = torch.from_numpy(np.sign(q) * size)
        b.pools[0][at] = (key * 64).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy() if e4m3 else key.to(b.dtype).double().numpy()
    planes = b.planes()
    out, lse = attend(b, p, planes=planes)
    torch.cuda.synchronize()
    w_out, w_lse, weight, reach = b.want()
    ds = (dim + 16) * 2.0 ** -24 * reach + 2.0 ** -20
    got, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.all(np.abs(l - w_lse) <= 2 * ds + 768 * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(w_lse) + reach))
    u = unit(b.dtype)
    bound = (4 * ds[..., None] + 768 * 2.0 ** -24 + u) * weight + u * np.abs(w_out) * 1.01
    assert np.all(np.abs(got - w_out) <= bound)
    assert np.abs(w_out).max() > 20 * bound.max()
    assert np.exp(w_lse.min()) < 2.5 * 5 * np.exp(11.6)         # (the five keys have that share)


def rotated(x, rope, positions):
    """Halves, in 64 bits, on the device."""
    half = rope.shape[1]
    c, s = rope[positions].double()[:, None].unbind(-1)
    a, b = x[..., :half].double(), x[..., half:2 * half].double()
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * half:].double()], -1)


def near(got, want, x, dtype):
    """As near_turned, on the device."""
    bound = unit(dtype) * want.abs() * 1.0001 + 6 * 2.0 ** -24 * float(x.abs().max())
    assert bool(((got.double() - want).abs() <= bound).all())


def rope_table(n, half):
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return torch.stack([angle.cos(), angle.sin()], -1).float()


@pytest.mark.parametrize("in_place", [False, True])
def test_queries_of_an_8_bit_append_in_a_launch_of_their_own(in_place):
    """From 5 * 2^20 tasks on (64 heads of 128: 10,240 tokens): the same codes as without queries, queries turned."""
    hit, app, bs = [70, 0, 5000], [4000, 6001, 300], 64
    need = [(h + a + bs - 1) // bs for h, a in zip(hit, app)]
    at = np.cumsum([0] + need)
    order = np.random.default_rng(2).permutation(at[-1] + 1).astype(np.int32)
    tables = [order[x:y].copy() for x, y in zip(at[:-1], at[1:])]
    lay = K.make_attn_layout(bs, 64, 8, 128, len(order), torch.bfloat16, torch.float8_e4m3fn, rope_dim=64)
    p = K.kvl_attn_plan(lay, hit, app, tables, K.KVL_SCATTER)
    assert p.tokens * 64 * 8 > 5 << 20
    gen = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn(p.tokens, 80, 128, device="cuda", generator=gen).bfloat16()
    q, k, v = qkv.split([64, 8, 8], dim=1)
    rope = rope_table(6002, 32)
    planes = [[torch.randint(0, 120, (len(order), bs, 8, 128), device="cuda", dtype=torch.uint8, generator=gen) for _ in range(2)] +
              [torch.exp2(torch.randint(-9, 0, (len(order), 8), device="cuda", generator=gen).float()) for _ in range(2)]]
    planes.append([t.clone() for t in planes[0]])
    before = qkv.clone()
    K.kvl_append_layer(p, k, v, planes[0], rope)
    out = q if in_place else torch.full((p.tokens, 64, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    K.kvl_append_layer(p, k, v, planes[1], rope, q, out)
    torch.cuda.synchronize()
    for x, y in zip(*planes):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    positions = torch.cat([torch.arange(h, h + a, device="cuda") for h, a in zip(hit, app)])
    near(out, rotated(before[:, :64], rope, positions), before, torch.bfloat16)
    assert torch.equal(qkv[:, 64:], before[:, 64:])


def test_queries_beyond_one_launch():
    """A launch takes 2^30 tasks: 4095 tokens of 65536 heads of 64 (and one key and value).  Every token's queries are the same ones."""
    n, heads = 4100, 65536
    lay = K.make_attn_layout(64, heads, 1, 64, 80, torch.bfloat16, rope_dim=64)
    p = K.kvl_attn_plan(lay, [11], [n], [np.arange(65, dtype=np.int32)], K.KVL_SCATTER)
    gen = torch.Generator(device="cuda").manual_seed(4)
    one = torch.randn(1, heads, 64, device="cuda", generator=gen).bfloat16()
    q = torch.empty(n, heads, 64, device="cuda", dtype=torch.bfloat16)
    q[:] = one
    k, v = (torch.randn(n, 1, 64, device="cuda", generator=gen).bfloat16() for _ in range(2))
    planes = [torch.zeros(80, 64, 1, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    rope = rope_table(11 + n, 32)
    K.kvl_append_layer(p, k, v, planes, rope, q)
    torch.cuda.synchronize()
    for t in (0, 1, 2047, 4093, 4094, 4095, 4096, n - 1):
        near(q[t:t + 1], rotated(one, rope, torch.tensor([11 + t], device="cuda")), one, torch.bfloat16)
    rows = slice(11, 11 + n)
    assert torch.equal(planes[1].view(-1, 1, 64)[rows], v)
    near(planes[0].view(-1, 1, 64)[rows], rotated(k, rope, torch.arange(11, 11 + n, device="cuda")), k, torch.bfloat16)
    assert not planes[0].view(-1, 64)[:11].any() and not planes[1].view(-1, 64)[11 + n:].any()
    del q
    torch.cuda.empty_cache()                    # (34 GB)
