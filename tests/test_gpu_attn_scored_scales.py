"""Other scores and masks over 8-bit caches whose scales lie beyond fp16's range, far apart, or between powers of two.

Tolerances.  Scores, biases and caps: as in test_gpu_attn_scored.py.  A weight that carries its value's scale has the scale's logarithm in its exponent: E = 64 (of a
scale up to 2^63) + 2 log2(e) cap + log2(e) (the largest bias) bounds what is added up there, in at most five roundings of 2^-24 E each (in powers of two, ln 2 of that of the
weight): 4 * 2^-24 E of a weight, and as much of their sum.  It is held in two bf16 numbers, 2^-16 of it, and outputs are rounded to fp16 once (test_gpu_attn_scales.py).
"""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from test_gpu_attn import unit
from test_gpu_attn_scales import RANGES, scaled, wanted
from test_gpu_attn_scored import BATCHES, Scored, attend, close, join_plan, some_parts

pytestmark = pytest.mark.gpu


# Scores of exactly 0 where scale / cap times a block's scale is more than floats hold -----------------------------------------------------

# one tile of 16 rows, two of them, two wavefronts' two, and many rows
ROWS = [([100, 0, 700], [1, 3, 2], (4, 2)), ([130], [6], (8, 2)), ([900], [12], (8, 2)), ([70, 0], [40, 50], (8, 2))]


FACTORS = [(2.0 ** -10, 2.0 ** 60), (50.0, 2.0 ** 74), (0.0, 2.0 ** 66)]


@pytest.mark.parametrize("hit,app,heads,cap,scale,dim,dtype", [(*rows, *factor, dim, [torch.bfloat16, torch.float16][(i + j + dim // 64) % 2]) for i, rows in enumerate(ROWS)
                                                               for j, factor in enumerate(FACTORS) for dim in (64, 128)])
def test_zero_products_under_factors_beyond_floats(hit, app, heads, dim, dtype, cap, scale):
    """Queries of zeros see all keys alike; with a cap, queries of one 1 give codes that are zeros a score of 0, and others the cap or its negative."""
    b = Scored(hit, app, 16, heads, dim, dtype, True, cap=cap, seed=9)
    b.scale = scale
    b.scales[0] = np.where(np.isnan(b.scales[0]), np.nan, 2.0 ** 63).astype(np.float32)
    b.q.zero_()
    if cap:
        b.q[::2, :, 5] = 1
        third = b.g.random(b.pools[0].shape[:3]) < 0.3
        b.pools[0][..., 5] = np.where(third & b.held[..., None], 0, b.pools[0][..., 5])
    w_out, w_lse, weight, reach = b.want()
    # (such scores are exact: what a product's sum may be off by does not count)
    close(b, *attend(b), (w_out, w_lse, weight, 0 * reach))


@pytest.mark.parametrize("hit,app,heads", ROWS)
@pytest.mark.parametrize("dim", [64, 128])
def test_scores_that_floats_hold_of_factors_that_they_do_not(hit, app, heads, dim):
    """Queries of 2^-120 over codes of 1/16 to 5/32 with scales of 2^62 and 2^63, times 2^66: scores of 32 to 40, of which a factor held to the largest float makes others."""
    b = Scored(hit, app, 16, heads, dim, torch.bfloat16, True, seed=4)
    b.scale = 2.0 ** 66
    low = b.g.random(b.scales[0].shape) < 0.5
    b.scales[0] = np.where(np.isnan(b.scales[0]), np.nan, np.where(low, 2.0 ** 62, 2.0 ** 63)).astype(np.float32)
    b.q.zero_()
    b.q[..., 5] = 2.0 ** -120
    # (codes of 1/16 times 1, 9/8, 10/8; twice that under the lower scale)
    codes = 0x18 + b.g.integers(0, 3, size=b.pools[0].shape[:3]) + 8 * low[:, None, :]
    b.pools[0][..., 5] = np.where(b.held[..., None], codes, 0x7F)
    close(b, *attend(b), b.want())


# Every block of K, of V or of both out of fp16's range, and scales between powers of two --------------------------------------------------

def other(b, cap, slopes, prefix, documents):
    """A batch of scaled() with other scores and a mask."""
    b.__class__ = Scored
    b.cap, b.prefix, b.documents, b.slopes = cap, prefix, documents, None
    if slopes:
        b.slopes = torch.exp2(-8 * torch.arange(1, b.q_heads + 1) / b.q_heads)
        b.slopes[0] = 0
    return b


def near(b, out, lse, want, some_within=False):
    """`some_within`: tiles of many rows whose scales are in fp16's range, where a weight is rounded to fp16 (2^-11 of it; of those below 2^-22 of the largest, up to 2^-33
    of that), beside others."""
    w_out, w_lse, weight, reach = want
    n = max(h + a for h, a in zip(b.hit, b.app))
    far = 0 if b.slopes is None else float(b.slopes.max()) * n
    e = 64 + 3 * b.cap + 1.45 * far
    ds = (b.dim + 16) * 2.0 ** -24 * reach + 2.0 ** -20 + 2.0 ** -20 * b.cap + 6 * 2.0 ** -24 * far + 4 * 2.0 ** -24 * e
    bound = (4 * ds[..., None] + n * 2.0 ** -24 + 2.0 ** -16) * weight + unit(b.dtype) * np.abs(w_out) * 1.01 + 2.0 ** -25
    if some_within:
        bound = bound + unit(b.dtype) * weight + n * 2.0 ** -33 * np.nanmax(np.abs(b.values()[1]))
    got, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.all(np.isfinite(got)), f"{np.sum(~np.isfinite(got))} outputs are not finite"
    over = np.abs(got - w_out) - bound
    assert over.max() <= 0, f"off by {np.abs(got - w_out).flat[over.argmax()]:.3g}, bound {bound.flat[over.argmax()]:.3g} at {np.unravel_index(over.argmax(), over.shape)}"
    empty = np.isneginf(w_lse)
    assert np.array_equal(np.isneginf(l), empty)
    assert np.all((np.abs(l - w_lse) <= 2 * ds + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(w_lse) + reach))[~empty])


# a row, three rows, two tiles of them, two wavefronts' two, and more than 64; the last one with keys in pieces
SHAPES = [([100, 0, 700], [1, 1, 1], (4, 4)), ([300], [3], (2, 2)), ([100, 410], [6, 5], (8, 2)), ([900], [12], (8, 2)), ([100, 0], [40, 90], (8, 2)), ([1200], [1], (8, 2)),
          ([2600], [33], (4, 2))]
SCORES = {
    "cap": dict(cap=3.0),
    "slopes": dict(slopes=True),
    "cap_slopes": dict(cap=6.0, slopes=True),
    "masks": dict(masked=True),
    "cap_slopes_masks": dict(cap=4.0, slopes=True, masked=True, window=90, sinks=3),
}


ALL_RANGES = RANGES + [((-30, 20), (-20, 12))]


# (three ranges for each shape and form, all of them for each shape and for each form)
@pytest.mark.parametrize("hit,app,heads,form,k_range,v_range,dim,powers", [(*shape, form, *ALL_RANGES[(i + j + 2 * k) % 5], *[(64, False), (128, True), (128, False)][(i + k) % 3])
                                                                           for i, shape in enumerate(SHAPES) for j, form in enumerate(SCORES) for k in range(3)])
def test_scales_beyond_fp16(hit, app, heads, dim, powers, k_range, v_range, form):
    kw = dict(SCORES[form])
    cap, slopes, masked = kw.pop("cap", 0.0), kw.pop("slopes", False), kw.pop("masked", False)
    some_within = (k_range, v_range) == ALL_RANGES[-1] and max(app) * heads[0] // heads[1] > 64
    # (codes times scales between powers of two would be rounded to fp16 there, too)
    b = scaled(hit, app, heads, dim, k_range, v_range, powers or some_within, **kw)
    total = [h + a for h, a in zip(hit, app)]
    b = other(b, cap, slopes, [t // 2 + 3 * i for i, t in enumerate(total)] if masked else None, [sorted({t // 3, max(0, t - 2)}) for t in total] if masked else None)
    if slopes and not cap and b.scale < 2.0 ** -64:
        with pytest.raises(K.KvlError) as e:
            attend(b)
        assert e.value.code == K.KVL_EINVAL
        return
    out, lse = attend(b)
    torch.cuda.synchronize()
    near(b, out, lse, wanted(b), some_within)


@pytest.mark.parametrize("form", SCORES)
@pytest.mark.parametrize("at", [5, 6])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scales_between_powers_of_two_many_rows(at, form, dtype):
    """Within fp16's range: codes times scale are rounded to the type once."""
    kw = dict(SCORES[form])
    masked = kw.pop("masked", False)
    total = [h + a for h, a in zip(*BATCHES[at][:2])]
    if masked:
        kw.update(prefix=[t // 2 for t in total], documents=[[t // 3, t - 2] for t in total])
    b = Scored(*BATCHES[at], dtype=dtype, e4m3=True, powers=False, spread=0.2, seed=at, **kw)
    close(b, *attend(b), b.want(), foreign=True)


# A bias without a cap in tiles of which it is no line --------------------------------------------------------------------------------------

# prefixes that end inside the tail, behind it and before it; first tokens in the tile where a window's keys go on, and some tiles before
FORMS = {
    "prefix_in_the_tail": dict(prefix=lambda h, a: h + a // 2),
    "prefix_behind_the_tail": dict(prefix=lambda h, a: h + a + 5),
    "prefix_before_the_tail": dict(prefix=lambda h, a: h // 2, window=40),
    "first_tokens": dict(window=37, sinks=3),
    "many_first_tokens": dict(window=50, sinks=70),
    "all": dict(window=33, sinks=5, prefix=lambda h, a: h + a // 3, documents=lambda h, a: sorted({h // 2, h + a // 4, h + a // 2})),
}


TYPES = [(torch.bfloat16, False), (torch.float16, True), (torch.bfloat16, True), (torch.float16, False)]


@pytest.mark.parametrize("at,form,dtype,e4m3", [(at, form, *t) for at in range(len(BATCHES)) for i, form in enumerate(FORMS) for t in (TYPES[:2] if (at + i) % 2 else TYPES[2:])])
def test_a_bias_that_is_no_line(at, form, dtype, e4m3):
    hit, app = BATCHES[at][:2]
    kw = {k: [v(h, a) for h, a in zip(hit, app)] if callable(v) else v for k, v in FORMS[form].items()}
    b = Scored(*BATCHES[at], dtype=dtype, e4m3=e4m3, seed=at, slopes=True, **kw)
    close(b, *attend(b), b.want())


# Joins -------------------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 2, 5, 16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_join_of_rows_with_infinite_or_nan_lses(n, dtype):
    """A row with an lse of +inf or NaN becomes NaN, its lse too; the others are as they were."""
    tokens, heads, dim = 9, 6, 64
    p = join_plan(tokens, heads, dim, dtype)
    parts, lses = some_parts(n, tokens, heads, dim, dtype, seed=n)
    parts = [x.cuda() for x in parts]
    out, lse = torch.zeros(tokens, heads, dim, dtype=dtype, device="cuda"), torch.zeros(tokens, heads, device="cuda")
    K.kvl_attn_join(p, parts, [l.cuda() for l in lses], out, lse)
    hurt = torch.zeros(tokens, heads, dtype=torch.bool)
    for i, (t, h, x) in enumerate([(0, 1, float("inf")), (2, 3, float("nan")), (2, 5, float("inf")), (5, 0, -float("nan")), (8, 2, float("inf"))]):
        lses[i % n][t, h] = x
        hurt[t, h] = True
    lses[-1][8, 2] = float("inf")           # (of two parts)
    got, got_lse = torch.zeros_like(out), torch.zeros_like(lse)
    K.kvl_attn_join(p, parts, [l.cuda() for l in lses], got, got_lse)
    hurt = hurt.cuda()
    assert bool(got[hurt].isnan().all()) and bool(got_lse[hurt].isnan().all())
    assert torch.equal(got[~hurt], out[~hurt]) and torch.equal(got_lse[~hurt], lse[~hurt])
