"""Attention over 8-bit caches whose scales lie beyond fp16's range, or far apart: c * scale is what a code stands for, with any
scale from 2^-32 to 2^63, in the kernels for few rows and for many.

Tolerances.  Scores and what they are made of: as in test_gpu_attn.py.  A weight with its value's scale is held in two bf16 numbers, each off by at
most 2^-9 of what it has to hold: 2^-18 of the weight, 2^-16 with the roundings of the parts' difference and products.  Outputs are rounded to fp16 once: 2^-11 of them,
and half of fp16's least step, 2^-25, below its least normal.
"""
import numpy as np
import pytest
import torch

from test_gpu_attn import Batch, attend

pytestmark = pytest.mark.gpu


def scaled(hit, app, heads, dim, k_range, v_range, powers=True, seed=3, **kw):
    """A batch in fp16 over codes with scales 2^e, e from these ranges; values that keep outputs within fp16, scores of a few units."""
    b = Batch(hit, app, 16, heads, dim, torch.float16, True, seed=seed, **kw)
    for x, (lo, hi) in enumerate((k_range, v_range)):
        e = b.g.integers(lo, hi + 1, size=b.scales[x].shape)
        more = 1.0 if powers else 1 + 0.9 * b.g.random(b.scales[x].shape)
        b.scales[x] = np.where(np.isnan(b.scales[x]), np.nan, np.ldexp(more, e)).astype(np.float32)
        if x == 1:
            most = np.minimum(448.0, np.ldexp(1.0, 14 - e))[:, None, :, None]
            codes = torch.from_numpy(np.clip(b.g.standard_normal(b.pools[x].shape) * most / 3, -most, most)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            b.pools[x] = np.where(b.held[..., None, None], codes, b.pools[x])
    b.scale = float(np.float32(2.0 ** -k_range[1] / (60 * dim ** 0.5)))
    return b


def wanted(b):
    """The oracle's result with scales as they are taken: from 2^-32 to 2^63 (some of the ranges go beyond)."""
    b.scales = [np.clip(s, np.float32(2.0 ** -32), np.float32(2.0 ** 63)) for s in b.scales]
    return b.want()


def close(b, out, lse, want):
    w_out, w_lse, weight, reach = want
    n = max(h + a for h, a in zip(b.hit, b.app))
    ds = (b.dim + 16) * 2.0 ** -24 * reach + 2.0 ** -20
    bound = (4 * ds[..., None] + n * 2.0 ** -24 + 2.0 ** -16) * weight + 2.0 ** -11 * np.abs(w_out) * 1.01 + 2.0 ** -25
    got, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.all(np.isfinite(got)), f"{np.sum(~np.isfinite(got))} outputs are not finite"
    far = np.abs(got - w_out) - bound
    assert far.max() <= 0, f"off by {np.abs(got - w_out).flat[far.argmax()]:.3g}, bound {bound.flat[far.argmax()]:.3g} at {np.unravel_index(far.argmax(), far.shape)}"
    empty = np.isneginf(w_lse)
    assert np.array_equal(np.isneginf(l), empty)
    assert np.all((np.abs(l - w_lse) <= 2 * ds + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(w_lse) + reach))[~empty])


# (every block of K, of V or of both is out of fp16's range: no tile takes the other way)
RANGES = [((8, 20), (8, 13)), ((-32, -16), (-22, -16)), ((40, 63), (-3, 3)), ((-3, 3), (8, 12))]
MANY = [([100, 0], [40, 90], (8, 2)), ([1200], [33], (4, 2))]


@pytest.mark.parametrize("k_range,v_range", RANGES)
@pytest.mark.parametrize("hit,app,heads", MANY)
@pytest.mark.parametrize("dim,powers", [(64, True), (128, True), (128, False)])
def test_many_rows(hit, app, heads, dim, k_range, v_range, powers):
    b = scaled(hit, app, heads, dim, k_range, v_range, powers)
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, wanted(b))


@pytest.mark.parametrize("dim", [64, 128])
def test_many_rows_with_a_window_and_spoilt_values(dim):
    """Masks and a NaN among values beside such scales: rows that do not see it stay as they are."""
    b = scaled([70], [90], (4, 2), dim, (9, 20), (8, 12), window=60, sinks=2)
    at = 115
    b.pools[1][b.tables[0][at // 16], at % 16, :, 5] = 0xFF
    out, lse = attend(b)
    torch.cuda.synchronize()
    clean = np.array([i for i in range(90) if 70 + i < at or 70 + i - at >= 60])
    spoilt = np.setdiff1d(np.arange(90), clean)
    assert np.all(np.isnan(out.cpu().float().numpy()[spoilt][:, :, 5]))
    b.pools[1][b.tables[0][at // 16], at % 16, :, 5] = 0
    w_out, w_lse, weight, reach = wanted(b)
    keep = np.ones(w_out.shape, dtype=bool)
    keep[spoilt, :, 5] = False
    got = out.double().cpu().numpy()
    close(b, torch.from_numpy(np.where(keep, got, w_out)), lse, (w_out, w_lse, weight, reach))


# a tile of 16 rows, two of them, and two wavefronts' two
FEW = [([100, 0, 700], [1, 1, 1], (8, 2)), ([100, 410], [6, 5], (8, 2)), ([900], [12], (8, 2)), ([2600], [2], (8, 1))]


@pytest.mark.parametrize("k_range,v_range", RANGES + [((-30, 20), (-20, 12))])
@pytest.mark.parametrize("hit,app,heads", FEW)
@pytest.mark.parametrize("dim,powers", [(64, True), (128, True), (128, False)])
def test_few_rows(hit, app, heads, dim, k_range, v_range, powers):
    b = scaled(hit, app, heads, dim, k_range, v_range, powers)
    out, lse = attend(b)
    torch.cuda.synchronize()
    close(b, out, lse, wanted(b))


# The first blocks' values are zeros under a scale 2^34 times that of the others: what the others hold is all there is.
@pytest.mark.parametrize("app,heads", [(40, (8, 2)), (70, (2, 2))])
@pytest.mark.parametrize("dim", [64, 128])
def test_zeros_under_a_large_scale_many_rows(app, heads, dim):
    zeros_under_a_large_scale(app, heads, dim)


@pytest.mark.parametrize("app,heads", [(1, (8, 2)), (6, (8, 2)), (12, (8, 2))])
@pytest.mark.parametrize("dim", [64, 128])
def test_zeros_under_a_large_scale_few_rows(app, heads, dim):
    zeros_under_a_large_scale(app, heads, dim)


def zeros_under_a_large_scale(app, heads, dim):
    b = scaled([330], [app], heads, dim, (-3, 3), (-24, -24))
    for block in b.tables[0][:6]:
        b.pools[1][block], b.scales[1][block] = 0, 2.0 ** 10
    for block in b.tables[0][6:]:
        b.pools[1][block] = np.where(b.held[block][:, None, None], 0x70 + b.pools[1][block] % 15, 0x7F)     # (codes of 128 to 448)
    out, lse = attend(b)
    torch.cuda.synchronize()
    want = wanted(b)
    assert want[0].min() > 2.0 ** -18
    close(b, out, lse, want)
