"""Other scores over 8-bit caches whose scales lie far beyond fp16's range.  Tolerances are those of test_gpu_attn_scored.py."""
import numpy as np
import pytest
import torch

from test_gpu_attn_scored import Scored, attend, close

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
