"""Appending where test_gpu_attn.py does not go: stored scales out of their range."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as O
from test_gpu_attn import Batch, appended, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stored", [0.0, 2.0 ** -40, 2.0 ** -33, -1.0, float("nan"), float("inf"), 2.0 ** 70])
@pytest.mark.parametrize("spread", [0.0, 2.0 ** -24, 1.0])
def test_stored_scales_are_taken_as_attention_takes_them(stored, spread):
    """Held codes keep what they stand for to attention, whatever scale was there, and the scale that is written is in the range."""
    b = Batch([3, 20], [2, 1], 16, (2, 2), 64, torch.bfloat16, True, hold="hit", rope_dim=32)
    b.k, b.v = (b.k * spread).to(b.dtype), (b.v * spread).to(b.dtype)
    for x in range(2):
        b.scales[x][[b.tables[0][0], b.tables[1][1]]] = stored
    _, planes = appended(b)
    for x, new in ((0, turned(b, b.k)), (1, b.v.double().numpy())):
        pool, scales = b.pools[x].copy(), b.scales[x].astype(np.float64)
        O.append(b.hit, b.app, b.tables, 16, new, pool, scales)
        got = planes[2 + x].double().cpu().numpy()
        assert np.array_equal(got, scales, equal_nan=True)
        touched = got[[b.tables[0][0], b.tables[1][1]]]
        assert np.all((touched >= 2.0 ** -32) & (touched <= 2.0 ** 63))
        assert np.array_equal(O.e4m3_values(planes[x].cpu().numpy()), O.e4m3_values(pool), equal_nan=True)
