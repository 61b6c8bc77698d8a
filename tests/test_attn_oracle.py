"""The attention oracle's rules that its other tests leave out."""
import numpy as np
import pytest

from oracle import attn_oracle as O


@pytest.mark.parametrize("stored,taken", [(0.0, 2.0 ** -32), (2.0 ** -40, 2.0 ** -32), (-1.0, 2.0 ** -32), (float("nan"), 2.0 ** -32), (2.0 ** -32, 2.0 ** -32),
                                          (0.3, 0.3), (2.0 ** 63, 2.0 ** 63), (2.0 ** 70, 2.0 ** 63), (float("inf"), 2.0 ** 63)])
def test_held_codes_keep_what_they_stand_for(stored, taken):
    """A new row that needs no larger scale leaves the codes and writes the scale as it is taken; one that does moves them to the new one."""
    assert O.taken_scale(stored) == taken
    codes = np.array([1, 8, 126, 0x80 | 50], dtype=np.uint8)
    for new in (0.0, 200.0 * 2.0 ** 20):
        pool, scales = np.full((1, 4, 1, 4), 0x7F, dtype=np.uint8), np.array([[stored]])
        pool[0, :2, 0] = codes
        O.append([2], [1], [np.array([0])], 4, np.full((1, 1, 4), new), pool, scales)
        assert scales[0, 0] == max(taken, O.least_scale(new))
        kept = O.e4m3_values(pool[0, :2, 0]) * scales[0, 0]
        want = O.e4m3_values(codes) * taken
        assert np.all(np.abs(kept - want) <= np.abs(want) * 2.0 ** -4 + 2.0 ** -10 * (scales[0, 0] if scales[0, 0] != taken else 0))
