"""What the binding of a pool's pages takes and refuses, before anything of it goes to a device (host only)."""
import numpy as np
import pytest

import paper_2602_21548_amd as K


class NoPools:
    """Pools that no call may come to."""

    @property
    def handle(self):
        raise AssertionError("the copies were taken")


@pytest.mark.parametrize("copies", [np.array([[-2 ** 63, 5]]), np.array([[2 ** 63, 5]], dtype=np.uint64), np.array([[5, 2 ** 64 - 1]], dtype=np.uint64), np.array([[5, -2 ** 31 - 1]]),
                                    np.array([[2 ** 31, 5]]), np.array([[2 ** 32, 5]]), [[-2 ** 63, 5]], [[5, 2 ** 63]], [[5, 2 ** 70]]])
def test_copies_of_blocks_that_32_bits_do_not_hold(copies):
    with pytest.raises(ValueError):
        K.kvl_copy_blocks(NoPools(), copies)
