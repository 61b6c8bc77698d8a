"""The largest blocks that one copy takes: as many lanes as a launch holds, in vectors of 16, 4 and 1 bytes."""
import pytest
import torch

import paper_2602_21548_amd as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,shift,taken,refused", [
    (1 << 32, 0, 15, 16),               # 2^28 + 256 lanes a layer
    (1 << 32, 4, 3, 4),                 # 2^30 + 256
    ((1 << 31) + 1, 0, 1, 2),           # 2^31 + 257
])
def test_the_largest_blocks(size, shift, taken, refused):
    """Layers are the same memory here: what it holds is copied to the same places from each."""
    whole = torch.zeros(2 * size + shift + 8, dtype=torch.uint8, device="cuda")
    plane = whole[shift:shift + 2 * size]
    for at in (0, 1 << 20, size // 2 + 5, size - 4096):
        plane[at:at + 4096] = torch.randint(1, 256, (4096,), dtype=torch.uint8, device="cuda")
    with K.kvl_page_pools([size], 2, [[plane]] * refused) as pools:
        with pytest.raises(K.KvlError) as e:
            K.kvl_copy_blocks(pools, [[0, 1]])
        assert e.value.code == K.KVL_ERANGE
    assert not plane[size:].any()
    with K.kvl_page_pools([size], 2, [[plane]] * taken) as pools:
        K.kvl_copy_blocks(pools, [[0, 1]])
    torch.cuda.synchronize()
    assert torch.equal(plane[:size], plane[size:]) and bool(plane[0] != 0)
    assert not whole[:shift].any() and not whole[shift + 2 * size:].any()
