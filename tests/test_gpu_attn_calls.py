"""Calls of the attention operators: outputs in place of the queries."""
import pytest
import torch

import paper_2602_21548_amd as K
from test_gpu_attn import Batch, attend

pytestmark = pytest.mark.gpu


# one tile of rows; each kernel; keys cut into pieces; strided queries
@pytest.mark.parametrize("hit,app,heads", [([30, 0], [1, 1], (8, 2)), ([100], [6], (8, 2)), ([300], [12], (8, 2)), ([0, 31, 200], [200, 65, 33], (8, 4)),
                                           ([2500, 100], [1, 70], (8, 2)), ([1900], [70], (8, 1))])
@pytest.mark.parametrize("e4m3", [False, True])
def test_in_place(hit, app, heads, e4m3):
    b = Batch(hit, app, 16, heads, 128, torch.float16, e4m3)
    p, planes = b.plan(), b.planes()
    want, want_lse = attend(b, p, planes=planes)
    for wide in (False, True):
        q = b.q.cuda()
        if wide:
            room = torch.zeros(b.tokens, b.q_heads + 3, 128, dtype=b.dtype, device="cuda")
            room[:, 1:-2] = q
            q = room[:, 1:-2]
        out, lse = attend(b, p, q=q, out=q, planes=planes)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_in_place_with_another_stride_is_refused():
    b = Batch([30], [3], 16, (4, 2), 64)
    p, planes = b.plan(), b.planes()
    room = torch.zeros(6, 4, 64, dtype=b.dtype, device="cuda")
    for q, out in ((room[::2], room[:3]), (room[:3], room[::2])):
        with pytest.raises(K.KvlError) as e:
            K.kvl_attn_layer(p, q, planes, out)
        assert e.value.code == K.KVL_EINVAL
    torch.cuda.synchronize()
