"""Calls of the attention operators: outputs in place of the queries, streams, plans that are dropped early."""
import pytest
import torch

import paper_2602_21548_amd as K
from test_gpu_attn import Batch, appended, attend, close, near_turned, turned

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


# Streams.  Everything is on the device and set up before; the stream in question then waits for a while, gets the real inputs by copies on the
# device, and runs the call, so that a launch on any other stream sees NaN.

class Ready:
    """A batch's tensors, outputs and workspace on the device, with NaN in place of the inputs that come late."""

    def __init__(self, b, flags):
        self.b, self.p = b, b.plan(flags)
        self.planes = b.planes()
        self.late = [(torch.full_like(x, float("nan"), device="cuda"), x.cuda()) for x in (b.q, b.k, b.v)]
        self.q, self.k, self.v = (x for x, _ in self.late)
        self.rope = None if b.rope is None else b.rope.cuda()
        self.turned, self.out = (torch.full_like(self.q, float("nan")) for _ in range(2))
        self.lse = torch.full((b.tokens, b.q_heads), float("nan"), device="cuda")
        self.ws = torch.full((max(64, self.p.workspace_bytes // 4),), float("nan"), device="cuda")

    def arrive(self):
        torch.cuda._sleep(20_000_000)
        for to, what in self.late:
            to.copy_(what)

    def append(self, **kw):
        K.kvl_append_layer(self.p, self.k, self.v, self.planes, self.rope, self.q, self.turned, **kw)

    def attend(self, q, **kw):
        K.kvl_attn_layer(self.p, q, self.planes, self.out, self.ws, scale=self.b.scale, lse=self.lse, **kw)


@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("hit,app,e4m3", [([2500, 300], [1, 2], True), ([100, 0], [1, 90], True), ([700, 5], [1, 1], False)])
def test_attention_runs_on_its_stream(hit, app, e4m3, named):
    r = Ready(Batch(hit, app, 16, (8, 2), 128, torch.bfloat16, e4m3), K.KVL_GATHER)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r.arrive()
        if not named:
            r.attend(r.q)
    if named:
        r.attend(r.q, stream=side)
    side.synchronize()
    close(r.b, r.out, r.lse, r.b.want())


@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_runs_on_its_stream(e4m3, named):
    b = Batch([100, 0, 31], [1, 90, 3], 16, (8, 2), 128, torch.bfloat16, e4m3, hold="hit", rope_dim=64)
    wanted = appended(b)
    r = Ready(b, K.KVL_SCATTER)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r.arrive()
        if not named:
            r.append()
    if named:
        r.append(stream=side)
    side.synchronize()
    for x, y in zip([r.turned, *r.planes], [wanted[0], *wanted[1]]):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("side", [False, True])
def test_plans_dropped_while_their_work_waits(side):
    """Both calls of many plans behind a wait, each plan dropped at once and the next one made: lists that are used again too early
    would be another batch's."""
    ready = []
    for seed in range(8):
        b = Batch([1500 + 100 * seed, 10 * seed], [1 + seed % 3, 3], 16, (8, 2), 64, torch.bfloat16, seed=seed, hold="hit", rope_dim=32)
        ready.append((b, Ready(b, K.KVL_GATHER | K.KVL_SCATTER)))
    for _, r in ready:
        for to, what in r.late:
            to.copy_(what)
        r.p.destroy()
    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    torch.cuda.synchronize()
    waits = torch.cuda.Event()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)
        for b, r in ready:
            r.p = b.plan(K.KVL_GATHER | K.KVL_SCATTER)
            r.append()
            r.attend(r.turned)
            r.p.destroy()
        waits.record()
    assert not waits.query()                    # (all of it was enqueued behind the wait)
    torch.cuda.synchronize()
    for b, r in ready:
        near_turned(r.turned, turned(b, b.q), b.q, b.dtype)
        b.q = r.turned.cpu()
        b.pools = [t.double().cpu().numpy() for t in r.planes]
        close(b, r.out, r.lse, b.want())
