"""The attention operators' calls through the binding's module: what is plainly in order is taken, with the same results as by the
general path, and the rest is left to it."""
import numpy as np
import pytest
import torch

import paper_2602_21548_amd as K
from paper_2602_21548_amd import attn as A
from paper_2602_21548_amd import binding as B

NOT_TAKEN = 1
pytestmark = pytest.mark.skipif(B._native is None, reason="the module is not built here")


def make(flags, requests=3, rope_dim=64):
    layout = K.make_attn_layout(block_tokens=16, q_heads=4, kv_heads=2, head_dim=64, pool_blocks=24, dtype=torch.bfloat16,
                                cache_dtype=torch.float8_e4m3fn, rope_dim=rope_dim)
    hit, app = np.array([20, 0, 33][:requests], dtype=np.uint32), np.array([3, 40, 1][:requests], dtype=np.uint32)
    tables = [np.arange(8 * r, 8 * r + 8, dtype=np.int32) for r in range(requests)]
    return K.kvl_attn_plan(layout, hit, app, tables, flags | K.KVL_TOKENS_ALL)


def test_what_is_not_in_order_is_left_to_the_general_path():
    plan = make(K.KVL_GATHER | K.KVL_SCATTER | K.KVL_HOST_ONLY)
    x = torch.zeros(plan.tokens, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(plan.tokens, 2, 64, dtype=torch.bfloat16)
    planes = [torch.zeros(24 * 16 * 128, dtype=torch.uint8)] * 2 + [torch.zeros(48)] * 2
    for args in [(plan, x, planes, x, None, None, None, None), (None, x, planes, x, None, None, None, None), (plan, x, planes), ()]:
        assert A._fast_attn(*args) == NOT_TAKEN
    for args in [(plan, kv, kv, planes, None, None, None, None), ("p", kv, kv, planes, None, None, None, None), (plan,)]:
        assert A._fast_append(*args) == NOT_TAKEN
    with pytest.raises(TypeError):
        K.kvl_attn_layer(plan, x, planes, x)
    with pytest.raises(ValueError):
        K.kvl_append_layer(plan, kv, kv, planes[:2])
    plan.destroy()
    plan.destroy()
    with pytest.raises(ValueError):
        plan.handle


def inputs(plan):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    n = plan.tokens
    qkv = torch.randn(n, 8, 64, device="cuda", generator=gen).bfloat16()
    planes = [torch.randn(24, 16, 2, 64, device="cuda", generator=gen).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
    planes += [torch.ones(24, 2, device="cuda") for _ in range(2)]
    rope = torch.randn(80, 32, 2, device="cuda", generator=gen)
    workspace = torch.empty(max(256, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    return qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], planes, rope, workspace


@pytest.mark.gpu
def test_each_argument_out_of_order_is_left_to_the_general_path():
    """One at a time, the others in order."""
    plan, gone = (make(K.KVL_GATHER | K.KVL_SCATTER) for _ in range(2))
    gone.destroy()
    q, k, v, planes, rope, workspace = inputs(plan)
    n = plan.tokens
    out, lse = torch.zeros(n, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 4, device="cuda")
    short = [planes[0].flatten()[:-1], *planes[1:]]
    bad_planes = [None, [], planes[:3], short, [None] * 4, iter(planes), [p.cpu() for p in planes]]
    bad_rows = [None, 7, out.cpu(), out.float(), out.half(), out[:-1], out[:, :3], out[..., :32], out.flatten(), out.transpose(1, 2),
                torch.zeros(n, 4, 128, dtype=torch.bfloat16, device="cuda")[..., ::2], torch.zeros(n, 260, dtype=torch.bfloat16, device="cuda")[:, 4:].unflatten(1, (4, 64)),
                torch.zeros(n * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(n, 4, 64), out[:1].expand(n, 4, 64)]
    calls = [(A._fast_attn, [plan, q, planes, out, workspace, 0.125, lse, None],
              {0: [None, gone, "p"], 1: bad_rows, 2: bad_planes, 3: bad_rows, 4: [7, workspace.cpu(), workspace[::2]], 5: [1, "1"],
               6: [lse.half(), lse[:-1], lse.t(), lse.cpu(), out], 7: ["s", 1.5]}),
             (A._fast_append, [plan, k, v, planes, rope, q, out, None],
              {0: [None, gone], 1: [None, q, k.cpu(), k.float(), k[:-1]], 2: [None, q], 3: bad_planes,
               4: [None, rope.double(), rope[:, :16], rope.cpu(), rope.transpose(0, 1), rope.flatten()],
               5: bad_rows, 6: bad_rows[1:], 7: ["s"]})]
    for call, args, bad in calls:
        assert call(*args) == K.KVL_OK, call
        for at, values in bad.items():
            for x in values:
                assert call(*args[:at], x, *args[at + 1:]) == NOT_TAKEN, (call, at, type(x), getattr(x, "shape", x))
        assert call(*args[:-1]) == NOT_TAKEN
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("requests", [3, 1])
def test_both_ways_give_the_same(requests, monkeypatch):
    plan = make(K.KVL_GATHER | K.KVL_SCATTER, requests)
    q, k, v, planes, rope, workspace = inputs(plan)
    taken, results = [], []
    for way in ("module", "general"):
        for f in ("_fast_append", "_fast_attn"):
            def spied(*a, call=getattr(A, f)):
                rc = call(*a)
                taken.append(rc)
                return rc
            monkeypatch.setattr(A, f, spied if way == "module" else lambda *a: NOT_TAKEN)
        side = torch.cuda.Stream()
        for stream in (None, side, side.cuda_stream):
            mine = [p.clone() for p in planes]
            turned = torch.zeros(plan.tokens, 4, 64, dtype=torch.bfloat16, device="cuda")
            out, lse = torch.zeros_like(turned), torch.zeros(plan.tokens, 4, device="cuda")
            torch.cuda.synchronize()
            K.kvl_append_layer(plan, k, v, mine, rope=rope, q=q, q_out=turned, stream=stream)
            K.kvl_attn_layer(plan, turned, mine, out, workspace, lse=lse, stream=stream)
            torch.cuda.synchronize()
            results.append([turned, out, lse, *mine])
    assert taken == [K.KVL_OK] * 6
    for other in results[1:]:
        for x, y in zip(results[0], other):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert bool(results[0][1].float().abs().max() > 0)


@pytest.mark.gpu
def test_the_librarys_refusals_come_through():
    plan = make(K.KVL_GATHER)                   # (not for appending)
    q, k, v, planes, rope, workspace = inputs(plan)
    with pytest.raises(K.KvlError) as e:
        K.kvl_append_layer(plan, k, v, planes, rope=rope)
    assert e.value.code == K.KVL_EINVAL
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(K.KvlError) as e:
            K.kvl_attn_layer(plan, q, planes, torch.zeros_like(q.contiguous()), workspace, scale=scale)
        assert e.value.code == K.KVL_EINVAL
    both = make(K.KVL_SCATTER)
    with pytest.raises(K.KvlError) as e:
        K.kvl_append_layer(both, k, v, planes, rope=rope[:39])        # (positions up to 39)
    assert e.value.code == K.KVL_ESPACE
    torch.cuda.synchronize()
