"""Layer-wise prefill on a cached prefix: each layer's keys and values come out of pinned host memory into one of a few resident slots
while the layer before is computed; the computation appends the new tokens' rotated keys and values to the slot and attends over it.

    python examples/layerwise_prefill.py [--layers 8] [--cache 8|16] [--window 0] [--sinks 0]
"""
import argparse
import os
import sys

import numpy as np
import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_21548_amd as K  # noqa: E402


def make_batch(hit, app, block_tokens, seed=0):
    """(pool blocks, tables) of a batch: blocks of the pool in no order."""
    need = [(h + a + block_tokens - 1) // block_tokens for h, a in zip(hit, app)]
    blocks = sum(need) + 2
    order = np.random.default_rng(seed).permutation(blocks).astype(np.int32)
    at = np.cumsum([0] + need)
    return blocks, [order[x:y].copy() for x, y in zip(at[:-1], at[1:])]


def prefill(hit, app, layers=4, slots=2, block_tokens=64, q_heads=32, kv_heads=8, head_dim=128, eight_bit=True, window=0, sinks=0,
            dtype=torch.bfloat16, seed=0):
    """Runs it on synthetic contents.  Returns the outputs of each layer, what went in, and the slots as the last layers left them."""
    L, S, bs = layers, slots, block_tokens
    cache_dtype = torch.float8_e4m3fn if eight_bit else dtype
    row = kv_heads * head_dim * (1 if eight_bit else 2)
    blocks, tables = make_batch(hit, app, bs, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    # What a batch needs once, for all layers: the load's plan, the scales' (a float a head for each block), the attention's.
    layout = K.make_layout(L, bs, (row, row), blocks)
    scatter = K.kvl_plan(layout, hit, app, tables, K.KVL_SCATTER)
    gather = K.kvl_plan(layout, hit, app, tables, K.KVL_GATHER)
    held = [(h + bs - 1) // bs for h in hit]
    scale_layout = K.make_layout(L, 1, (4 * kv_heads, 4 * kv_heads), blocks)
    none = [0] * len(held)
    scale_scatter = K.kvl_plan(scale_layout, held, none, tables, K.KVL_SCATTER)
    scale_gather = K.kvl_plan(scale_layout, held, none, tables, K.KVL_GATHER)
    attn_layout = K.make_attn_layout(block_tokens=bs, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, pool_blocks=blocks, dtype=dtype,
                                     cache_dtype=cache_dtype, window=window, sinks=sinks, rope_dim=head_dim)
    plan = K.kvl_attn_plan(attn_layout, hit, app, tables, K.KVL_SCATTER | K.KVL_GATHER | K.KVL_TOKENS_ALL)
    workspace = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda") if plan.workspace_bytes else None
    positions = max([h + a for h, a in zip(hit, app)] + [1])
    frequency = 10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device="cuda") / head_dim)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * frequency
    rope = torch.stack([angle.cos(), angle.sin()], dim=-1).float()

    # The cached prefix of each layer, in pinned host memory; the new tokens' queries, keys and values, one projection's output.
    def planes(make):
        return [make(blocks, bs, kv_heads, head_dim, dtype=torch.uint8 if eight_bit else dtype, device="cuda") for _ in range(2)]

    def scale_planes():
        return [torch.ones(blocks, kv_heads, device="cuda") for _ in range(2)] if eight_bit else []

    host, host_scales, qkv, out = [], [], [], []
    for _ in range(L):
        source = [torch.randn(blocks, bs, kv_heads, head_dim, device="cuda", generator=gen) for _ in range(2)]
        source = [x.to(cache_dtype).view(torch.uint8) if eight_bit else x.to(dtype) for x in source]
        host.append(torch.empty(gather.payload_bytes, dtype=torch.uint8, pin_memory=True))
        K.kvl_pack_layer(gather, source, host[-1])
        host_scales.append(torch.empty(scale_gather.payload_bytes, dtype=torch.uint8, pin_memory=True))
        if eight_bit:
            scales = [torch.exp2(torch.randint(-3, 2, (blocks, kv_heads), device="cuda", generator=gen).float()) for _ in range(2)]
            K.kvl_pack_layer(scale_gather, scales, host_scales[-1])
        qkv.append(torch.randn(plan.tokens, q_heads + 2 * kv_heads, head_dim, device="cuda", generator=gen).to(dtype))
        out.append(torch.empty(plan.tokens, q_heads, head_dim, device="cuda", dtype=dtype))
    resident = [planes(torch.zeros) for _ in range(S)]
    resident_scales = [scale_planes() for _ in range(S)]
    torch.cuda.synchronize()

    def compute(layer, slot, stream):
        """One layer's attention on the compute stream, once the layer's prefix is in its slot."""
        pool = resident[slot] + resident_scales[slot]
        if eight_bit:
            K.kvl_unpack_layer(scale_scatter, host_scales[layer], resident_scales[slot], stream=stream)
        q, k, v = qkv[layer].split([q_heads, kv_heads, kv_heads], dim=1)
        K.kvl_append_layer(plan, k, v, pool, rope=rope, q=q, stream=stream)         # (the queries are rotated where they are)
        K.kvl_attn_layer(plan, q, pool, out[layer], workspace, stream=stream)

    streams = [torch.cuda.Stream() for _ in range(3)]
    stats = K.kvl_stream_layers(scatter, host, resident, None, 0, 0, *streams, n_layers=L, compute=compute)
    torch.cuda.synchronize()
    return {"out": out, "q": [x[:, :q_heads] for x in qkv], "tables": tables, "slots": [a + b for a, b in zip(resident, resident_scales)],
            "stats": stats, "scale": head_dim ** -0.5}


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--layers", type=int, default=8)
    p.add_argument("--cache", choices=["8", "16"], default="8")
    p.add_argument("--window", type=int, default=0)
    p.add_argument("--sinks", type=int, default=0)
    a = p.parse_args()
    rng = np.random.default_rng(1)
    hit, app = rng.integers(1000, 8000, 8).tolist(), rng.integers(64, 512, 8).tolist()
    r = prefill(hit, app, layers=a.layers, eight_bit=a.cache == "8", window=a.window, sinks=a.sinks)
    s = r["stats"]
    print(f"{a.layers} layers, {sum(hit)} cached and {sum(app)} new tokens: {s['total_ms']:.2f} ms, {s['h2d_bytes'] / 1e6:.0f} MB loaded at "
          f"{s['link_gbps']:.1f} GB/s, {s['exposed_ms']:.2f} ms of it not under the computation")


if __name__ == "__main__":
    main()
