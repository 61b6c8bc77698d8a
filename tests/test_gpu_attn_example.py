"""The example that loads, appends and attends layer by layer: its last layers against the oracle's 64 bits, all of them against a run
in which every layer has a slot of its own."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import attn_oracle as O

pytestmark = pytest.mark.gpu


def load():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "layerwise_prefill.py")
    spec = importlib.util.spec_from_file_location("layerwise_prefill", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("eight_bit", [True, False])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_layers_loaded_appended_and_attended(eight_bit, window, sinks):
    hit, app, L = [100, 0, 37], [5, 40, 1], 5
    sizes = dict(layers=L, block_tokens=16, q_heads=8, kv_heads=2, head_dim=64, eight_bit=eight_bit, window=window, sinks=sinks, seed=3)
    example = load()
    r, apart = example.prefill(hit, app, slots=2, **sizes), example.prefill(hit, app, slots=L, **sizes)
    for x, y in zip(r["out"], apart["out"]):
        assert torch.equal(x, y)
    # Tolerance: weights and outputs are rounded to bf16, 2^-8 each at most; sums of 140 keys and of 64 products in 32 bits, with the exponential's
    # own error, are far below 2^-12 of the weights' sum (scores here are below 32).
    for layer in (L - 1, L - 2):
        pool = [x.cpu() for x in r["slots"][layer % 2]]
        if eight_bit:
            k, v = (O.e4m3_values(c.numpy()) * s.numpy().astype(np.float64)[:, None, :, None] for c, s in zip(pool[:2], pool[2:]))
        else:
            k, v = (x.double().numpy() for x in pool)
        want, _, weight, reach = O.attend(hit, app, r["tables"], 16, r["q"][layer].cpu().double().numpy(), k, v, r["scale"], "all", window, sinks)
        assert reach.max() < 32
        got = r["out"][layer].cpu().double().numpy()
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * (weight + np.abs(want)) + 2.0 ** -12 * weight)
