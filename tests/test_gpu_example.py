"""The example end to end: rounded integers are held exactly, the cache holds
what the products gave, and the served scores are near the unrounded layer's."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import eightbit as eb  # noqa: E402

pytestmark = pytest.mark.gpu


def test_rounded_layer_is_served():
    import serve_rounded
    r = serve_rounded.run(width=128, heads=4, kv_heads=2, vocab=200, prompt=70, page_size=16)
    for n, m in r["rounded"].items():
        step = (m.blocks.values().double() / m.step)
        assert (step - m.Z.double()).abs().max() <= 2.0 ** -20 * 16, n  # the scale's product with the step rounds once
    assert torch.isfinite(r["served"].logprob).all()
    cache, table = r["cache"], r["table"]
    n = r["prompt"] + 8
    slots = cache.slots(table, torch.zeros(1, dtype=torch.int32, device="cuda"), n)
    k, v = cache.read(slots, torch.float32)
    for got, x in ((k, r["k"]), (v, r["v"])):
        t = x.double().view(n, cache.heads, cache.dim)
        s = eb.scale_of(t.abs().amax(-1))
        assert torch.equal(got.double().view_as(t), (eb.codes_of(t, s[..., None]) * s[..., None]).float().double())
    # log probabilities follow the unrounded layer's
    a, b = r["served"].logprob.double(), r["unrounded"]
    assert torch.corrcoef(torch.stack([r["logits"].double().flatten(), r["reference"].flatten()]))[0, 1] > 0.9
    assert (a - b).abs().mean() < 2.0
    assert (r["served"].tops[:, 0] >= r["served"].logprob - 1e-5).all()
