"""The example's calibration: what each matrix takes in and the gradient at what it
gives out are those of the layer in 64 bits, which torch differentiates."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_calibration_is_the_layer():
    import serve_rounded
    gen = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    vocab, width, kv_heads, heads, seqs, t = 150, 64, 2, 4, 3, 20
    dim = width // heads
    weights = {"q": randn(width, width), "k": randn(kv_heads * dim, width), "v": randn(kv_heads * dim, width),
               "o": randn(width, width), "head": 4 * randn(vocab, width)}
    weights = {n: w / width ** 0.5 for n, w in weights.items()}
    embed = randn(vocab, width)
    tokens, target = (torch.randint(vocab, (seqs, t), generator=gen, device="cuda") for _ in range(2))
    seen = serve_rounded.calibrate(weights, embed, tokens, target, kv_heads)

    w = {n: m.double() for n, m in weights.items()}
    x = embed.double()[tokens.flatten()]
    out = {n: (x @ w[n].T).requires_grad_() for n in "qkv"}
    rows = []
    for b in range(seqs):  # one sequence and head at a time
        s = slice(b * t, b * t + t)
        for h in range(heads):
            c, kc = slice(h * dim, h * dim + dim), slice(h // (heads // kv_heads) * dim, (h // (heads // kv_heads) + 1) * dim)
            z = out["q"][s, c] @ out["k"][s, kc].T * dim ** -0.5
            z = z.masked_fill(~torch.ones(t, t, dtype=torch.bool, device="cuda").tril(), float("-inf"))
            rows.append(torch.softmax(z, 1) @ out["v"][s, kc])
    a = torch.stack(rows).view(seqs, heads, t, dim).transpose(1, 2).reshape(seqs * t, width)
    out["o"] = a @ w["o"].T
    h = x + out["o"]
    out["head"] = h @ w["head"].T
    for n in ("o", "head"):
        out[n].retain_grad()
    torch.log_softmax(out["head"], 1).gather(1, target.flatten()[:, None]).sum().backward()
    inputs = {"q": x, "k": x, "v": x, "o": a, "head": h}
    assert seen.keys() == weights.keys()
    for n, (rows_in, gradient) in seen.items():
        assert not rows_in.requires_grad
        # 32 bits: sums of 64 terms up to about ten
        assert (rows_in.double() - inputs[n]).abs().max() <= 1e-4, n
        # eight bits in the head's product and in its gradient (2^-4 of a value at most, 3 % on average; logits
        # are off by 0.2 of 4 or so, probabilities by a fifth): directions agree
        assert gradient.shape == out[n].shape
        cosine = float((gradient.double() * out[n].grad).sum() / (gradient.double().norm() * out[n].grad.norm()))
        assert cosine >= 0.95, (n, cosine)
        ratio = float(gradient.double().norm() / out[n].grad.norm())
        assert 0.9 <= ratio <= 1.1, (n, ratio)
