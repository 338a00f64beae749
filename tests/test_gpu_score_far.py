"""Log probabilities, entropies and alternatives of rows far from zero: a common
offset, whole rows at one large value, at a type's lowest and at its largest. They
depend on differences of logits only, so their bounds do too.

With m a row's largest logit, D the largest a (m - x) that counts (e^-104 is below
32 bits' range) and n terms:
  sum of exponentials: relative s = (n / 256 + 32) 2^-24 + (D + 4) 2^-22
  log probability: r = s + 2^-22 (a (m - x) + log n + 4)
  entropy: 2 s (H + 1) + 2^-22 (H + 1)
"""
import math

import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb

pytestmark = pytest.mark.gpu


def _rows(dtype, vocab):
    """(names, logits): one row a kind."""
    dt = eb.DTYPE[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    x = 4 * torch.randn(vocab, generator=g, device="cuda")
    low, high = torch.finfo(dt).min, torch.finfo(dt).max
    far = {f"offset {o:g}": x + o for o in (300.0, -300.0, 1e4, -1e4) + ((1e6, -1e6) if dtype != "f16" else ())}
    far |= {f"all {o:g}": torch.full_like(x, o) for o in (1e4, -1e4, low, high) + ((-1e6, -1e9, 1e30) if dtype != "f16"
                                                                                    else ())}
    two = torch.full_like(x, low)
    two[::3] = -3e4
    odd = torch.full_like(x, low)
    odd[vocab // 2] = -math.inf
    far |= {"two levels": two, "lowest and -inf": odd, "plain": x}
    return list(far), torch.stack([v.to(dt) for v in far.values()])


def _reference(x, target, scale):
    """In 64 bits, relative to the row's largest logit."""
    x = x.double()
    m = x.amax(1, keepdim=True)
    d = scale * (x - m)
    s = d.exp().sum(1, keepdim=True)
    logp = d - s.log()
    p = logp.exp()
    H = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    n = x.shape[1]
    D = (-d).masked_fill(-d > 104, 0.0).amax(1, keepdim=True)
    rel = (n / 256 + 32) * 2.0 ** -24 + (D + 4) * 2.0 ** -22
    return logp, p, H, rel, rel + 2.0 ** -22 * (-d + math.log(n) + 4)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [200, 40000])
@pytest.mark.parametrize("scale", [1.0, 1.25, 0.5])
def test_values(dtype, vocab, scale):
    names, x = _rows(dtype, vocab)
    target = (torch.arange(len(names), device="cuda") * 37) % vocab
    got = binding.token_logprobs(x, target, scale, top=8)
    logp, p, H, rel, r = _reference(x, target, scale)
    best = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :8]
    assert torch.equal(got.ids.long(), best)
    at = target[:, None]
    for k, name in enumerate(names):
        for have, where in ((got.logprob[k:k + 1], at[k]), (got.tops[k], best[k])):
            want, bound = logp[k, where], r[k, where]
            fin = torch.isfinite(want.float())
            err = (have.double() - want).abs()
            assert (err <= bound)[fin].all(), f"{name}: {have.tolist()} is not {want.tolist()}"
            assert (have[~fin] == -math.inf).all(), name
        tol = float((2 * rel[k] + 2.0 ** -22) * (H[k] + 1))
        assert abs(float(got.entropy[k]) - float(H[k])) <= tol, f"{name}: entropy {float(got.entropy[k])}, {float(H[k])}"
