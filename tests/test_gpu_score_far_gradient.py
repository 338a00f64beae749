"""Gradients of log probabilities and entropies in rows far from zero (those of
tests/test_gpu_score_far.py, with its bounds): p is off by the relative r, the
gradient by a p (|g| + |g_H| (|log p| + H + 2)) r and half a unit of its type's
last place."""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb
from test_gpu_score_far import _reference, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [200, 40000])
@pytest.mark.parametrize("scale", [1.0, 1.25, 0.5])
def test_gradients(dtype, vocab, scale):
    names, x = _rows(dtype, vocab)
    rows = len(names)
    target = (torch.arange(rows, device="cuda") * 37) % vocab
    got = binding.token_logprobs(x, target, scale)
    logp, p, H, rel, r = _reference(x, target, scale)
    gl = torch.linspace(-1.5, 2.0, rows, device="cuda")
    gh = torch.linspace(1.0, -0.75, rows, device="cuda")
    hit = torch.zeros_like(p)
    hit[torch.arange(rows, device="cuda"), target] = 1
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    for a, b in ((gl, gh), (gl, None), (None, gh), (torch.zeros_like(gl), None)):
        ga = torch.zeros(rows, 1, device="cuda", dtype=torch.float64) if a is None else a.double()[:, None]
        gb = torch.zeros(rows, 1, device="cuda", dtype=torch.float64) if b is None else b.double()[:, None]
        want = scale * (ga * (hit - p) - gb * (plogp + p * H[:, None]))
        mag = scale * (p * ga.abs() + gb.abs() * (plogp.abs() + p * (H[:, None] + 2)))
        bound = mag * r.masked_fill(p == 0, 0.0) + hit * ga.abs() * scale * 2.0 ** -22 + want.abs() * eb.HALF_ULP[dtype] * 1.01
        bound += {"f16": 2.0 ** -25, "bf16": 1e-38, "f32": 1e-38}[dtype]
        d = binding.token_logprobs_backward(x, target, got, a, b, scale)
        err = (d.double() - want).abs()
        for k, name in enumerate(names):
            assert (err[k] <= bound[k]).all(), f"{name}: worst {float(err[k].max())}, {d[k, :4].tolist()} {want[k, :4].tolist()}"
        # in place, and with gradients that start off the logits' 16-byte boundaries
        same = x.clone()
        binding.gptq2d_token_logprobs_backward(same, target, scale, got.lse, got.entropy, a, b, same)
        assert torch.equal(same, d)
        off = torch.full((rows, vocab + 3), 7.0, dtype=x.dtype, device="cuda")
        binding.gptq2d_token_logprobs_backward(x, target, scale, got.lse, got.entropy, a, b, off[:, 1:vocab + 1])
        assert torch.equal(off[:, 1:vocab + 1], d) and (off[:, 0] == 7).all() and (off[:, vocab + 1:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_in_place(dtype):
    """More rows than work groups a row: ordinary and far rows side by side."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = 4 * torch.randn(2500, 5000, generator=g, device="cuda")
    x[::7] -= 2e4
    x = x.to(eb.DTYPE[dtype])
    target = torch.randint(5000, (2500,), generator=g, device="cuda")
    got = binding.token_logprobs(x, target)
    one = torch.ones(2500, device="cuda")
    d = binding.token_logprobs_backward(x, target, got, one)
    total = d.double().sum(1).abs()  # a gradient of log probabilities sums to zero
    # rounding: half a unit of 16 bits of each entry, of which the target's is up to 1
    assert (total <= 2 * eb.HALF_ULP[dtype] + 1e-4).all(), float(total.max())
    same = x.clone()
    binding.gptq2d_token_logprobs_backward(same, target, 1.0, got.lse, got.entropy, one, None, same)
    assert torch.equal(same, d)
