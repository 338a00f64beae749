"""Log probabilities, entropies, alternatives and their gradient through the C
ABI against the plain 64-bit form.

Bounds (32-bit sums of n terms in chains of at most n / 256 + 32, exponentials
and logarithms within 2^-22, logits up to Z = max |z|):
  sum of exponentials: relative s = (n / 256 + 32) 2^-24 + (Z + 4) 2^-22
  lse, log probability: s + 2^-22 (Z + |lse|)
  entropy: 2 s (H + 1) + 2^-22 (H + 1)
  p: relative r = s + 2^-22 (Z + |lse| + 4); the gradient: a p (|g| + |g_H| (|log p| + H + 2)) r
      + half a unit of its type's last place (and of its smallest step)
"""
import math

import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(seed, rows, vocab, dtype, pad=0, offset=0, spread=4.0):
    x = spread * torch.randn(rows, vocab, generator=_gen(seed), device="cuda")
    buf = torch.full((rows, vocab + pad + offset), 1e4, dtype=eb.DTYPE[dtype], device="cuda")
    v = buf[:, offset:offset + vocab]
    v.copy_(x)
    return v


def forward(x, target, scale, top):
    rows, vocab = x.shape
    out = [torch.full((rows,), 77.0, device="cuda") for _ in range(3)]
    ids = torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None
    tops = torch.full((rows, top), 77.0, device="cuda") if top else None
    need = binding.gptq2d_token_logprobs_workspace_size(rows, vocab, top)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.gptq2d_token_logprobs(x, target, scale, *out, ids, tops, ws)
    return out + [ids, tops]


def order(x, top):
    """Tokens of the largest values, the lower first among equal ones (stable sort)."""
    return torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]


def check(x, target, scale, top):
    rows, n = x.shape
    lp, H, lse, ids, tops = forward(x, target, scale, top)
    z = x.double() * scale
    logp = torch.log_softmax(z, 1)
    p = logp.exp()
    ref_lse = torch.logsumexp(z, 1)
    ref_h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    Z = z.masked_fill(torch.isinf(z), 0).abs().amax(1)
    s = (n / 256 + 32) * 2.0 ** -24 + (Z + 4) * 2.0 ** -22
    b = s + 2.0 ** -22 * (Z + ref_lse.abs())
    assert ((lse - ref_lse).abs() <= b).all()
    assert ((H - ref_h).abs() <= 2 * s * (ref_h + 1) + 2.0 ** -22 * (ref_h + 1)).all()
    if target is not None:
        given = target >= 0
        want = logp.gather(1, target.clamp(min=0)[:, None])[:, 0]
        fin = given & torch.isfinite(want)
        assert ((lp - want).abs() <= b)[fin].all() and (lp[~given] == 0).all()
        assert (lp[given & ~fin] == -math.inf).all()
    else:
        assert (lp == 0).all()
    if top:
        best = order(x, top)
        assert torch.equal(ids.long(), best)
        want = logp.gather(1, best)
        fin = torch.isfinite(want)
        assert ((tops - want).abs() <= b[:, None])[fin].all() and (tops[~fin] == -math.inf).all()
    again = forward(x, target, scale, top)
    for u, v in zip((lp, H, lse, ids, tops), again):
        assert u is None or torch.equal(u, v), "the same call gave other bits"
    return lse, H


SIZES = [(1, 1), (3, 2), (2, 63), (5, 1000), (1, 4096), (2, 4097), (1, 32000), (300, 515), (7, 50257), (1, 262144),
         (1200, 300), (2, 16384 * 3 + 5)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_scores(rows, vocab, dtype):
    print(f"[score] {rows}x{vocab} {dtype}", flush=True)
    for k, (pad, offset, scale) in enumerate(((0, 0, 1.0), (3, 1, 0.7), (5, 7, 2.5))):
        x = _logits(rows + vocab + k, rows, vocab, dtype, pad, offset)
        target = torch.randint(-1, vocab, (rows,), generator=_gen(k), device="cuda")
        check(x, target, scale, min(vocab, (0, 1, 64)[k]))
    check(x, None, 1.0, min(vocab, 20))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "few", "zeros", "blocks"])
@pytest.mark.parametrize("rows,vocab", [(1, 60000), (3, 20000)])
def test_orders_that_are_hard_on_the_alternatives(rows, vocab, kind, dtype):
    i = torch.arange(vocab, device="cuda").float()
    x = {"rising": i / vocab * 50, "falling": -i / vocab * 50, "equal": torch.full_like(i, 2.5),
         "few": (i % 3) - 1, "zeros": torch.where(i % 2 == 0, 0.0, -0.0),
         "blocks": torch.where((i // 4096) % 2 == 0, 0.0, 30.0) + (i % 17) / 17}[kind]
    x = x.to(eb.DTYPE[dtype]).repeat(rows, 1)
    check(x, torch.full((rows,), vocab - 1, device="cuda"), 1.0, 64)
    check(x, torch.zeros(rows, dtype=torch.int64, device="cuda"), 1.0, 5)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [200, 40000])
def test_masked_logits(vocab, dtype):
    """-inf and the type's lowest value, alone and as whole rows."""
    x = _logits(1, 6, vocab, dtype)
    low = torch.finfo(x.dtype).min
    x[0, ::2] = -math.inf
    x[1, 1:] = -math.inf
    x[2, :-1] = low if dtype != "f32" else -3e38
    x[3, 10:] = -math.inf
    x[4, 3:] = low
    target = torch.tensor([0, 0, vocab - 1, 3, 2, 5], device="cuda")
    check(x, target, 1.0, 20)
    x[5] = -math.inf
    lp, H, lse, ids, tops = forward(x, target, 1.0, 20)
    assert lse[5] == -math.inf and H[5] == 0 and lp[5] == -math.inf and (tops[5] == -math.inf).all()
    assert ids[5].tolist() == list(range(20))
    assert lp[0] == -math.inf and abs(float(H[1])) < 1e-6 and float(lp[1]) == 0.0
    d = torch.full_like(x, 9.0)
    g = torch.ones(6, device="cuda")
    binding.gptq2d_token_logprobs_backward(x, target, 1.0, lse, H, g, g, d)
    assert (d[5] == 0).all() and torch.isfinite(d.float()).all()


@pytest.mark.parametrize("vocab", [100, 40000])
def test_rows_that_are_not_finite(vocab):
    x = _logits(1, 4, vocab, "f32")
    x[0, 7] = math.nan
    x[1, vocab - 1] = math.inf
    x[2, 3] = -math.nan
    lp, H, lse, ids, tops = forward(x, torch.zeros(4, dtype=torch.int64, device="cuda"), 1.0, 4)
    for t in (lp, H, lse):
        assert torch.isnan(t).tolist() == [True, True, True, False]
    assert ids[0, 0] == 7 and ids[1, 0] == vocab - 1 and ids[2, 0] == 3
    d = torch.zeros_like(x)
    binding.gptq2d_token_logprobs_backward(x, torch.zeros(4, dtype=torch.int64, device="cuda"), 1.0, lse, H,
                                           torch.ones(4, device="cuda"), None, d)
    assert torch.isnan(d[:3]).all() and torch.isfinite(d[3]).all()


def test_targets_outside():
    x = _logits(1, 3, 50, "f32")
    target = torch.tensor([50, -1, -(2 ** 40)], device="cuda")
    lp, H, lse, _, _ = forward(x, target, 1.0, 0)
    assert torch.isnan(lp[0]) and lp[1:].tolist() == [0, 0]
    d = torch.zeros_like(x)
    binding.gptq2d_token_logprobs_backward(x, target, 1.0, lse, H, torch.ones(3, device="cuda"), None, d)
    assert torch.isnan(d[0]).all() and (d[1:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 3), (5, 1000), (1, 50257), (64, 4097), (3000, 40)])
def test_gradient(rows, vocab, dtype):
    print(f"[score gradient] {rows}x{vocab} {dtype}", flush=True)
    for k, (pad, offset, scale) in enumerate(((0, 0, 1.0), (3, 1, 0.7))):
        x = _logits(rows * 3 + vocab + k, rows, vocab, dtype, pad, offset)
        target = torch.randint(-1, vocab, (rows,), generator=_gen(k), device="cuda")
        gl, gh = (torch.randn(rows, generator=_gen(10 + k + i), device="cuda") for i in range(2))
        _, H, lse, _, _ = forward(x, target, scale, 0)
        leaf = x.double().requires_grad_()
        logp = torch.log_softmax(leaf * scale, 1)
        given = (target >= 0).double()
        lp = logp.gather(1, target.clamp(min=0)[:, None])[:, 0] * given
        ent = -(logp.exp() * logp).sum(1)
        p, ref_h = logp.exp().detach(), ent.detach()
        for a, b in ((gl, gh), (gl, None), (None, gh)):
            leaf.grad = None
            ((0 if a is None else (lp * a).sum()) + (0 if b is None else (ent * b).sum())).backward(retain_graph=True)
            buf = torch.full((rows, vocab + 2 * pad + offset), 5.0, dtype=x.dtype, device="cuda")
            for o in {offset, 0}:
                d = buf[:, o:o + vocab]
                binding.gptq2d_token_logprobs_backward(x, target, scale, lse, H, a, b, d)
                Z = (x.double() * scale).abs().amax(1, keepdim=True)
                L = torch.logsumexp(x.double() * scale, 1, keepdim=True).abs()
                r = (vocab / 256 + 32) * 2.0 ** -24 + (Z + 4) * 2.0 ** -22 + 2.0 ** -22 * (Z + L + 4)
                ga = torch.zeros(rows, 1, device="cuda") if a is None else (a * given.float()).abs()[:, None]
                gb = torch.zeros(rows, 1, device="cuda") if b is None else b.abs()[:, None]
                mag = scale * p * (ga + gb * (logp.detach().abs() + ref_h[:, None] + 2))
                hit = torch.zeros_like(p)
                hit[torch.arange(rows, device="cuda"), target.clamp(min=0)] = 1
                bound = mag * r + hit * ga * scale * 2.0 ** -22 + leaf.grad.abs() * eb.HALF_ULP[dtype] * 1.01
                bound += {"f16": 2.0 ** -25, "bf16": 1e-38, "f32": 1e-38}[dtype]
                assert ((d.double() - leaf.grad).abs() <= bound).all()
            assert (buf[:, max(offset, 0) + vocab:] == 5.0).all()
        inplace = x.clone()
        binding.gptq2d_token_logprobs_backward(inplace, target, scale, lse, H, gl, gh, inplace)
        d = torch.empty_like(inplace)
        binding.gptq2d_token_logprobs_backward(x, target, scale, lse, H, gl, gh, d)
        assert torch.equal(inplace, d)


def test_gradient_against_differences():
    rows, vocab, h = 2, 30, 2.0 ** -6
    x = _logits(1, rows, vocab, "f32", spread=1.0)
    target = torch.tensor([3, 20], device="cuda")
    gl, gh = torch.tensor([1.5, -0.5], device="cuda"), torch.tensor([0.25, 2.0], device="cuda")

    def value(v):
        lp, H, _, _, _ = forward(v, target, 1.5, 0)
        return float((lp.double() * gl).sum() + (H.double() * gh).sum())
    _, H, lse, _, _ = forward(x, target, 1.5, 0)
    d = torch.empty_like(x)
    binding.gptq2d_token_logprobs_backward(x, target, 1.5, lse, H, gl, gh, d)
    for i, j in ((0, 3), (0, 0), (1, 20), (1, 29)):
        up, down = x.clone(), x.clone()
        up[i, j] += h
        down[i, j] -= h
        # third derivatives are below 40, 32-bit values are good to 1e-5
        assert abs((value(up) - value(down)) / (2 * h) - float(d[i, j])) <= 40 * h * h / 6 + 1e-5 / h


def test_stream_and_graph():
    x = _logits(1, 2, 40000, "bf16").contiguous()
    target = torch.tensor([5, 7], device="cuda")
    want = forward(x, target, 1.0, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = forward(x, target, 1.0, 8)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = [torch.empty(2, device="cuda") for _ in range(3)]
    ids, tops = torch.empty(2, 8, dtype=torch.int32, device="cuda"), torch.empty(2, 8, device="cuda")
    ws = torch.empty(max(256, binding.gptq2d_token_logprobs_workspace_size(2, 40000, 8)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.gptq2d_token_logprobs(x, target, 1.0, *out, ids, tops, ws)
    for seed in (2, 3, 4):
        x.copy_(_logits(seed, 2, 40000, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + [ids, tops], forward(x, target, 1.0, 8)))


def test_refusals():
    x = torch.zeros(2, 100, device="cuda")
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    v = [torch.zeros(2, device="cuda") for _ in range(3)]
    with pytest.raises(TypeError, match="one dtype"):
        binding.gptq2d_token_logprobs(x.double(), t, 1.0, *v)
    with pytest.raises(TypeError, match="target must be"):
        binding.gptq2d_token_logprobs(x, t.int(), 1.0, *v)
    with pytest.raises(binding.Gptq2dError, match="scale must be"):
        binding.gptq2d_token_logprobs(x, t, 0.0, *v)
    ids, tops = torch.zeros(2, 65, dtype=torch.int32, device="cuda"), torch.zeros(2, 65, device="cuda")
    with pytest.raises(binding.Gptq2dError, match="top must lie"):
        binding.gptq2d_token_logprobs(x, t, 1.0, *v, ids, tops)
    with pytest.raises(binding.Gptq2dError, match="top must lie"):
        binding.gptq2d_token_logprobs(x[:, :3], t, 1.0, *v, ids[:, :4].contiguous(), tops[:, :4].contiguous())
    big = torch.zeros(1, 60000, device="cuda")
    with pytest.raises(ValueError, match="workspace"):
        binding.gptq2d_token_logprobs(big, t[:1], 1.0, *[u[:1] for u in v])
    with pytest.raises(binding.Gptq2dError, match="no gradient"):
        binding.gptq2d_token_logprobs_backward(x, t, 1.0, v[0], v[1], None, None, x)
    with pytest.raises(TypeError, match="one dtype"):
        binding.gptq2d_token_logprobs_backward(x, t, 1.0, v[0], v[1], v[2], None, x.half())
