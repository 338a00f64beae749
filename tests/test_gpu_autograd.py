"""The conveniences that take part in autograd give the gradients of the C entry
points, to the bit, and those that would be lost are refused."""
import pytest
import torch

from paper_2607_27042_amd import binding

import eightbit as eb

pytestmark = pytest.mark.gpu


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (70, 130, 257), (3, 16, 128)])
def test_linear(M, N, K, dtype):
    dt = eb.DTYPE[dtype]
    w = _randn(1, N, K) / K ** 0.5
    for pow2 in (False, True):
        W, WT = binding.block_quantize(w, pow2=pow2), binding.block_quantize(w, pow2=pow2, transposed=True)
        turned = W.transposed()
        assert torch.equal(turned.codes.view(torch.uint8), WT.codes.view(torch.uint8)) and torch.equal(turned.scales, WT.scales)
        x, g = _randn(2, M, K, dtype=dt), _randn(3, M, N, dtype=dt)
        plain = binding.block_linear(x, W, pow2)
        assert not plain.requires_grad
        want, _ = binding.block_linear_backward(g, x, WT, pow2)
        for wt in (None, WT):
            leaf = x.clone().requires_grad_()
            Y = binding.block_linear(leaf, W, pow2, WT=wt)
            assert torch.equal(Y, plain)
            Y.backward(g)
            assert torch.equal(leaf.grad, want)
        # as part of a graph, with a gradient that is an expanded view, and under no_grad
        leaf = x.clone().requires_grad_()
        (binding.block_linear(2 * leaf, W, pow2) * 0.5).sum().backward()
        want, _ = binding.block_linear_backward(torch.full_like(g, 0.5), x, WT, pow2)
        assert torch.equal(leaf.grad, 2 * want)
        with torch.no_grad():
            assert not binding.block_linear(leaf, W, pow2).requires_grad
    with pytest.raises(ValueError, match="WT must be"):
        binding.block_linear(x, W, WT=W)
    with pytest.raises(ValueError, match="tiles of 128"):
        binding.block_quantize(w, 1).transposed()


def test_linear_on_a_stream():
    w, x = _randn(1, 60, 200), _randn(2, 20, 200).requires_grad_()
    W = binding.block_quantize(w)
    want = binding.block_linear(x, W)
    grad, = torch.autograd.grad(want.sum(), x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Y = binding.block_linear(x, W, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    got, = torch.autograd.grad(Y.sum(), x)
    torch.cuda.synchronize()
    assert torch.equal(Y, want) and torch.equal(got, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores(dtype):
    x = _randn(1, 20, 700, dtype=eb.DTYPE[dtype])
    target = torch.randint(-1, 700, (20,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    gl, gh = _randn(2, 20), _randn(3, 20)
    plain = binding.token_logprobs(x, target, 1.5, top=4)
    for a, b in ((gl, gh), (gl, None), (None, gh)):
        leaf = x.clone().requires_grad_()
        s = binding.token_logprobs(leaf, target, 1.5, top=4)
        assert all(torch.equal(u, v) for u, v in zip(s, plain)) and not s.ids.requires_grad
        ((0 if a is None else (s.logprob * a).sum()) + (0 if b is None else (s.entropy * b).sum())).backward()
        assert torch.equal(leaf.grad, binding.token_logprobs_backward(x, target, plain, a, b, 1.5))
    leaf = x.clone().requires_grad_()
    s = binding.token_logprobs(leaf, target)
    s.logprob.mean().backward()  # (an expanded gradient)
    one = torch.full((20,), 1 / 20, device="cuda")
    assert torch.equal(leaf.grad, binding.token_logprobs_backward(x, target, binding.token_logprobs(x, target), one))
    # no target: a log probability is a constant
    leaf = x.clone().requires_grad_()
    binding.token_logprobs(leaf).logprob.sum().backward()
    assert (leaf.grad == 0).all()
    assert not any(t.requires_grad for t in plain)
    with torch.no_grad():
        assert not binding.token_logprobs(leaf, target).logprob.requires_grad
    for lost in ("lse", "tops"):
        with pytest.raises(RuntimeError, match="not of lse or tops"):
            getattr(binding.token_logprobs(leaf, target, top=2), lost).sum().backward()


def test_a_layer_and_its_scores():
    """Together, against differences of the loss where the layer is linear: inputs and
    weights that eight bits hold."""
    ints = lambda seed, *s: torch.randint(-4, 5, s, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    x, w = ints(1, 5, 130).float(), ints(2, 30, 130).float()
    W = binding.block_quantize(w, pow2=True)
    target = torch.tensor([3, 0, 29, 7, 7], device="cuda")
    leaf = x.clone().requires_grad_()
    loss = lambda v: binding.token_logprobs(binding.block_linear(v, W, pow2=True), target, 2.0 ** -6).logprob.double().sum()
    loss(leaf).backward()
    for i, j in ((0, 0), (4, 129), (2, 64)):
        up, down = x.clone(), x.clone()
        up[i, j] += 1
        down[i, j] -= 1
        # A step of 1 moves z by 4 / 64 at most, so the third difference is below (2 / 16)^3 / 6; values are
        # good to 1e-5; the gradient of a row's logits, 2 / 64 in all, is rounded to e4m3 by 2^-4 and meets
        # weights up to 4.
        bound = 2.0 ** -9 / 6 + 1e-5 + 4 * 2.0 ** -4 * 2.0 ** -5
        assert abs((float(loss(up)) - float(loss(down))) / 2 - float(leaf.grad[i, j])) <= bound
