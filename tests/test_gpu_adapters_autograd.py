"""adapters in autograd, by itself and beside block_linear."""
import pytest
import torch

from paper_2607_27042_amd import binding as g

pytestmark = pytest.mark.gpu


def problem(M=70, N=96, K=64, R=8, count=3, dtype=torch.bfloat16, seed=0):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=r, device="cuda")
    X, Y = randn(M, K).to(dtype), randn(M, N).to(dtype)
    A, B = (randn(count, R, K) * K ** -0.5).to(dtype), (randn(count, N, R) * R ** -0.5).to(dtype)
    index = torch.randint(-1, count, (M,), generator=r, device="cuda", dtype=torch.int32)
    return X, A, B, Y, torch.rand(count, generator=r, device="cuda") + 0.5, index, randn(M, N).to(dtype)


def plain(X, A, B, Y, scales, index):
    a = index.clamp(min=0).long()
    h = torch.matmul(A[a], X.unsqueeze(2))
    o = torch.matmul(B[a], h)[..., 0] * scales[a].unsqueeze(1)
    return Y + torch.where((index >= 0).unsqueeze(1), o, 0.0)


@pytest.mark.parametrize("dtype,half", [(torch.float32, 2.0 ** -24), (torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
def test_gradients(dtype, half):
    X, A, B, Y, scales, index, G = problem(dtype=dtype)
    leaves = [t.clone().requires_grad_() for t in (X, A, B, Y)]
    groups = g.adapter_groups(index, A.shape[0])
    O = g.adapters(*leaves[:3], groups, leaves[3], scales)
    O.backward(G)
    exact = [t.double().cpu().requires_grad_() for t in (X, A, B, Y)]
    o = plain(*exact, scales.double().cpu(), index.cpu())
    o.backward(G.double().cpu())
    # one rounding of a sum of at most 96 + 64 + 70 terms in 32 bits, and of h or p held to 2^-16 (relative to
    # the largest of a row's, by which sums of a few terms are judged)
    for a, e in zip((O, *(t.grad for t in leaves)), (o, *(t.grad for t in exact))):
        a, e = a.detach().double().cpu(), e.detach()
        off = half * e.abs() + (2.0 ** -24 * 230 + (2.0 ** -16 if half > 2.0 ** -20 else 0.0)) * 16 * e.abs().max()
        assert bool(((a - e).abs() <= off).all()), ((a - e).abs() / off).max()
    assert torch.equal(leaves[3].grad, G)


def test_which_gradients():
    """Only what is asked for; an expanded gradient; no gradient where none is enabled; scales have none."""
    X, A, B, Y, scales, index, G = problem()
    groups = g.adapter_groups(index, A.shape[0])
    full = g.adapters(X, A, B, groups, Y, scales)
    with torch.no_grad():
        assert torch.equal(g.adapters(X.requires_grad_(), A, B, groups, Y, scales), full)
    X.requires_grad_(False)
    ones = g.adapters_backward(torch.ones_like(full), X, A, B, groups, None, scales, wants=(True, True, False))
    for i in range(2):
        leaf = (X, A)[i].clone().requires_grad_()
        g.adapters(*((leaf, A) if i == 0 else (X, leaf)), B, groups, Y, scales).sum().backward()
        assert torch.equal(leaf.grad, ones[i].to(leaf.dtype))
    y = Y.clone().requires_grad_()
    g.adapters(X, A, B, groups, y, scales).backward(G)
    assert torch.equal(y.grad, G)
    with pytest.raises(ValueError, match="scales"):
        g.adapters(X, A, B, groups, Y, scales.clone().requires_grad_())
    with pytest.raises(RuntimeError):
        b = B.clone().requires_grad_()
        out = g.adapters(X, A, b, groups, Y)
        (first,) = torch.autograd.grad(out.float().square().sum(), b, create_graph=True)
        first.sum().backward()


def test_beside_a_rounded_projection():
    """Y and its gradient through block_linear: X's is the sum of both ways."""
    X, A, B, _, scales, index, G = problem(M=40, N=128, K=256)
    W = g.block_quantize(torch.randn(128, 256, device="cuda"))
    WT = W.transposed()
    groups = g.adapter_groups(index, A.shape[0])
    x = X.clone().requires_grad_()
    O = g.adapters(x, A, B, groups, g.block_linear(x, W, WT=WT), scales)
    O.backward(G)
    H = torch.empty(40, A.shape[1], device="cuda")
    Y = g.block_linear(X, W)
    out = torch.empty_like(Y)
    ws = torch.empty(g.gptq2d_adapters_workspace_size(40, 128, 256, 8, 3), dtype=torch.uint8, device="cuda")
    g.gptq2d_adapters(X, A, B, scales, groups, Y, out, H, ws)
    assert torch.equal(out, O)
    through = g.block_linear_backward(G, X, WT)[0]
    low, dA, dB = g.adapters_backward(G, X, A, B, groups, H, scales)
    assert torch.equal(x.grad, through + low)
    # one call: the projection's gradient as D, rounded once
    both = g.adapters_backward(G, X, A, B, groups, H, scales, D=through)[0]
    alone = g.adapters_backward(G.float(), X.float(), A.float(), B.float(), groups, H, scales, wants=(True, False, False))[0]
    want = through.double() + alone.double()
    assert bool(((both.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -14 * alone.abs().max()).all())


def test_on_a_stream():
    """Everything of a step on a stream of its own, twice the same bits."""
    X, A, B, Y, scales, index, G = problem(M=300, N=264, K=136, R=16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(2):
        with torch.cuda.stream(stream):
            leaves = [t.clone().requires_grad_() for t in (X, A, B)]
            groups = g.adapter_groups(index, 3)
            O = g.adapters(*leaves, groups, Y, scales)
            O.backward(G)
        stream.synchronize()
        got.append((O.detach(), *(t.grad for t in leaves)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
