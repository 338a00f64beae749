"""gptq2d_tree_verify at scales and logits of any size, against the scan in 64 bits, whose
products of a 32-bit logit and a 32-bit scale are exact and whose differences are rounded
once. What is kept and next has to be equal, log probabilities are bounded as in
test_gpu_verify.py."""
import math

import pytest
import torch

import serving
from test_gpu_verify import call, check, gen, likely, logits, tree

pytestmark = pytest.mark.gpu


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


@pytest.mark.parametrize("mode", ["certain", "drawn", "greedy"])
@pytest.mark.parametrize("scale", [1e7, 1e10, 1e12, 1e14, 1e18, 1e30, 2e38])
def test_large_scales(scale, mode):
    """Cold samplers: of logits in [1, 30] the largest ones alone are left, of those near zero some more."""
    r = gen(int(math.log2(scale)))
    seqs, width, scale = 6, 5, f32(scale)
    for vocab in (40, 5000):
        X = 1.0 + 29.0 * torch.rand(seqs * width, vocab, generator=r, device="cuda")
        X[:, ::3] = X.max(1, keepdim=True).values  # many of the same
        near = torch.rand(seqs * width, vocab, generator=r, device="cuda") * (4.0 / scale)
        X = torch.where((torch.arange(seqs * width, device="cuda") % 2 == 0).unsqueeze(1), X, near)
        parents = tree(r, seqs, width)
        tokens = likely(X, torch.zeros(seqs, width), parents, r)
        u = torch.rand(seqs, width, generator=r, device="cuda") if mode != "greedy" else None
        D = logits(r, seqs * width, vocab, "f32") if mode == "drawn" else None
        lse = torch.logsumexp(D.double(), 1).float() if mode == "drawn" else None
        got = check(X, tokens, parents, None, scale, u, D, lse)
        assert int(got[2].min()) >= 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.5, 0.75, 1.0])
@pytest.mark.parametrize("mode", ["certain", "drawn", "greedy"])
def test_lowest_values(dtype, scale, mode):
    """Masks of the type's lowest value: in part of a row, in all of it (then every token is as likely)."""
    r = gen(17)
    seqs, width = 6, 4
    for vocab in (33, 4100):
        X = logits(r, seqs * width, vocab, dtype)
        low = torch.finfo(X.dtype).min
        X.view(seqs, width, vocab)[1, 0] = low
        X.view(seqs, width, vocab)[2] = low
        X.view(seqs, width, vocab)[3, :, ::2] = low
        X.view(seqs, width, vocab)[4, 0, :30] = -math.inf
        X.view(seqs, width, vocab)[4, 0, 30:] = low
        tokens = torch.randint(vocab, (seqs, width), generator=r, device="cuda")
        u = torch.rand(seqs, width, generator=r, device="cuda") if mode != "greedy" else None
        D = logits(r, seqs * width, vocab, dtype) if mode == "drawn" else None
        lse = torch.logsumexp(D.double(), 1).float() if mode == "drawn" else None
        got = check(X, tokens, None, None, scale, u, D, lse)
        assert int(got[2].min()) >= 0


def test_far_drafts():
    """A draft's logits far from zero, and rows of it that are infinite or empty where nothing is drawn from them."""
    r = gen(19)
    seqs, width, vocab = 8, 5, 900
    X = logits(r, seqs * width, vocab, "f32")
    D = X + 0.5 * torch.randn(X.shape, generator=r, device="cuda") + 2.0 ** 14
    D[width:2 * width] -= 2.0 ** 15
    lse = torch.logsumexp(D.double(), 1).float()
    D[2 * width:3 * width, 7:] = -math.inf
    lse[2 * width:3 * width] = torch.logsumexp(D[2 * width:3 * width].double(), 1).float()
    tokens = torch.randint(7, (seqs, width), generator=r, device="cuda")
    parents = tree(r, seqs, width, 4)
    check(X, tokens, parents, None, 1.0, torch.rand(seqs, width, generator=r, device="cuda"), D, lse)


@pytest.mark.parametrize("mode", ["certain", "greedy"])
@pytest.mark.parametrize("scale", [2.5e38, 3.0e38, torch.finfo(torch.float32).max])
def test_largest_scales(scale, mode):
    """As cold as 32 bits go: the scale times log2(e) has no 32-bit number."""
    r = gen(23)
    seqs, width, vocab, scale = 6, 5, 300, f32(scale)
    X = logits(r, seqs * width, vocab, "f32")
    X[:, ::3] = X.max(1, keepdim=True).values
    parents = tree(r, seqs, width)
    tokens = likely(X, torch.zeros(seqs, width), parents, r)
    tokens[:, 1:3] = 3  # one of the largest
    u = torch.rand(seqs, width, generator=r, device="cuda") if mode == "certain" else None
    # (every logit below the largest is further from it than 32 bits tell: log p = -inf in 32 bits, if not in 64)
    got = call(X, tokens, parents, None, scale, u)
    ref = serving.verify(X, tokens, parents, None, scale, u)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(got[:3], ref[:3]))
    a, b = got[3].cpu(), ref[3].float()
    assert torch.equal(torch.isinf(a), torch.isinf(b)) and not bool(torch.isnan(a).any())
    fine = torch.isfinite(b)
    assert bool(((a[fine] - b[fine]).abs() <= 2.0 ** -24 * (48 + b[fine].abs())).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [8, 5000])
def test_drafts_like_the_target(vocab, dtype):
    """Drafts whose q is p to its last place or nearly: what is left of p after a rejection is
    nothing, or what sums round to. The next token is one that has something of p."""
    r = gen(29)
    seqs, V = 65535 if vocab == 8 else 6000, vocab
    for n in (1, 2, 3, 5, 6):
        # n tokens of one size and a last one of next to nothing (the other way round for the draft)
        X = torch.full((seqs, 2, V), -math.inf, device="cuda")
        X[..., :n], X[..., n] = 0.0, -(17.0 + 2.0 * torch.rand(seqs, 1, generator=r, device="cuda"))
        X = X.to(serving.DTYPE[dtype])
        size = n + torch.exp(X[:, 0, n].double())  # of the row
        lse = torch.log(size).float()
        off = torch.randint(-40, 41, (seqs,), generator=r, device="cuda").double() * 2.0 ** -52
        D = torch.full((seqs, 2, V), -math.inf, device="cuda")
        D[..., :n] = (lse.double() - torch.log(size) + off).float().view(seqs, 1, 1)
        D[..., n] = 5.0
        D = D.to(X.dtype)
        tokens = torch.full((seqs, 2), n, device="cuda")
        u = 0.4 + 0.5 * torch.rand(seqs, 2, generator=r, device="cuda")
        _, count, after, logprob = call(X.view(-1, V), tokens, None, None, 1.0, u, D.view(-1, V),
                                        lse.unsqueeze(1).expand(-1, 2).flatten())
        assert bool((count == 1).all())
        assert bool(((after >= 0) & (after <= n)).all()) and bool(torch.isfinite(logprob).all())
