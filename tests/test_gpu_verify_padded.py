"""Drafts that are padded with what is no token: gptq2d_tree_verify goes on as if it were not there."""
import pytest
import torch

from test_gpu_verify import call, check, gen, logits

pytestmark = pytest.mark.gpu

OUTSIDE = [-1, 5, 2 ** 31, -2 ** 40]


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("pattern", ["-", "d-", "-d", "d-d", "--"])
def test_distribution(drawn, pattern):
    """The first token kept or drawn is distributed as p, whichever of token 0's followers are
    padding: counts of 60000 sequences within five standard deviations."""
    r = gen(len(pattern) + drawn)
    seqs, width, vocab = 60000, 1 + len(pattern), 5
    X, D = (logits(r, width, vocab, "f32", 1.0).repeat(seqs, 1) for _ in range(2))
    lse = torch.logsumexp(D.double(), 1).float()
    p = torch.softmax(X[0].double(), 0).cpu()
    parents = torch.tensor([[-1] + [0] * (width - 1)], dtype=torch.int32, device="cuda").repeat(seqs, 1)
    u = torch.rand(seqs, width, generator=r, device="cuda")
    t = torch.multinomial(torch.softmax(D[0], 0), seqs * width, replacement=True, generator=r).view(seqs, width)
    if not drawn:
        t[:] = torch.arange(width, device="cuda")
    for i, kind in enumerate(pattern):
        if kind == "-":
            t[:, 1 + i] = torch.tensor(OUTSIDE, device="cuda")[torch.arange(seqs, device="cuda") % 4]
    path, count, following, _ = call(X, t, parents, None, 1.0, u, D if drawn else None, lse if drawn else None)
    first = torch.where(count > 1, t.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], following)
    n = torch.bincount(first, minlength=vocab).cpu().double()
    assert bool(((n - seqs * p).abs() <= 5 * torch.sqrt(seqs * p * (1 - p))).all()), (n, seqs * p)


@pytest.mark.parametrize("mode", ["drawn", "certain", "greedy"])
def test_as_if_not_there(mode):
    """The same trees with and without padding among the siblings: same tokens kept, same next token."""
    r = gen(3)
    seqs, vocab = 50, 700
    X = logits(r, seqs * 4, vocab, "bf16")
    D = (X.float() + torch.randn(X.shape, generator=r, device="cuda")).to(X.dtype) if mode == "drawn" else None
    lse = torch.logsumexp(D.double(), 1).float() if D is not None else None
    tokens = X.view(seqs, 4, vocab)[:, 0].float().topk(4).indices.flip(1).contiguous()
    u = torch.rand(seqs, 4, generator=r, device="cuda") if mode != "greedy" else None
    parents = torch.tensor([[-1, 0, 0, 0]] * seqs, dtype=torch.int32, device="cuda")
    short = check(X, tokens, parents, None, 1.0, u, D, lse)
    at = torch.tensor([0, 2, 4, 5], device="cuda")  # 1 and 3 are padding

    def wide(t, fill, rows=False):
        if t is None:
            return None
        t = t.view(seqs, 4, -1)
        out = torch.full((seqs, 6, t.shape[2]), fill, dtype=t.dtype, device="cuda")
        out[:, at] = t
        return out.view(seqs * 6, -1) if rows else out.view(seqs, 6)

    more = wide(lse, 0.0)
    longer = check(wide(X, float("nan"), True), wide(tokens, vocab), torch.tensor([[-1, 0, 0, 0, 0, 0]] * seqs, dtype=torch.int32,
                   device="cuda"), None, 1.0, wide(u, 0.0), wide(D, float("nan"), True), None if more is None else more.flatten())
    assert torch.equal(short[1], longer[1]) and torch.equal(short[2], longer[2]) and int(short[1].max()) == 2
    kept = short[1] > 1
    assert torch.equal(at[short[0][kept, 1].long()], longer[0][kept, 1].long())
