"""gptq2d_tree_verify against the scan in 64 bits. Kept tokens, counts and next tokens
have to be equal: the inputs' random numbers come nowhere near a border (tests of
tokens are decided to about 1e-7, samples to about 1e-13). Log probabilities are
differences of 32-bit terms' sums: exp2's argument is off by 2^-24 of itself (at most
about 100, of a term that is then nothing; 2^-24 * 30 of one that counts) and its result
by 2^-23, the 16 and more terms that a thread sums by 2^-24 each and step; the result
is rounded to 32 bits."""
import math

import pytest
import torch

import serving
from paper_2607_27042_amd import binding as g

pytestmark = pytest.mark.gpu


def gen(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return r


def call(X, tokens, parents=None, drafts=None, scale=1.0, uniform=None, D=None, lse=None, draft_scale=1.0):
    seqs, width = tokens.shape
    out = (torch.full((seqs, width), -7, dtype=torch.int32, device="cuda"),
           torch.full((seqs,), -7, dtype=torch.int32, device="cuda"),
           torch.full((seqs,), -7, dtype=torch.int64, device="cuda"),
           torch.full((seqs, width), -7.0, device="cuda"))
    ws = torch.full((g.gptq2d_tree_verify_workspace_size(seqs, width, X.shape[1]),), 0xff, dtype=torch.uint8, device="cuda")
    g.gptq2d_tree_verify(X, tokens, parents, drafts, scale, uniform, D, lse, draft_scale, *out, ws)
    return out


def check(X, tokens, parents=None, drafts=None, scale=1.0, uniform=None, D=None, lse=None, draft_scale=1.0, got=None):
    if got is None:
        got = call(X, tokens, parents, drafts, scale, uniform, D, lse, draft_scale)
    ref = serving.verify(X, tokens, parents, drafts, scale, uniform, D, lse, draft_scale)
    for a, b, what in zip(got[:3], ref[:3], ("path", "count", "next")):
        assert torch.equal(a.cpu(), b), (what, a.cpu(), b)
    a, b = got[3].double().cpu(), ref[3]
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(a == -math.inf, b == -math.inf)
    fine = torch.isfinite(b)
    # sum: 2^-24 (30 + 2 + steps) of itself at worst; rounding 2^-24 |lp|
    steps = -(-X.shape[1] // 4096) * 16
    bound = 2.0 ** -24 * (32 + steps + b[fine].abs())
    assert bool(((a[fine] - b[fine]).abs() <= bound).all()), (a[fine] - b[fine]).abs().max()
    return got


def logits(r, rows, vocab, dtype, wide=2.0):
    return (wide * torch.randn(rows, vocab, generator=r, device="cuda")).to(serving.DTYPE[dtype])


def tree(r, seqs, width, branch=3):
    """Random parents: mostly recent tokens; some follow the context."""
    back = torch.randint(1, branch + 1, (seqs, width), generator=r, device="cuda")
    p = torch.arange(width, device="cuda") - back
    p = torch.where(p < 0, torch.where(torch.rand(seqs, width, generator=r, device="cuda") < 0.8, 0, -1), p)
    p[:, 0] = -1
    return p.to(torch.int32)


def likely(X, tokens, parents, r, some=4):
    """Drafted tokens out of the likeliest of their parent's row."""
    seqs, width = tokens.shape
    row = torch.arange(seqs, device="cuda").unsqueeze(1) * width + parents.clamp(min=0).long()
    k = min(some, X.shape[1])
    best = X.float().topk(k, dim=1).indices[row]
    return best.gather(2, torch.randint(k, (seqs, width, 1), generator=r, device="cuda"))[..., 0]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("seqs,width,vocab", [(1, 1, 1), (2, 2, 5), (3, 13, 127), (5, 64, 600), (4, 8, 4096), (2, 9, 4097),
                                              (3, 5, 50257), (1, 3, 300001)])
def test_certain_drafts(dtype, seqs, width, vocab):
    r = gen(seqs * 1000 + width)
    X = logits(r, seqs * width, vocab, dtype)
    parents = tree(r, seqs, width)
    tokens = likely(X, torch.zeros(seqs, width), parents, r)  # with repeated ones among siblings
    u = torch.rand(seqs, width, generator=r, device="cuda")
    check(X, tokens, parents, None, 1.25, u)
    check(X, tokens, None, torch.randint(0, width + 2, (seqs,), generator=r, device="cuda", dtype=torch.int32), 0.5, u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [3, 1000, 32001])
@pytest.mark.parametrize("chain", [True, False])
def test_drawn_drafts(dtype, vocab, chain):
    """Chains and trees whose siblings are drawn independently from one distribution."""
    r = gen(vocab)
    seqs, width = 12, 11
    X = logits(r, seqs * width, vocab, dtype)
    D = (X.float() + 0.8 * torch.randn(X.shape, generator=r, device="cuda")).to(X.dtype)
    lse = torch.logsumexp(D.double() * 0.9, 1).float()
    parents = None if chain else tree(r, seqs, width, 6)
    row = torch.arange(width, device="cuda").expand(seqs, -1) - 1 if chain else parents
    row = torch.arange(seqs, device="cuda").unsqueeze(1) * width + row.clamp(min=0).long()
    q = torch.softmax(D.double() * 0.9, 1)[row].view(-1, vocab)
    tokens = torch.multinomial(q.float().cpu(), 1, generator=torch.Generator().manual_seed(vocab)).view(seqs, width).cuda()
    u = torch.rand(seqs, width, generator=r, device="cuda")
    got = check(X, tokens, parents, None, 1.1, u, D, lse, 0.9)
    assert int(got[1].max()) > 2  # something was kept


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["certain", "drawn", "greedy"])
@pytest.mark.parametrize("seqs,width,vocab", [(3, 4, 70001), (2, 3, 128000), (2, 3, 250001), (2, 3, 300008), (600, 2, 6001)])
def test_long_rows(dtype, mode, seqs, width, vocab):
    """Parts of the last row of several steps: of fewer than a turn has, of as many, of more."""
    r = gen(vocab + width)
    X = logits(r, seqs * width, vocab, dtype)
    if mode != "drawn":
        tokens = likely(X, torch.zeros(seqs, width), tree(r, seqs, width), r)
        check(X, tokens, None, None, 1.0, torch.rand(seqs, width, generator=r, device="cuda") if mode == "certain" else None)
        return
    D = (X.float() + torch.randn(X.shape, generator=r, device="cuda")).to(X.dtype)
    lse = torch.logsumexp(D.double(), 1).float()
    q = torch.softmax(D.float(), 1).view(seqs, width, vocab)[:, :-1].reshape(-1, vocab)
    u = torch.rand(seqs, width, generator=r, device="cuda")
    tokens = torch.randint(vocab, (seqs, width), generator=r, device="cuda")
    cut = torch.rand(q.shape[0], 1, generator=r, device="cuda")
    tokens[:, 1:] = torch.searchsorted(q.cumsum(1), cut).clamp(max=vocab - 1).view(seqs, -1)
    check(X, tokens, None, None, 1.0, u, D, lse, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1, 9, 5000, 33333])
def test_greedy(dtype, vocab):
    r = gen(vocab)
    X = logits(r, 6 * 16, vocab, dtype)
    top = X.max()
    X[torch.rand(X.shape, generator=r, device="cuda") < 3.0 / vocab] = top + 1  # equal largest logits
    parents = tree(r, 6, 16)
    check(X, likely(X, torch.zeros(6, 16), parents, r, 1), parents)
    check(X, likely(X, torch.zeros(6, 16), parents, r, 3), parents, scale=3.0)


def test_views():
    """Rows with a stride, off the 16-byte boundaries, of both sides."""
    r = gen(3)
    for vocab, off in ((1000, 1), (4100, 3), (517, 0)):
        X = logits(r, 24, vocab + 11, "bf16")[:, off:off + vocab]
        D = logits(r, 24, vocab + 5, "bf16")[:, 2:2 + vocab]
        lse = torch.logsumexp(D.double(), 1).float()
        u = torch.rand(4, 6, generator=r, device="cuda")
        tokens = torch.randint(vocab, (4, 6), generator=r, device="cuda")
        check(X, tokens, None, None, 1.0, u, D, lse)
        check(X, tokens, None, None, 1.0, u)


def test_far_logits():
    """Logits of any size: only differences count."""
    r = gen(5)
    X = logits(r, 12, 700, "f32") + 1e4
    X[3:6] -= 3e4
    X[6:9] *= 1e3
    u = torch.rand(3, 4, generator=r, device="cuda")
    parents = torch.tensor([[-1, 0, 0, 1]] * 3, dtype=torch.int32, device="cuda")
    tokens = likely(X, torch.zeros(3, 4), parents, r, 2)
    check(X, tokens, parents, None, 1.0, u)


def test_odd_rows_and_tokens():
    """NaN, infinities and empty rows; tokens outside the vocabulary; unused rows with NaN."""
    r = gen(7)
    for drawn in (False, True):
        X = logits(r, 8 * 6, 300, "f32")
        X.view(8, 6, 300)[0, 1, 5] = math.nan
        X.view(8, 6, 300)[1, 0, 299] = math.inf
        X.view(8, 6, 300)[2, 0] = -math.inf
        X.view(8, 6, 300)[3, 0, 1:] = -math.inf
        X.view(8, 6, 300)[4, :, ::2] = -math.inf
        X.view(8, 6, 300)[5, 3:] = math.nan
        parents = torch.tensor([[-1, 0, 1, 2, 0, 1]] * 8, dtype=torch.int32, device="cuda")
        tokens = likely(torch.nan_to_num(X, nan=-9.0, posinf=-9.0), torch.zeros(8, 6), parents, r, 2)
        tokens[6, 1], tokens[6, 4], tokens[7, 1] = -1, 300, 2 ** 40
        drafts = torch.tensor([6, 6, 6, 6, 6, 3, 6, 6], dtype=torch.int32, device="cuda")
        u = 0.01 * torch.rand(8, 6, generator=r, device="cuda")
        D = logits(r, 8 * 6, 300, "f32") if drawn else None
        lse = torch.logsumexp(D.double(), 1).float() if drawn else None
        check(X, tokens, parents, drafts, 1.0, u, D, lse)
        if not drawn:
            check(X, tokens, parents, drafts)


def test_ends_of_the_unit_interval():
    r = gen(9)
    X = logits(r, 10, 50, "f32")
    X[:, 7:9], X[:, 49] = -math.inf, -math.inf
    tokens = torch.randint(50, (5, 2), generator=r, device="cuda")
    for u in (0.0, 1.0 - 2.0 ** -24):
        check(X, tokens, None, None, 1.0, torch.full((5, 2), u, device="cuda"))
    # all that p has was rejected (a test's last place): p itself
    X = torch.full((2, 30), -math.inf, device="cuda")
    X[:, 11] = 3.0
    tokens = torch.tensor([[0, 11]], device="cuda")
    got = call(X, tokens, None, None, 1.0, torch.tensor([[0.5, 1.0]], device="cuda"))
    assert got[1].tolist() == [1] and got[2].tolist() == [11]


def test_distribution():
    """The first token kept or drawn is distributed as p: counts of 60000 sequences
    within five standard deviations."""
    r = gen(11)
    seqs, width, vocab = 60000, 3, 5
    X = logits(r, width, vocab, "f32", 1.0).repeat(seqs, 1)
    D = logits(r, width, vocab, "f32", 1.0).repeat(seqs, 1)
    lse = torch.logsumexp(D.double(), 1).float()
    p = torch.softmax(X[0].double(), 0).cpu()
    parents = torch.tensor([[-1, 0, 0]], dtype=torch.int32, device="cuda").repeat(seqs, 1)
    for drawn in (True, False):
        u = torch.rand(seqs, width, generator=r, device="cuda")
        if drawn:
            t = torch.multinomial(torch.softmax(D[0], 0), 2 * seqs, replacement=True, generator=r).view(seqs, 2)
        else:
            t = torch.tensor([[1, 3]], device="cuda").repeat(seqs, 1)
        tokens = torch.cat([torch.zeros(seqs, 1, dtype=torch.long, device="cuda"), t], 1)
        path, count, following, _ = call(X, tokens, parents, None, 1.0, u, D if drawn else None, lse if drawn else None)
        first = torch.where(count > 1, tokens.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], following)
        n = torch.bincount(first, minlength=vocab).cpu().double()
        assert bool(((n - seqs * p).abs() <= 5 * torch.sqrt(seqs * p * (1 - p))).all()), (n, seqs * p)


def test_graph_and_streams():
    """Captured with its workspace, replayed on other inputs, beside a call on another stream."""
    r = gen(13)
    seqs, width, vocab = 4, 6, 9000
    make = lambda: (logits(r, seqs * width, vocab, "bf16"), torch.randint(vocab, (seqs, width), generator=r, device="cuda"),
                    torch.rand(seqs, width, generator=r, device="cuda"))
    X, tokens, u = make()
    out = (torch.empty(seqs, width, dtype=torch.int32, device="cuda"), torch.empty(seqs, dtype=torch.int32, device="cuda"),
           torch.empty(seqs, dtype=torch.int64, device="cuda"), torch.empty(seqs, width, device="cuda"))
    ws = torch.empty(g.gptq2d_tree_verify_workspace_size(seqs, width, vocab), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.gptq2d_tree_verify(X, tokens, None, None, 1.0, u, None, None, 1.0, *out, ws)
    other = torch.cuda.Stream()
    for _ in range(3):
        for a, b in zip((X, tokens, u), make()):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(other):
            beside = call(X, tokens, None, None, 1.0, u)
        torch.cuda.synchronize()
        check(X, tokens, None, None, 1.0, u, got=out)
        check(X, tokens, None, None, 1.0, u, got=beside)
        again = call(X, tokens, None, None, 1.0, u)
        assert all(torch.equal(a, b) for a, b in zip(again, out))
