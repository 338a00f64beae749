"""gptq2d_cache_commit, _cache_copy and _pages_update: whole numbers and moved bytes,
which have to be equal."""
import random

import pytest
import torch

import serving
from paper_2607_27042_amd import binding as g

pytestmark = pytest.mark.gpu


def caches(layers, pages, heads, page, dim, code=torch.int8, seed=0):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    out = []
    for _ in range(layers):
        c = [torch.randint(0, 256, (pages, heads, page, dim), generator=r, device="cuda", dtype=torch.uint8).view(code)
             for _ in range(2)]
        s = [torch.rand((pages, heads, page), generator=r, device="cuda") for _ in range(2)]
        out.append((*c, *s))
    return out


def raw(cache):
    return [t.clone() if t.dtype == torch.float32 else t.view(torch.uint8).clone() for t in cache]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(raw(a), b))


@pytest.mark.parametrize("layers,seqs,width,heads,dim,page", [(1, 1, 1, 1, 16, 16), (2, 3, 8, 2, 64, 16), (3, 5, 64, 3, 48, 32),
                                                              (1, 7, 13, 5, 128, 64), (2, 2, 64, 1, 256, 16),
                                                              (100, 2, 5, 1, 16, 16), (2, 3, 33, 2, 144, 48)])
def test_commit(layers, seqs, width, heads, dim, page):
    rng = random.Random(width + dim)
    context = [rng.randint(0, 3 * page) for _ in range(seqs)]
    context[0] = page - 1
    per = 4 + -(-width // page)
    pages = seqs * per + 2
    names = rng.sample(range(pages), seqs * per)
    table = [names[i * per:(i + 1) * per] for i in range(seqs)]
    if seqs > 2:
        table[2][context[2] // page] = -1  # positions without a page, or one that is none
        table[1][(context[1] + width - 1) // page] = pages
    path = [sorted(rng.sample(range(1, width), rng.randint(0, width - 1))) for _ in range(seqs)]
    path = [([0] + p + [-1] * width)[:width] for p in path]
    if seqs > 3:
        path[3] = list(range(width))  # nothing moves
        rng.shuffle(path[4])          # entries below their place are skipped
        path[4][0] = width            # and those past the tree
    c = caches(layers, pages, heads, page, dim, torch.float8_e4m3fn, seed=dim)
    want = [raw(x) for x in c]
    for old, new in zip([raw(x) for x in c], want):
        for b in range(seqs):
            for i, p in enumerate(path[b]):
                if not i < p < width:
                    continue
                at = [(table[b][q // page], q % page) for q in (context[b] + p, context[b] + i)]
                if all(0 <= pg < pages for pg, _ in at):
                    for x, y in zip(old, new):
                        y[at[1][0], :, at[1][1]] = x[at[0][0], :, at[0][1]]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    g.gptq2d_cache_commit(c, ints(table), ints(context), ints(path))
    for x, y in zip(c, want):
        assert same(x, y)


def test_commit_past_the_table():
    c = caches(1, 6, 2, 16, 32)
    before = raw(c[0])
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32, device="cuda")
    context = torch.tensor([31, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 2, 3, -1], [0, 3, -1, -1], [0, 2, 3, -1]], dtype=torch.int32, device="cuda")
    g.gptq2d_cache_commit(c, table, context, path)
    for t, b in zip(raw(c[0]), before):
        b[2, :, 0] = b[2, :, 2]  # only -1 + 3 to -1 + 1
        assert torch.equal(t, b)


def test_commit_strided_table():
    """Rows of a wider table; a wide one whose offsets pass 32 bits is not needed: page
    numbers are 32-bit, places are taken in 64."""
    c = caches(2, 8, 1, 16, 16)
    want = [raw(x) for x in c]
    wide = torch.full((2, 9), -5, dtype=torch.int32, device="cuda")
    wide[:, 2:5] = torch.tensor([[7, 0, 3], [2, 6, 1]], device="cuda")
    context = torch.tensor([14, 3], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 4, 7, -1, -1, -1, -1, -1], [0, 1, 5, 6, -1, -1, -1, -1]], dtype=torch.int32, device="cuda")
    g.gptq2d_cache_commit(c, wide[:, 2:5], context, path)
    for new in want:
        for y in new:
            y[7, :, 15], y[0, :, 0] = y[0, :, 2].clone(), y[0, :, 5].clone()
            y[2, :, 5], y[2, :, 6] = y[2, :, 8].clone(), y[2, :, 9].clone()
    for x, y in zip(c, want):
        assert same(x, y)


def test_commit_far_offsets():
    """A cache past 2^32 bytes."""
    pages, heads, page, dim = 2 ** 32 // (16 * 256 * 16) + 9, 16, 16, 256
    kc = torch.zeros(pages, heads, page, dim, dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    ks, vs = (torch.zeros(pages, heads, page, device="cuda") for _ in range(2))
    last = pages - 1
    for t, base in ((kc, 1), (vc, 2), (ks, 3), (vs, 4)):
        t[last, :, 9] = base
        t[last, :, 3] = 50 + base
    g.gptq2d_cache_commit([(kc, vc, ks, vs)], torch.tensor([[last]], dtype=torch.int32, device="cuda"),
                          torch.tensor([2], dtype=torch.int32, device="cuda"),
                          torch.tensor([[0, 7] + [-1] * 6], dtype=torch.int32, device="cuda"))
    g.gptq2d_cache_copy([(kc, vc, ks, vs)], torch.tensor([[last, 0, 10]], dtype=torch.int32, device="cuda"))
    for t, base in ((kc, 1), (vc, 2), (ks, 3), (vs, 4)):
        assert bool((t[last, :, 3] == base).all()) and bool((t[0, :, 9] == base).all()) and bool((t[0, :, 3] == base).all())
        assert int(torch.count_nonzero(t[1:last])) == 0 and int(torch.count_nonzero(t[0, :, 10:])) == 0


@pytest.mark.parametrize("layers,heads,dim,page", [(1, 1, 16, 16), (3, 5, 48, 48), (100, 2, 64, 16), (2, 9, 256, 128),
                                                   (1, 2, 32, 4096)])
def test_copy(layers, heads, dim, page):
    pages = 12
    copies = [[0, 5, page], [0, 6, 1], [3, 7, page - 1], [-1, -1, 0], [2, -1, 4], [12, 8, 3], [1, 12, 3], [4, 4, 5], [11, 9, 0],
              [11, 10, page + 7], [3, 1, -4]]
    c = caches(layers, pages, heads, page, dim)
    want = [raw(x) for x in c]
    for new in want:
        for s, d, n in copies:
            if 0 <= s < pages and 0 <= d < pages and n > 0:
                for y in new:
                    y[d, :, :n] = y[s, :, :n]
    g.gptq2d_cache_copy(c, torch.tensor(copies, dtype=torch.int32, device="cuda"))
    for x, y in zip(c, want):
        assert same(x, y)


def update(table, length, source, want, held, pages, page, stride=0):
    """The call on lists, with tables of wider rows."""
    ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")
    rows, width = len(want), len(table[0])
    t = torch.full((len(table), width + stride), 77, dtype=torch.int32, device="cuda")
    t[:, :width] = ints(table)
    out = torch.full((rows, width + 2 * stride), -9, dtype=torch.int32, device="cuda")
    copies = torch.full((rows, 3), -9, dtype=torch.int32, device="cuda")
    left = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((g.gptq2d_pages_update_workspace_size(rows, pages),), 0xa5, dtype=torch.uint8, device="cuda")
    g.gptq2d_pages_update(t[:, :width], ints(length), ints(source), ints(want), ints(held), pages, page, out[:, :width], copies,
                          left, ws)
    assert bool((out[:, width:] == -9).all())
    return out[:, :width].tolist(), copies.tolist(), int(left)


def check_update(*a, **k):
    got, ref = update(*a, **k), serving.pages_update(*a)
    assert got == ref


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("big", [False, True])
def test_update(seed, big):
    """Random tables that share pages; `big`: more than one work group's."""
    rng = random.Random(seed)
    page = rng.choice([16, 32, 48, 4096])
    old, rows, width = rng.randint(1, 40), rng.randint(1, 60), rng.randint(1, 30)
    if big:
        width += 1200 if seed % 2 else 0
    pages = rng.randint(1, 2 * rows * width) + (40000 if big else 0)
    table = [[rng.randrange(-1, pages + 1) if rng.random() < 0.1 else rng.randrange(pages) for _ in range(width)]
             for _ in range(old)]
    for i in range(1, old):  # common beginnings
        n = rng.randint(0, width)
        table[i][:n] = table[rng.randrange(i)][:n]
    length = [rng.randint(0, width * page + 5) for _ in range(old)]
    source = [rng.randint(-1, old) for _ in range(rows)]
    want = [rng.choice([0, -3, rng.randint(0, width * page), (length[s] if 0 <= s < old else 7) + rng.randint(0, page),
                        width * page + 100]) for s in source]
    held = [int(rng.random() < 0.1) * rng.choice([1, -1, 2 ** 30]) for _ in range(pages)] if seed % 3 else None
    check_update(table, length, source, want, held, pages, page, stride=seed % 4)
    if rows <= old:
        check_update(table, length, None, want, held, pages, page)


def test_update_beams():
    """Four beams of a prompt: the first to go on from a beam keeps its last page, the others copy it."""
    table = [[3, 1, -1, -1], [3, 2, -1, -1], [3, 4, -1, -1], [3, 5, -1, -1]]
    out, copies, left = update(table, [20] * 4, [1, 1, 3, 1], [21] * 4, None, 8, 16)
    assert out == [[3, 2, -1, -1], [3, 0, -1, -1], [3, 5, -1, -1], [3, 1, -1, -1]]
    assert copies == [[-1, -1, 0], [2, 0, 4], [-1, -1, 0], [2, 1, 4]] and left == 3
    # a page that another row keeps whole is copied by all that end in it
    out, copies, _ = update([[3, 1]], [32], [0, 0, 0], [24, 32, 32], None, 8, 16)
    assert out == [[3, 0], [3, 1], [3, 1]] and copies == [[1, 0, 8], [-1, -1, 0], [-1, -1, 0]]


def test_update_in_a_graph():
    """Captured with the copies, replayed after eager work."""
    c = caches(2, 16, 1, 16, 16)
    table = torch.tensor([[3, 1], [3, 2]], dtype=torch.int32, device="cuda")
    length, want, source = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([20, 20], [21, 21], [1, 1]))
    out, copies = torch.empty_like(table), torch.empty(2, 3, dtype=torch.int32, device="cuda")
    ws = torch.empty(g.gptq2d_pages_update_workspace_size(2, 16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.gptq2d_pages_update(table, length, source, want, None, 16, 16, out, copies, None, ws)
        g.gptq2d_cache_copy(c, copies)
    for last in (2, 7, 11):
        table[1, 1] = last
        before = [raw(x) for x in c]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert out.tolist() == [[3, last], [3, 0]] and copies.tolist() == [[-1, -1, 0], [last, 0, 4]]
        for x, y in zip(c, before):
            for z in y:
                z[0, :, :4] = z[last, :, :4]
            assert same(x, y)
