"""gptq2d_cache_commit, _cache_copy and _pages_update at the sizes of loaded servers, where they
take other routes: several layers a wave, tables of many entries, rows and pages."""
import random

import pytest
import torch

from paper_2607_27042_amd import binding as g
from test_gpu_pages import caches, check_update, raw, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers,seqs,heads,dim,page", [(7, 64, 20, 48, 16), (5, 300, 6, 64, 32), (9, 80, 13, 112, 16),
                                                        (6, 90, 16, 128, 48), (7, 70, 18, 144, 16), (5, 128, 13, 256, 16),
                                                        (99, 40, 9, 16, 16), (2, 260, 16, 32, 16)])
def test_commit_of_many(layers, seqs, heads, dim, page):
    """More heads, sequences and layers than waves run at once, layers that four do not divide."""
    assert -(-seqs * heads // 4) * min(layers, 96) > 2048
    rng = random.Random(layers * seqs)
    width, per = 24, 3
    pages = seqs * per + 1
    names = rng.sample(range(pages), seqs * per)
    table = [names[i * per:(i + 1) * per] for i in range(seqs)]
    context = [rng.randint(0, per * page - width) for _ in range(seqs)]
    path = [([0] + sorted(rng.sample(range(1, width), rng.randint(0, width - 1))) + [-1] * width)[:width] for _ in range(seqs)]
    table[3][(context[3] + 9) // page] = -1
    moves = []
    for b in range(seqs):
        for i, p in enumerate(path[b]):
            at = [(table[b][q // page], q % page) for q in (context[b] + p, context[b] + i)]
            if i < p and all(a[0] >= 0 for a in at):
                moves.append((*at[0], *at[1]))
    fp, ft, tp, tt = (torch.tensor(m, device="cuda") for m in zip(*moves))
    c = caches(layers, pages, heads, page, dim, seed=dim)
    want = [raw(x) for x in c]
    for new in want:
        for y in new:
            y[tp, :, tt] = y[fp, :, ft]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    g.gptq2d_cache_commit(c, ints(table), ints(context), ints(path))
    for x, y in zip(c, want):
        assert same(x, y)


@pytest.mark.parametrize("heads,dim,page", [(20, 128, 512), (3, 256, 4096), (40, 48, 1024)])
def test_copy_of_large_pages(heads, dim, page):
    """Pages of more pieces than the work groups of one copy take in a turn."""
    assert heads * dim * page // 16 > 65536
    c = caches(2, 6, heads, page, dim)
    want = [raw(x) for x in c]
    copies = [[0, 3, page], [1, 4, page - 1], [1, 5, page // 2 + 3]]
    for new in want:
        for s, d, n in copies:
            for y in new:
                y[d, :, :n] = y[s, :, :n]
    g.gptq2d_cache_copy(c, torch.tensor(copies, dtype=torch.int32, device="cuda"))
    for x, y in zip(c, want):
        assert same(x, y)


def prompts(rng, old, width, pages, page, shared):
    """Tables of groups of sequences that share the pages of a prompt and end in pages of their own."""
    names = rng.sample(range(pages), pages)
    table, length, at, prompt, kept = [], [], 0, [], 0
    for i in range(old):
        if i % shared == 0:
            kept = rng.randint(width // 2, width - 2)
            prompt, at = names[at % (pages - width):][:kept], at + kept
        n = rng.randint(1, width - kept)
        own = names[at % (pages - width):][:n]
        at += n
        table.append(prompt + own + [-1] * (width - kept - n))
        length.append((kept + n) * page - rng.randint(0, page - 1))
    return table, length


@pytest.mark.parametrize("rows,width,pages,page", [(130, 300, 9000, 16), (200, 700, 28672, 16), (400, 600, 20000, 64),
                                                   (300, 257, 15000, 48), (1024, 256, 28672, 32), (1023, 65, 5000, 16),
                                                   (129, 64, 28671, 16), (60, 1100, 28000, 16)])
def test_update_of_many(rows, width, pages, page):
    """One launch: long beginnings that are kept whole, more rows than the waves take at once."""
    assert rows <= 1024 and pages <= 28672 and rows * width <= 1 << 18
    rng = random.Random(rows + width)
    table, length = prompts(rng, rows, width, pages, page, 8)
    source = [rng.choice([rng.randrange(rows), i, i // 8 * 8, -1 if rng.random() < 0.1 else i]) for i in range(rows)]
    want = [rng.choice([(length[s] if s >= 0 else 5) + rng.randint(0, 2 * page), 0 if rng.random() < 0.2 else length[s]])
            for s in source]
    held = [int(rng.random() < 0.05) for _ in range(pages)]
    check_update(table, length, source, want, held, pages, page, stride=rows % 3)


@pytest.mark.parametrize("rows,width,pages", [(1025, 40, 20000), (2500, 30, 60000), (3000, 100, 28672), (5000, 9, 28673),
                                              (40, 20, 28673), (1500, 180, 12000)])
def test_update_of_more(rows, width, pages):
    """More rows, pages or entries than one work group marks: several launches, the sums over rows in turns."""
    page = 16
    assert rows > 1024 or pages > 28672 or rows * width > 1 << 18
    rng = random.Random(rows + width)
    old = min(rows, 1200)
    table, length = prompts(rng, old, width, pages, page, 6)
    source = [rng.randrange(-1 if rng.random() < 0.1 else 0, old) for _ in range(rows)]
    want = [(length[s] if s >= 0 else 40) + rng.randint(-2 * page, page) for s in source]
    check_update(table, length, source, want, [int(rng.random() < 0.05) for _ in range(pages)], pages, page)
