"""Plain counterparts of the operators that end a serving step (oracle of their
tests): one token, one row, one page after the other, in 64 bits, on the CPU."""
import math

import torch

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def verify(X, tokens, parents, drafts, scale, uniform, D=None, draft_lse=None, draft_scale=1.0):
    """(path, count, next, logprob) as gptq2d_tree_verify defines them."""
    seqs, width = tokens.shape
    vocab = X.shape[1]
    z = X.double().cpu().view(seqs, width, vocab) * scale
    tokens = tokens.tolist()
    parents = [list(range(-1, width - 1))] * seqs if parents is None else parents.tolist()
    drafts = [width] * seqs if drafts is None else [min(max(n, 0), width) for n in drafts.tolist()]
    u = None if uniform is None else uniform.double().tolist()
    if D is not None:
        q = torch.exp(D.double().cpu().view(seqs, width, vocab) * draft_scale
                      - draft_lse.double().cpu().view(seqs, width, 1))
    path = torch.full((seqs, width), -1, dtype=torch.int32)
    count, following = torch.zeros(seqs, dtype=torch.int32), torch.full((seqs,), -1, dtype=torch.int64)
    logprob = torch.zeros(seqs, width, dtype=torch.float64)
    for b in range(seqs):
        def row(t):
            """log p of what follows t, or None after a row that has none"""
            x = z[b, t]
            bad = bool(torch.isnan(x).any()) or bool((x == math.inf).any()) or bool((x == -math.inf).all())
            return None if bad else torch.log_softmax(x, 0)

        n = drafts[b]
        if n == 0:
            continue
        lps = {}
        for t in range(1, n):
            c = parents[b][t]
            if not 0 <= c < t:
                continue
            lps.setdefault(c, row(c))
            y = tokens[b][t]
            logprob[b, t] = math.nan if lps[c] is None else float(lps[c][y]) if 0 <= y < vocab else -math.inf
        cur, way, gone, beta = 0, [0], [], 0.0
        for t in range(1, n):
            if parents[b][t] != cur:
                continue
            y, lp = tokens[b][t], lps[cur]
            p = 0.0 if lp is None or not 0 <= y < vocab else math.exp(float(lp[y]))
            if lp is None or not 0 <= y < vocab:
                passes = False
            elif u is None:
                passes = int((z[b, cur] == z[b, cur].max()).nonzero()[0]) == y
            elif D is not None:
                M = 1.0 if not gone else float((lp.exp() - beta * q[b, cur]).clamp(min=0).sum())
                passes = u[b][t] * M * float(q[b, cur, y]) < p - beta * float(q[b, cur, y])
            else:
                passes = y not in gone and u[b][t] * (1.0 - sum(math.exp(float(lp[w])) for w in gone)) < p
            if passes:
                cur, gone, beta = t, [], 0.0
                way.append(t)
                continue
            if D is not None:
                if not 0 <= y < vocab:  # not drawn from q: no rejection
                    continue
                if lp is not None:
                    beta += 1.0 if not gone else float((lp.exp() - beta * q[b, cur]).clamp(min=0).sum())
                gone.append(y)
            elif 0 <= y < vocab and y not in gone:
                gone.append(y)
        path[b, :len(way)] = torch.tensor(way, dtype=torch.int32)
        count[b] = len(way)
        lp = row(cur)
        if lp is None:
            logprob[b, 0] = math.nan
            continue
        if u is None:
            following[b] = int((z[b, cur] == z[b, cur].max()).nonzero()[0])
        else:
            r = lp.exp()
            less = r.clone()
            if D is not None and gone:
                less = (r - beta * q[b, cur]).clamp(min=0)
            elif D is None and gone:
                less[gone] = 0.0
            r = less if float(less.sum()) > 0 else r
            sums = torch.cumsum(r, 0)
            over = (sums > u[b][0] * float(sums[-1])).nonzero()
            following[b] = int(over[0]) if len(over) else int((r > 0).nonzero()[-1])
        logprob[b, 0] = float(lp[following[b]])
    return path, count, following, logprob


def pages_update(table, length, source, want, held, pages, page):
    """(table, copies, left) as gptq2d_pages_update defines them, from lists."""
    width, rows = len(table[0]), len(want)
    source = list(range(rows)) if source is None else source
    held = [0] * pages if held is None else held
    room = width * page
    want = [min(max(w, 0), room) for w in want]
    kept = [min(max(length[r], 0), w) if 0 <= r < len(length) else 0 for r, w in zip(source, want)]
    name = lambda r, j: table[r][j] if 0 <= table[r][j] < pages else -1
    whole = {name(r, j) for r, k in zip(source, kept) for j in range(k // page)}
    ends = {}
    for i, (r, k) in enumerate(zip(source, kept)):
        if k % page:
            ends.setdefault(name(r, k // page), i)
    free = [p for p in range(pages) if not held[p] and p not in whole and p not in ends]
    out, copies, lacking = [], [], 0
    for i in range(rows):
        new, copy = [], [-1, -1, 0]
        for j in range(width):
            p = name(source[i], j) if j * page < kept[i] else -1
            mine = p < 0 or (ends.get(p) == i and p not in whole and not held[p])
            if j < kept[i] // page or (j * page < kept[i] and mine):
                new.append(p)
            elif j * page < want[i]:
                lacking += not free
                new.append(free.pop(0) if free else -1)
                if j * page < kept[i]:
                    copy = [p, new[-1], kept[i] % page]
            else:
                new.append(-1)
        out.append(new)
        copies.append(copy)
    return out, copies, len(free) - lacking
