"""The operators that end a serving step with drafted tokens, and low-rank adapters, as cases to be timed.

A case is a dict of plain values. Its "op" names the operator:

  verify      which drafted tokens are kept, from the target's logits and given
              random numbers, and the token after them; "draft": the drafts were
              drawn from logits of their own (a chain), otherwise they are certain
              (a tree); "greedy": without random numbers
  commit      the kept tokens' keys and values moved up in the caches of all layers
  fork        the page tables of beams that go on, end and begin, and the copies
              of pages that they share but will write
  adapters    Y + s_a (X A_a^T) B_a^T with the adapter a of every row
  gradients   of the adapters, of X and (through it) of what it was made of

`own` selects the library's kernels; otherwise the same is computed with
elementary torch operations.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ES = {"f32": 4, "f16": 2, "bf16": 2}
_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _verify(seqs, width, branch, vocab, draft, greedy, dtype):
    return {"op": "verify", "seqs": seqs, "width": width, "branch": branch, "vocab": vocab, "draft": draft,
            "greedy": greedy, "dtype": dtype}


def _commit(layers, seqs, width, branch, heads, dim, page, context, code):
    return {"op": "commit", "layers": layers, "seqs": seqs, "width": width, "branch": branch, "heads": heads, "dim": dim,
            "page": page, "context": context, "code": code}


def _fork(layers, groups, beams, heads, dim, page, prompt, grown, code):
    return {"op": "fork", "layers": layers, "groups": groups, "beams": beams, "heads": heads, "dim": dim, "page": page,
            "prompt": prompt, "grown": grown, "code": code}


def _adapters(op, tokens, n, k, rank, count, dtype):
    return {"op": op, "tokens": tokens, "n": n, "k": k, "rank": rank, "count": count, "dtype": dtype}


def listed():
    cases = {
        # one sequence and a chain drawn from a small model: the latency of a step
        "verify 1x8 chain 32000 f32": _verify(1, 8, 1, 32000, True, False, "f32"),
        # a batch with trees of the likeliest tokens, odd vocabulary
        "verify 16x13 tree 50257 f16": _verify(16, 13, 3, 50257, False, False, "f16"),
        # a loaded server with drawn chains and a large vocabulary
        "verify 64x8 chain 128000 bf16": _verify(64, 8, 1, 128000, True, False, "bf16"),
        # the kept tokens of one sequence's tree, all layers of a model
        "commit 32 layers 1x8": _commit(32, 1, 8, 2, 8, 128, 64, 1000, "e4m3"),
        # those of a batch of wide trees, short pages
        "commit 32 layers 64x64": _commit(32, 64, 64, 2, 8, 64, 16, 2000, "int8"),
        # four beams of one prompt
        "fork 32 layers 1x4": _fork(32, 1, 4, 8, 128, 64, 1000, 20, "e4m3"),
        # four beams of each of 64 prompts, many short pages
        "fork 16 layers 64x4": _fork(16, 64, 4, 2, 64, 16, 2000, 40, "int8"),
        # one token through a projection with its adapter
        "adapters 1x4096x4096 r16 bf16": _adapters("adapters", 1, 4096, 4096, 16, 8, "bf16"),
        # one token of each of 64 requests, with 48 adapters
        "adapters 64x4096x4096 r16 of 48 bf16": _adapters("adapters", 64, 4096, 4096, 16, 48, "bf16"),
        # prompts of requests with 16 adapters through an MLP's first matrix
        "adapters 4096x11008x4096 r64 of 16 bf16": _adapters("adapters", 4096, 11008, 4096, 64, 16, "bf16"),
        # a ragged batch of a small odd layer
        "gradients 333x1000x700 r8 of 3 f32": _adapters("gradients", 333, 1000, 700, 8, 3, "f32"),
        # a step of tuning, four adapters side by side
        "gradients 8192x4096x4096 r16 of 4 bf16": _adapters("gradients", 8192, 4096, 4096, 16, 4, "bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def draw(rng):
    def size(lo, hi, step=1):
        d = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, d // step * step)

    def layer():  # half as layers have them, half as they come
        return size(128, 11008, 128) if rng.random() < 0.5 else size(64, 11008)

    op = rng.choice(["verify", "verify", "commit", "fork", "adapters", "adapters", "gradients", "gradients"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    heads, dim, page = rng.randint(1, 16), 16 * rng.randint(1, 16), rng.choice([16, 32, 48, 64, 128])
    code = rng.choice(["e4m3", "int8"])
    while True:
        if op == "verify":
            draft = rng.random() < 0.5
            c = _verify(size(1, 64), size(1, 64), 1 if draft else rng.choice([1, 2, 3, 4]), size(128, 262144), draft,
                        rng.random() < (0.0 if draft else 0.4), dtype)
            fits = c["seqs"] * c["width"] * c["vocab"] <= 65_000_000
        elif op == "commit":
            c = _commit(size(1, 48), size(1, 64), size(2, 64), rng.choice([2, 3, 4]), heads, dim, page,
                        size(16, 4096), code)
            fits = c["layers"] * heads * dim * page * (c["context"] / page + c["seqs"] * (2 + c["width"] / page)) <= 400_000_000
        elif op == "fork":
            c = _fork(size(1, 48), size(1, 64), rng.randint(1, 8), heads, dim, page, size(16, 4096), size(1, 100), code)
            tokens = c["groups"] * (c["prompt"] + c["beams"] * (c["grown"] + 3 * page))
            fits = 1.5 * c["layers"] * heads * dim * tokens <= 400_000_000
        else:
            c = _adapters(op, size(1, 8192), layer(), layer(), rng.choice([1, 4, 8, 16, 16, 20, 32, 64, 128]),
                          size(1, 64), dtype)
            fits = (c["tokens"] * (c["n"] + c["k"]) * (1 if op == "adapters" else 0.9) <= 60_000_000
                    and c["count"] * c["rank"] <= 1024 and c["count"] * c["rank"] * (c["n"] + c["k"]) <= 15_000_000)
        if fits:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 41)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols, dtype):
    """Gaussian with a few loud channels, as activations have them."""
    x = _normal(g, rows, cols)
    x *= torch.where(_uniform(g, cols) < 0.01, 20.0, 1.0)
    return x.to(dtype)


def _tree(width, branch):
    """Parents of a tree in which every token has `branch` followers, as long as there are tokens."""
    t = torch.arange(width, device="cuda")
    return torch.where(t == 0, -1, (t - 1) // branch).to(torch.int32)


def _verify_inputs(case, g):
    b, t, v, dt = case["seqs"], case["width"], case["vocab"], _DT[case["dtype"]]
    s = {"scale": 1.25, "draft_scale": 1.0, "D": None, "draft_lse": None, "uniform": None}
    s["X"] = torch.empty(b * t, v, dtype=dt, device="cuda")
    s["parents"] = _tree(t, case["branch"]).expand(b, t).contiguous()
    s["tokens"] = torch.randint(v, (b, t), generator=g, device="cuda")
    if case["draft"]:
        s["D"] = torch.empty(b * t, v, dtype=dt, device="cuda")
        s["draft_lse"] = torch.empty(b * t, device="cuda")
    for i in range(b):  # a language model's logits: wide, with a long right tail
        x = _normal(g, t, v)
        x = 2.0 * x + 0.4 * x * x * x.sign()
        s["X"][i * t:(i + 1) * t] = x.to(dt)
        if case["draft"]:  # a smaller model's, much the same; the chain is drawn from it
            d = (1.1 * x + 0.5 * _normal(g, t, v)).to(dt)
            z = d.float() * s["draft_scale"]
            s["D"][i * t:(i + 1) * t] = d
            s["draft_lse"][i * t:(i + 1) * t] = torch.logsumexp(z.double(), 1).float()
            noise = -torch.log(-torch.log(_uniform(g, t, v).clamp(1e-7, 1 - 1e-7)))
            s["tokens"][i, 1:] = (z + noise).argmax(1)[:-1]
        elif t > 1:  # the likeliest tokens, as a smaller model sees them
            nodes = -(-(t - 1) // case["branch"])
            near = (x[:nodes] + 0.3 * _normal(g, nodes, v)).topk(case["branch"], dim=1).indices
            s["tokens"][i, 1:] = near.reshape(-1)[:t - 1]
    if not case["greedy"]:
        s["uniform"] = _uniform(g, b, t)
    at = torch.arange(t, device="cuda")
    anc = at == at.unsqueeze(1)  # [t, u]: u is t or one of its ancestors
    for u in range(1, t):
        anc[u] |= anc[(u - 1) // case["branch"]]
    s["ancestors"] = anc
    return s


def _cache(case, pages, g):
    """The caches of all layers, one behind the other."""
    shape = case["layers"], pages, case["heads"], case["page"], case["dim"]
    n = math.prod(shape)
    s = {}
    for c in "KV":
        bits = torch.randint(0, 2 ** 31 - 1, (-(-n // 4),), generator=g, device="cuda", dtype=torch.int32)
        bits = bits.view(torch.uint8)[:n].view(shape)
        if case["code"] == "e4m3":
            bits.bitwise_and_(0xf7)  # no NaN codes
        s[c + "C"] = bits.view(_CODE[case["code"]])
        s[c + "S"] = 0.01 + _uniform(g, *shape[:-1])
    return s


def _commit_inputs(case, g):
    b, t, page, branch = case["seqs"], case["width"], case["page"], case["branch"]
    context = (case["context"] * (0.25 + 0.75 * _uniform(g, b))).long()
    context[0] = case["context"]
    before = case["context"] // page + 1  # pages of a prompt that all share
    extra = -(-(page - 1 + t) // page)    # pages of a sequence's own
    s = _cache(case, before + b * extra, g)
    at = torch.arange(before + extra, device="cuda").expand(b, -1)
    first = (context // page).unsqueeze(1)
    mine = before + torch.arange(b, device="cuda").unsqueeze(1) * extra + (at - first)
    s["table"] = torch.where(at < first, at, torch.where(at < first + extra, mine, -1)).to(torch.int32).contiguous()
    s["context"] = context.to(torch.int32)
    s["path"] = torch.full((b, t), -1, dtype=torch.int32, device="cuda")
    s["path"][:, 0] = 0
    node, on = torch.zeros(b, dtype=torch.long, device="cuda"), torch.ones(b, dtype=torch.bool, device="cuda")
    for i in range(1, t):  # a way down the tree; the first sequence's is as long as it can be
        keep = _uniform(g, b) < 0.8
        keep[0] = True
        node = node * branch + 1 + (_uniform(g, b) * branch).long()
        node[0] = -(-node[0] // branch) * branch if branch > 1 and node[0] > 0 else node[0]
        on &= keep & (node < t)
        node = node.clamp(max=t)
        s["path"][:, i] = torch.where(on, node, -1).to(torch.int32)
    return s


def _fork_inputs(case, g):
    groups, beams, page = case["groups"], case["beams"], case["page"]
    b = groups * beams
    shared, grown = case["prompt"] // page, case["prompt"] % page + case["grown"]  # pages a group shares; a beam's own tokens
    extra = -(-grown // page)
    used = 1 + groups * shared + b * extra  # page 0 is nobody's
    pages = used + b * 2
    s = _cache(case, pages, g)
    width = shared + extra + 2
    row = torch.arange(b, device="cuda").unsqueeze(1)
    at = torch.arange(width, device="cuda").expand(b, -1)
    order = 1 + torch.randperm(pages - 1, generator=g, device="cuda")
    name = torch.where(at < shared, row // beams * shared + at, groups * shared + row * extra + at - shared)
    s["table"] = torch.where(at < shared + extra, order[name.clamp(max=pages - 2)], -1).to(torch.int32).contiguous()
    s["length"] = torch.full((b,), shared * page + grown, dtype=torch.int32, device="cuda")
    s["held"] = (torch.arange(pages, device="cuda") == 0).to(torch.int32)
    # every beam goes on from one of its group's, a few end, a few begin anew
    source = row[:, 0] // beams * beams + torch.randint(beams, (b,), generator=g, device="cuda")
    u = _uniform(g, b)
    want = torch.where(u < 0.05, 0, s["length"] + 1)
    s["source"] = torch.where((u > 0.95) & (b > 16), -1, source).to(torch.int32)
    s["want"] = torch.where(s["source"] < 0, page + 1, want).to(torch.int32)
    return s


def _adapter_inputs(case, g):
    m, n, k, r, count, dt = (case["tokens"], case["n"], case["k"], case["rank"], case["count"], _DT[case["dtype"]])
    s = {"X": _activations(g, m, k, dt), "Y": _normal(g, m, n).to(dt)}
    s["A"] = (_normal(g, count, r, k) / math.sqrt(k)).to(dt)
    s["B"] = (_normal(g, count, n, r) / math.sqrt(r)).to(dt)
    s["scales"] = 0.25 + _uniform(g, count)
    # requests lie behind one another, a token each of many or some tokens of a few; a few rows have no adapter
    long = max(1, m // (2 * count)) if m > 256 else 1
    pieces = -(-m // long)
    index = torch.randint(count, (pieces,), generator=g, device="cuda")
    index = torch.where(torch.arange(pieces, device="cuda") % 16 == 15, -1, index)
    s["index"] = index.repeat_interleave(long)[:m].to(torch.int32).contiguous()
    if case["op"] == "gradients":
        s["G"] = (1e-3 * _normal(g, m, n)).to(dt)
        s["Din"] = (1e-3 * _normal(g, m, k)).to(dt)
        a = s["index"].clamp(min=0).long()
        h = (s["X"].float() @ s["A"].float().view(count * r, k).T).view(m, count, r)
        s["H"] = torch.where(s["index"].unsqueeze(1) >= 0, h[torch.arange(m, device="cuda"), a], 0.0)
    return s


_INPUTS = {"verify": _verify_inputs, "commit": _commit_inputs, "fork": _fork_inputs, "adapters": _adapter_inputs,
           "gradients": _adapter_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, _generator(seed))
    s["case"] = case
    if own:
        s["call"], s["out"] = _PLANS[case["op"]](s)
    return s


# ---------------------------------------------------------------------------
# the library's calls: outputs, workspaces and prepared calls are what a program keeps
# ---------------------------------------------------------------------------

def _empty(*shape, dtype):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _space(size):
    return _empty(max(size, 256), dtype=torch.uint8)


def _layers(s):
    return [tuple(s[c][i] for c in ("KC", "VC", "KS", "VS")) for i in range(s["KC"].shape[0])]


def _plan_verify(s):
    from paper_2607_27042_amd import binding

    b, t = s["tokens"].shape
    out = (_empty(b, t, dtype=torch.int32), _empty(b, dtype=torch.int32), _empty(b, dtype=torch.int64),
           _empty(b, t, dtype=torch.float32))
    ws = _space(binding.gptq2d_tree_verify_workspace_size(b, t, s["X"].shape[1]))
    call = binding.gptq2d_tree_verify(s["X"], s["tokens"], s["parents"], None, s["scale"], s["uniform"], s["D"],
                                      s["draft_lse"], s["draft_scale"], *out, ws, prepare=True)
    return call, out


def _plan_commit(s):
    from paper_2607_27042_amd import binding

    call = binding.gptq2d_cache_commit(_layers(s), s["table"], s["context"], s["path"], prepare=True)
    return call, (s["KC"], s["VC"], s["KS"], s["VS"])


def _plan_fork(s):
    from paper_2607_27042_amd import binding

    b, pages, page = s["table"].shape[0], s["KC"].shape[1], s["KC"].shape[3]
    out, copies, left = (torch.empty_like(s["table"]), _empty(b, 3, dtype=torch.int32), _empty(1, dtype=torch.int32))
    ws = _space(binding.gptq2d_pages_update_workspace_size(b, pages))
    update = binding.gptq2d_pages_update(s["table"], s["length"], s["source"], s["want"], s["held"], pages, page, out,
                                         copies, left, ws, prepare=True)
    copy = binding.gptq2d_cache_copy(_layers(s), copies, prepare=True)
    return lambda: (update(), copy()), (out, copies, left, s["KC"], s["VC"], s["KS"], s["VS"])


def _plan_adapters(s):
    from paper_2607_27042_amd import binding

    (m, k), (count, n, r) = s["X"].shape, s["B"].shape
    groups = _empty(binding.gptq2d_adapter_groups_size(m, count), dtype=torch.int32)
    group = binding.gptq2d_adapter_groups(s["index"], count, groups, prepare=True)
    ws = _space(binding.gptq2d_adapters_workspace_size(m, n, k, r, count))
    out = torch.empty_like(s["Y"])
    call = binding.gptq2d_adapters(s["X"], s["A"], s["B"], s["scales"], groups, s["Y"], out, None, ws, prepare=True)
    return lambda: (group(), call()), (out,)


def _plan_gradients(s):
    from paper_2607_27042_amd import binding

    (m, k), (count, n, r) = s["X"].shape, s["B"].shape
    groups = _empty(binding.gptq2d_adapter_groups_size(m, count), dtype=torch.int32)
    group = binding.gptq2d_adapter_groups(s["index"], count, groups, prepare=True)
    ws = _space(binding.gptq2d_adapters_backward_workspace_size(m, n, k, r, count))
    out = (torch.empty_like(s["X"]), _empty(count, r, k, dtype=torch.float32), _empty(count, n, r, dtype=torch.float32))
    call = binding.gptq2d_adapters_backward(s["G"], s["X"], s["A"], s["B"], s["scales"], groups, s["H"], s["Din"], *out,
                                            ws, prepare=True)
    return lambda: (group(), call()), out


_PLANS = {"verify": _plan_verify, "commit": _plan_commit, "fork": _plan_fork, "adapters": _plan_adapters,
          "gradients": _plan_gradients}


def run(s):
    if own:
        s["call"]()
        return s["out"]
    return _PLAIN[s["case"]["op"]](s)


# ---------------------------------------------------------------------------
# the same in elementary torch operations, 32 bits (64 where a border decides)
# ---------------------------------------------------------------------------

def _plain_verify(s):
    x, tok, parents, scale, u = s["X"], s["tokens"], s["parents"].long(), s["scale"], s["uniform"]
    (b, t), v = tok.shape, x.shape[1]
    top, best = x.max(1)
    if u is None:  # the lowest of the largest logits
        best = torch.where(x == top.unsqueeze(1), torch.arange(v, device="cuda"), v).amin(1)
    total = torch.exp((x.float() - top.float().unsqueeze(1)) * scale).sum(1, dtype=torch.float64)
    row = torch.arange(b, device="cuda").unsqueeze(1) * t + parents.clamp(min=0)  # of each token's parent
    z = (x[row, tok].double() - top[row].double()) * scale
    p = torch.exp(z) / total[row]
    at = torch.arange(t, device="cuda")
    there = at > 0
    earlier = (parents.unsqueeze(2) == parents.unsqueeze(1)) & (at < at.unsqueeze(1)) & there  # [b, t, u]: a sibling before t
    if u is None:
        ok = best[row] == tok
    elif s["D"] is not None:
        q = torch.exp(s["D"][row, tok].double() * s["draft_scale"] - s["draft_lse"][row].double())
        ok = u.double() * q < p
    else:
        again = (earlier & (tok.unsqueeze(2) == tok.unsqueeze(1))).any(2)
        p = torch.where(again, 0.0, p)
        ok = u.double() * (1.0 - (earlier * p.unsqueeze(1)).sum(2)) < p
    ok &= ~(earlier & ok.unsqueeze(1)).any(2)  # the first of siblings
    on = (ok.unsqueeze(1) | ~s["ancestors"] | ~there).all(2)
    path = torch.sort(torch.where(on, at, t), 1).values
    path = torch.where(path < t, path, -1)
    last = torch.where(on, at, 0).amax(1)
    end = torch.arange(b, device="cuda") * t + last
    if u is None:
        chosen = best[end]
    else:
        e = torch.exp((x[end].double() - top[end].double().unsqueeze(1)) * scale)
        left = e / e.sum(1, keepdim=True)
        if s["D"] is not None:
            q = torch.exp(s["D"][end].double() * s["draft_scale"] - s["draft_lse"][end].double().unsqueeze(1))
            less = (left - q).clamp(min=0.0)
            left = torch.where(((last < t - 1) & (less.sum(1) > 0)).unsqueeze(1), less, left)
        else:
            child = (parents == last.unsqueeze(1)) & there
            keep = torch.ones(b, v + 1, dtype=torch.float64, device="cuda").scatter(1, torch.where(child, tok, v), 0.0)
            less = left * keep[:, :v]
            left = torch.where((less.sum(1) > 0).unsqueeze(1), less, left)
        sums = left.cumsum(1)
        chosen = (sums <= u[:, :1].double() * sums[:, -1:]).sum(1)
    logprob = z - torch.log(total[row])
    first = (x[end, chosen].double() - top[end].double()) * scale - torch.log(total[end])
    logprob = torch.where(there, logprob, first.unsqueeze(1)).float()
    return path.to(torch.int32), on.sum(1).to(torch.int32), chosen, logprob


def _plain_commit(s):
    path, page = s["path"].long(), s["case"]["page"]
    to = s["context"].long().unsqueeze(1) + torch.arange(path.shape[1], device="cuda")
    at = torch.where(path >= 0, s["context"].long().unsqueeze(1) + path, to)  # past the path: each stays
    table = s["table"].long()
    fp, fo = table.gather(1, at // page).flatten(), (at % page).flatten()
    tp, to = table.gather(1, to // page).flatten(), (to % page).flatten()
    kc, vc = s["KC"].view(torch.uint8), s["VC"].view(torch.uint8)
    kc[:, tp, :, to] = kc[:, fp, :, fo]
    vc[:, tp, :, to] = vc[:, fp, :, fo]
    s["KS"][:, tp, :, to] = s["KS"][:, fp, :, fo]
    s["VS"][:, tp, :, to] = s["VS"][:, fp, :, fo]
    return s["KC"], s["VC"], s["KS"], s["VS"]


def _plain_fork(s):
    table, page = s["table"].long(), s["case"]["page"]
    b, width = table.shape
    pages = s["KC"].shape[1]
    source, want = s["source"].long(), s["want"].long()
    kept = torch.where(source >= 0, torch.minimum(s["length"].long()[source.clamp(min=0)], want), 0)
    at = torch.arange(width, device="cuda")
    old = table[source.clamp(min=0)]
    whole, part = (kept // page).unsqueeze(1), (kept % page).unsqueeze(1)
    full = at < whole
    ends = (at == whole) & (part > 0)
    row = torch.arange(b, device="cuda").unsqueeze(1)
    # of each page: 0 if a row holds it whole, else the first row (plus 1) that it ends in, else b + 1
    mark = torch.where(full, 0, torch.where(ends, row + 1, b + 1))
    by = torch.full((pages,), b + 1, device="cuda").scatter_reduce(0, old.clamp(min=0).flatten(), mark.flatten(), "amin")
    held = s["held"] != 0
    free = (by == b + 1) & ~held
    copied = ends & ((by[old.clamp(min=0)] != row + 1) | held[old.clamp(min=0)])
    fresh = copied | ((at >= whole + (part > 0)) & (at < -(-want.unsqueeze(1) // page)))
    order = torch.argsort((~free).to(torch.int32), stable=True)  # free pages first
    nth = fresh.flatten().cumsum(0).view(b, width) - 1
    new = torch.where(nth < free.sum(), order[nth.clamp(0, pages - 1)], -1)
    out = torch.where(fresh, new, torch.where(full | ends, old, -1))
    has = copied.any(1)
    src = torch.where(copied, old, -1).amax(1)
    dst = torch.where(copied, out, -1).amax(1)
    copies = torch.stack([src, dst, torch.where(has, part[:, 0], 0)], 1)
    go = dst >= 0
    src, dst = torch.where(go, src, 0), torch.where(go, dst, 0)  # page 0 onto itself for the others
    first = torch.arange(page, device="cuda") < part
    kc, vc = s["KC"].view(torch.uint8), s["VC"].view(torch.uint8)
    kc[:, dst] = torch.where(first[:, None, :, None], kc[:, src], kc[:, dst])
    vc[:, dst] = torch.where(first[:, None, :, None], vc[:, src], vc[:, dst])
    s["KS"][:, dst] = torch.where(first[:, None], s["KS"][:, src], s["KS"][:, dst])
    s["VS"][:, dst] = torch.where(first[:, None], s["VS"][:, src], s["VS"][:, dst])
    left = free.sum() - fresh.sum()
    return (out.to(torch.int32), copies.to(torch.int32), left.to(torch.int32).view(1), s["KC"], s["VC"], s["KS"], s["VS"])


def _of_adapter(s, x, w):
    """x times the weights of all adapters (count R rows), with zeros outside the row's own."""
    count, r = s["A"].shape[:2]
    own_ = torch.arange(count, device="cuda").repeat_interleave(r) == s["index"].unsqueeze(1)
    return torch.where(own_, x.float() @ w.T, 0.0)


def _plain_adapters(s):
    count, r, k = s["A"].shape
    a = s["A"].float().view(count * r, k)
    b = s["B"].float().transpose(1, 2).reshape(count * r, -1)
    h = _of_adapter(s, s["X"], a)
    return ((s["Y"].float() + (h * s["scales"].repeat_interleave(r)) @ b).to(s["X"].dtype),)


def _plain_gradients(s):
    count, r, k = s["A"].shape
    n = s["B"].shape[1]
    a = s["A"].float().view(count * r, k)
    b = s["B"].float().transpose(1, 2).reshape(count * r, n)
    scales = s["scales"].repeat_interleave(r)
    mine = torch.arange(count, device="cuda").repeat_interleave(r) == s["index"].unsqueeze(1)
    h = torch.where(mine, s["H"].repeat(1, count), 0.0) * scales
    p = _of_adapter(s, s["G"], b) * scales
    dx = (s["Din"].float() + p @ a).to(s["X"].dtype)
    da = (p.T @ s["X"].float()).view(count, r, k)
    db = (h.T @ s["G"].float()).view(count, r, n).transpose(1, 2).contiguous()
    return dx, da, db


_PLAIN = {"verify": _plain_verify, "commit": _plain_commit, "fork": _plain_fork, "adapters": _plain_adapters,
          "gradients": _plain_gradients}


# ---------------------------------------------------------------------------
# the same from the definitions, 64 bits
# ---------------------------------------------------------------------------

def _exact_verify(case, s):
    """One token after the other, as the scan is defined."""
    b, t, v = case["seqs"], case["width"], case["vocab"]
    path = torch.full((b, t), -1, dtype=torch.int32)
    count, chosen = torch.zeros(b, dtype=torch.int32), torch.zeros(b, dtype=torch.int64)
    logprob = torch.zeros(b, t, dtype=torch.float64)
    for i in range(b):
        lp = torch.log_softmax(s["X"][i * t:(i + 1) * t].double() * s["scale"], 1)
        tok, parent = s["tokens"][i].tolist(), s["parents"][i].tolist()
        u = [0.0] * t if case["greedy"] else s["uniform"][i].double().tolist()
        if case["draft"]:
            q = torch.exp(s["D"][i * t:(i + 1) * t].double() * s["draft_scale"]
                          - s["draft_lse"][i * t:(i + 1) * t].double().unsqueeze(1))
        given = lp[parent[1:], tok[1:]].tolist() if t > 1 else []
        proposed = q[parent[1:], tok[1:]].tolist() if t > 1 and case["draft"] else []
        likely = torch.sort(lp, dim=1, descending=True, stable=True).indices[:, 0].tolist() if case["greedy"] else []
        cur, way, gone = 0, [0], []
        for j in range(1, t):
            logprob[i, j] = given[j - 1]
            if parent[j] != cur:
                continue
            p = 0.0 if tok[j] in gone else math.exp(given[j - 1])
            if case["greedy"]:
                taken = likely[cur] == tok[j]
            elif case["draft"]:
                taken = u[j] * proposed[j - 1] < p
            else:
                taken = u[j] * (1.0 - sum(math.exp(float(lp[cur, w])) for w in gone)) < p
            if taken:
                cur, gone = j, []
                way.append(j)
            elif tok[j] not in gone:
                gone.append(tok[j])
        path[i, :len(way)] = torch.tensor(way, dtype=torch.int32)
        count[i] = len(way)
        if case["greedy"]:
            chosen[i] = likely[cur]
        else:
            r = lp[cur].exp()
            less = r.clone()
            if case["draft"]:
                less = torch.clamp(r - q[cur], min=0.0) if gone else r
            elif gone:
                less[gone] = 0.0
            r = less if float(less.sum()) > 0 else r
            sums = torch.cumsum(r, 0)
            chosen[i] = int(torch.searchsorted(sums, u[0] * sums[-1], right=True))
        logprob[i, 0] = lp[cur, chosen[i]]
    return path, count, chosen, logprob


def _exact_commit(case, s):
    page = case["page"]
    table, path, context = s["table"].tolist(), s["path"].tolist(), s["context"].tolist()
    moves = [(table[i][(context[i] + p) // page], (context[i] + p) % page, table[i][(context[i] + j) // page],
              (context[i] + j) % page) for i in range(case["seqs"]) for j, p in enumerate(path[i]) if p >= 0]
    a, c, d, e = (torch.tensor(x, device="cuda") for x in zip(*moves))
    out = []
    for name in ("KC", "VC", "KS", "VS"):
        new = s[name].clone().view(torch.uint8) if name[1] == "C" else s[name].double()
        new.transpose(2, 3)[:, d, e] = new.transpose(2, 3)[:, a, c].clone()
        out.append(new.view(s[name].dtype) if name[1] == "C" else new)
    return tuple(x if x.dtype == torch.int8 else x.float() if x.dtype == _CODE["e4m3"] else x for x in out)


def _exact_fork(case, s):
    """Row by row; of whole numbers and moved bytes only the scales are wanted in 64 bits."""
    page = case["page"]
    table, length, source, want = (s[k].tolist() for k in ("table", "length", "source", "want"))
    held = s["held"].tolist()
    width, rows = len(table[0]), len(source)
    kept = [min(length[r], w) if r >= 0 else 0 for r, w in zip(source, want)]
    whole = {table[r][i] for r, k in zip(source, kept) for i in range(k // page)}
    ends = {}
    for i in range(rows):
        if kept[i] % page:
            ends.setdefault(table[source[i]][kept[i] // page], i)
    free = [p for p in range(len(held)) if not held[p] and p not in whole and p not in ends]
    ks, vs = s["KS"].double(), s["VS"].double()
    out, copies, lacking = [], [], 0
    for i in range(rows):
        new, copy = [], [-1, -1, 0]
        for j in range(width):
            p = table[source[i]][j] if source[i] >= 0 else -1
            if j < kept[i] // page:
                new.append(p)
            elif j * page < kept[i] and ends[p] == i and p not in whole and not held[p]:
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
    for a, c, n in copies:
        if c >= 0:
            ks[:, c, :, :n] = ks[:, a, :, :n]
            vs[:, c, :, :n] = vs[:, a, :, :n]
    return (torch.tensor(out, dtype=torch.int32), torch.tensor(copies, dtype=torch.int32),
            torch.tensor([len(free) - lacking], dtype=torch.int32), None, None, ks, vs)


def exact(case, seed):
    s = _INPUTS[case["op"]](case, _generator(seed))
    if case["op"] == "verify":
        return _exact_verify(case, s)
    if case["op"] == "commit":
        return _exact_commit(case, s)
    if case["op"] == "fork":
        return _exact_fork(case, s)
    # adapter by adapter
    x, out = s["X"].double(), s["Y"].double()
    da, db = torch.zeros(s["A"].shape, dtype=torch.float64), torch.zeros(s["B"].shape, dtype=torch.float64)
    if case["op"] == "gradients":
        g, dx = s["G"].double(), s["Din"].double()
    for a in range(case["count"]):
        at = (s["index"] == a).nonzero()[:, 0]
        wa, wb, c = s["A"][a].double(), s["B"][a].double(), float(s["scales"][a])
        if case["op"] == "adapters":
            out[at] += torch.matmul(torch.matmul(x[at], wa.T), wb.T) * c
        else:
            p = torch.matmul(g[at], wb) * c
            dx[at] += torch.matmul(p, wa)
            da[a] = torch.matmul(p.T, x[at]).cpu()
            db[a] = torch.matmul(g[at].T, s["H"][at].double()).cpu() * c
    return (out,) if case["op"] == "adapters" else (dx, da, db)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "verify":
        # the rows of tokens that others follow (their log probabilities are wanted), and of
        # drafted chains one row of the draft's logits
        rows = max(1, -(-(case["width"] - 1) // case["branch"])) + (1 if case["draft"] and case["width"] > 1 else 0)
        cells = float(case["seqs"]) * rows * case["vocab"]
        return {"bytes": _ES[case["dtype"]] * cells + 24.0 * case["seqs"] * case["width"], "flops": 4 * cells}
    if case["op"] == "commit":
        # the tokens of a way down the tree with four steps in five taken, but for a first one in its place
        depth = int(math.log(case["width"] * (case["branch"] - 1) + 1, case["branch"]))
        moved = case["seqs"] * (sum(0.8 ** i for i in range(1, depth + 1)) - 0.8 / case["branch"])
        return {"bytes": 4.0 * moved * case["layers"] * case["heads"] * (case["dim"] + 4) + 4.0 * case["seqs"] * case["width"],
                "flops": 0}
    if case["op"] == "fork":
        rows = case["groups"] * case["beams"]
        width = case["prompt"] // case["page"] + -(-(case["prompt"] % case["page"] + case["grown"]) // case["page"]) + 2
        part = (case["prompt"] + case["grown"]) % case["page"]
        copied = rows * 0.3 * part * case["layers"] * case["heads"] if case["beams"] > 1 else 0.0
        return {"bytes": 8.0 * rows * width + 4.0 * copied * (case["dim"] + 4), "flops": 0}
    es, m, n, k, r = _ES[case["dtype"]], float(case["tokens"]), case["n"], case["k"], case["rank"]
    used = min(case["count"], m)
    if case["op"] == "adapters":
        return {"bytes": es * m * (k + 2 * n) + es * used * r * (n + k) + 4 * m, "flops": 2 * m * r * (n + k)}
    return {"bytes": es * m * (n + 3 * k) + 4 * m * (r + 1) + es * used * r * (n + k) + 4 * case["count"] * r * (n + k),
            "flops": 4 * m * r * (n + k)}
